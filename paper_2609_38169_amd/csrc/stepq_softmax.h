// Shared by the attention kernels: a running softmax, and the join of the parts that a row's keys were split into.
#pragma once

#include "stepq_mma.h"
#include "stepq_plan.h"

namespace stepq {
namespace {                  // kernels of each source's own

__device__ __forceinline__ int fdiv(int n, FastDiv d)
{
    const uint32_t u = static_cast<uint32_t>(n);
    return static_cast<int>((__umulhi(u, d.mul) + u) >> d.shift);
}

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float swap_max16(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float swap_max32(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float swap_add16(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float swap_add32(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// The scale goes into the exponent, one fma from a score: rounded before the maximum is taken off, scores of 4096
// and more would lose what tells them apart.  That needs it positive (the maximum is taken before): its sign goes
// into the queries, and 0 makes them 0.
__device__ __forceinline__ float scale_of(float scale) { return scale == 0.0f ? 1.0f : fabsf(scale); }
__device__ __forceinline__ u32x4 with_sign(u32x4 q, float scale, uint32_t signs)
{
    return scale > 0.0f ? q : scale == 0.0f ? u32x4{} : q ^ signs;
}

// A running softmax: maximum and sum of what was seen; next() returns the
// factor on everything so far when scores of maximum m join.
struct Running {
    float m = -INFINITY, l = 0.0f, base = 0.0f;
    __device__ __forceinline__ float next(float top)
    {
        const float to = fmaxf(m, top), b = to == -INFINITY ? 0.0f : to, f = __builtin_amdgcn_exp2f(m - b);
        m = to, base = b, l *= f;
        return f;
    }
};

struct JoinArgs {
    const float2 *ml;        // [parts][rows]: a part's maximum (in powers of two) and sum
    const float *acc;        // [parts][rows][D]: its unnormalised output
    void *o;
    float *lse;              // NULL: not wanted
    size_t rows;
    int32_t parts;
    // lengths not NULL: rows b Hq .. + Hq - 1 have as many parts as lengths[b] tokens (at most `most`) take, `chunk` each;
    // of one part or none the row is there already
    const int32_t *lengths;
    int32_t Hq, most, chunk;
};

// The parts of each row joined: W waves per row take parts in turn, a few at a
// time so that their loads overlap.  Few rows (up to 1024): 4 waves, as latency
// counts; a request over 16384 tokens, 16 heads of 256 in 65 parts, in all: 37 us
// with one load after the other in a wave, 20 so.  More: a wave each, bound by
// the parts' bytes; 9 x 8192 rows of 256 (75 MB) in 14 us, 3 more with 4 waves.
// Whole calls, one wave / 4, us, 64 dimensions over 1024 tokens: 32 rows 8.6 / 7.3,
// 1024 13.5 / 12.1, 2048 17.9 / 17.1, 8192 48 / 50; 256 over 4096: 128 19.3 / 17.5,
// 1024 51.5 / 50.7, 2048 50.5 / 53.2, 16384 178 / 185.
// (Joined in attn_rows_kernel instead, which has few waves to wait with, 512
// requests take 225 us in all, not 208.)
template <typename T, int D, int W>
__global__ __launch_bounds__(256) void attn_join_kernel(JoinArgs a)
{
    constexpr int E = D / 64, U = 4;
    using Piece = __attribute__((ext_vector_type(E))) float;
    __shared__ alignas(16) float sum[4][D];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = w % W, lane = threadIdx.x & 63;
    const size_t total = a.rows, row = static_cast<size_t>(blockIdx.x) * (4 / W) + w / W;
    if (W == 1 && row >= total) return;
    int parts = a.parts;
    if (a.lengths) {
        const int len = min(a.lengths[row / a.Hq], a.most);
        if (len <= a.chunk) return;
        parts = (len + a.chunk - 1) / a.chunk;
    }
    const auto stats = [&](int c) { return c + lane < parts ? a.ml[(c + lane) * total + row] : make_float2(-INFINITY, 0.0f); };
    const float2 first = stats(0);
    float top = first.x;
    for (int c = 64; c < parts; c += 64) top = fmaxf(top, stats(c).x);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
    const float base = top == -INFINITY ? 0.0f : top;
    Piece y = {};
    float z = 0.0f;
    for (int c = 0; c < parts; c += 64) {
        const float2 ml = c == 0 ? first : stats(c);
        const float f = __builtin_amdgcn_exp2f(ml.x - base);
        z = fmaf(ml.y, f, z);
        const int n = min(64, parts - c);
        for (int p = wave; p < n; p += W * U) {
            Piece x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                x[u] = reinterpret_cast<const Piece *>(a.acc + ((c + min(p + W * u, n - 1)) * total + row) * D)[lane];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (p + W * u < n) y += x[u] * __shfl(f, p + W * u);
        }
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) z += __shfl_xor(z, x);
    T *o = static_cast<T *>(a.o) + row * D;
    if constexpr (W == 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) o[lane * E + e] = narrow<T>(z == 0.0f ? 0.0f : y[e] / z);
    } else {
        *reinterpret_cast<Piece *>(&sum[w][lane * E]) = y;
        __syncthreads();
        const int d = threadIdx.x;
        if (d < D) o[d] = narrow<T>(z == 0.0f ? 0.0f : (sum[0][d] + sum[1][d] + sum[2][d] + sum[3][d]) / z);
    }
    if (wave == 0 && lane == 0 && a.lse) a.lse[row] = z == 0.0f ? -INFINITY : (base + log2f(z)) * kLn2;
}

template <typename T, int D>
void join_parts(const JoinArgs &a, hipStream_t st)
{
    const unsigned rows = static_cast<unsigned>(a.rows);
    if (rows <= 1024) attn_join_kernel<T, D, 4><<<dim3(rows), 256, 0, st>>>(a);
    else attn_join_kernel<T, D, 1><<<dim3((rows + 3) / 4), 256, 0, st>>>(a);
}

}  // namespace
}  // namespace stepq
