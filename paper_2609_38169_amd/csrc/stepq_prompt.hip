// Prompts: packed sequences through the gated recurrences of stepq_rule.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "stepq_mma.h"

namespace stepq {
namespace {

struct PromptArgs {
    const int32_t *cu;       // NULL: one sequence of all tokens
    const void *q, *k, *v;
    Gate alpha, beta;        // beta.p NULL: 1
    void *o;
    const float *state_in;   // NULL: zeros
    const int32_t *in_ids;
    float *state_out;
    int64_t sq, sk, sv, so;  // token strides
    int32_t T, n_seq, Hv, Hqk, dk, dv, n_in;
};

// ---------------------------------------------------------------------------
// Chunks of 64 tokens.  With G_i the product of the gates from the chunk's
// first token to token i, D_ij = G_i / G_j (i >= j, else 0), S the state
// before the chunk, and V, K, Q, O the chunk's rows:
//   R = V - G (K S)            (Delta; R = V for the decay rule)
//   U = T' R,  T' = (I + M)^-1 diag(beta),  M = strict lower part of beta_i D_ij (k_i . k_j)
//   O = G (Q S) + P U,  P = D (Q K^T)
//   S <- G_last S + K^T (w U),  w_j = G_last / G_j
// (the decay rule has U = beta V).
// Operands on the matrix cores are bfloat16 planes of the values, three (24 bits,
// the value itself) each but for bfloat16 keys and queries, which are one.  Their
// exponents are fp32's: tokens of very different size share a chunk, and with
// two binary16 planes under a power of two for a tile or a column (22 bits; 32
// sequences 485 us, not 533; 24 fp32 ones 78, not 98) a token 2^28 times the others
// left nothing of those before it.
// T' and the gates' products depend on no state: a first launch forms them
// for every chunk at once; the second walks each sequence's chunks in order.
constexpr int kC = 64;

// Per (chunk, head) of the workspace: the gates' products, then for the Delta
// rule T', lane by lane as operand A wants it.
struct ChunkGates {
    double lg[kC];           // log2 G_i: differences of them stay exact where G itself is 0 or tiny
    float g[kC], w[kC], b[kC];
    int32_t bad;             // Delta: first token whose key, gate or row of T' is not finite, or whose alpha is below 0 (kC: none)
    int32_t pad[31];
};
static_assert(sizeof(ChunkGates) == 1408, "record size");
constexpr size_t kTBytes = 6 * 2048;
constexpr int kGateWords = 5 * kC + 1;   // lg, g, w, b, bad

struct ChunkArgs {
    PromptArgs p;
    uint8_t *ws;
    size_t record;           // bytes per (chunk, head)
    int32_t slots;           // chunk slots: sequence s owns those from cu[s] / 64 + s on
    int32_t seg;             // chunks per segment; 0: sequences are not cut
    int32_t seg_slots;       // segment slots, numbered as the chunks' are, with 64 seg tokens each
    float *segs;             // per (segment, head): SegmentHead, B or the state after it [dk][dv], A [DKP][DKP] (Delta)
    size_t seg_floats;
    int32_t near;            // 64 tokens of q, k and v lie within 2^32 bytes
    int4 *order;             // [n_seq] sequences, longest first: number, bounds, initial state; NULL: they are walked in their own order
};

__device__ __forceinline__ int2 seq_bounds(const PromptArgs &a, int s)
{
    if (!a.cu) return make_int2(0, a.T);
    const int from = min(max(a.cu[s], 0), a.T);
    return make_int2(from, min(max(a.cu[s + 1], from), a.T));
}

// The index of the state sequence s starts from; -1: zeros.
__device__ __forceinline__ int initial_index(const PromptArgs &a, int s)
{
    const int src = a.state_in ? (a.in_ids ? a.in_ids[s] : s) : -1;
    return src < a.n_in ? src : -1;
}

// First slot of sequence s where a slot holds `unit` tokens.
__device__ __forceinline__ int first_slot(const PromptArgs &a, int s, int unit = kC)
{
    return a.cu ? min(max(a.cu[s], 0), a.T) / unit + s : 0;
}

// The sequence that owns a chunk slot: the last one whose first slot is at most
// x, found by the wave's 64 lanes at a time.
__device__ __forceinline__ int owner(const PromptArgs &a, int x, int lane, int unit = kC)
{
    int lo = 0, n = a.n_seq;            // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) / 64, at = lo + lane * step;
        const bool le = at < lo + n && first_slot(a, at, unit) <= x;
        const uint64_t yes = __ballot(le);
        const int k = yes ? 63 - __clzll(yes) : 0;
        const int end = lo + n;
        lo += k * step;
        n = min(step, end - lo);
    }
    return lo;
}

template <typename T>
struct Act;
template <>
struct Act<bf16_t> {
    static constexpr int planes = 1;
    u32x4 x;
};
template <>
struct Act<float> {
    static constexpr int planes = 3;
    f32x4 x[2];
};

// Row r of rows `stride` elements apart: one 64-bit multiply-add per lane, so
// that no row's address is kept in scalar registers.
template <typename T>
__device__ __forceinline__ T *row_of(T *base, uint32_t r, int64_t stride)
{
    const uint64_t at = static_cast<uint64_t>(r) * static_cast<uint32_t>(stride * sizeof(T));
    using B = std::conditional_t<std::is_const_v<T>, const uint8_t, uint8_t>;
    return reinterpret_cast<T *>(reinterpret_cast<B *>(base) + at);
}

// 8 elements from an address that is a multiple of ALIGN bytes (the hardware
// takes 16-byte loads at any).
template <int ALIGN, typename T>
__device__ __forceinline__ Act<T> load_wide(const T *p)
{
    struct __attribute__((packed, aligned(ALIGN))) Raw {
        u32x4 x;
    };
    const Raw *r = reinterpret_cast<const Raw *>(p);
    if constexpr (sizeof(T) == 2) return Act<T>{r[0].x};
    else return Act<T>{{__builtin_bit_cast(f32x4, r[0].x), __builtin_bit_cast(f32x4, r[1].x)}};
}

// 8 elements of a row of n valid ones from element i on; elements past n are
// anything until settle() (nothing here waits for the data).  VEC: everything is
// 16-byte aligned and n a multiple of 8.
template <bool VEC, typename T>
__device__ __forceinline__ Act<T> load8(const T *row, int i, int n)
{
    // past n, the first elements are read (no branch around the load)
    if constexpr (VEC) return load_wide<16>(row + (i < n ? i : 0));
    if (n >= 8) return load_wide<sizeof(T)>(row + min(i, n - 8));
    Act<T> r = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const T x = row[min(e, n - 1)];
        if constexpr (sizeof(T) == 2) r.x[e / 2] |= static_cast<uint32_t>(x) << (16 * (e % 2));
        else r.x[e / 4][e % 4] = x;
    }
    return r;
}

// What load8<false> gave for elements i .. i + 7, in place, zeros past n: the
// unit that n ends in was read from n - 8 on.
template <typename T>
__device__ __forceinline__ Act<T> settle(const Act<T> &v, int i, int n)
{
    const bool tail = i < n && i + 8 > n;
    const int shift = n >= 8 ? (8 - n % 8) % 8 : 0;       // the same for all lanes
    if constexpr (sizeof(T) == 2) {
        u32x4 x = v.x;
        if (shift & 4) x = u32x4{x[2], x[3], 0u, 0u};
        if (shift & 2) x = u32x4{x[1], x[2], x[3], 0u};
        if (shift & 1)
            x = u32x4{__builtin_amdgcn_alignbit(x[1], x[0], 16), __builtin_amdgcn_alignbit(x[2], x[1], 16),
                      __builtin_amdgcn_alignbit(x[3], x[2], 16), x[3] >> 16};
        Act<T> r;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t keep = (i + 2 * e < n ? 0xffffu : 0u) | (i + 2 * e + 1 < n ? 0xffff0000u : 0u);
            r.x[e] = (tail ? x[e] : v.x[e]) & keep;
        }
        return r;
    } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v.x[e / 4][e % 4];
#pragma unroll
        for (int b = 4; b > 0; b >>= 1)
            if (shift & b)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = e + b < 8 ? x[e + b] : 0.0f;
        Act<T> r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.x[e / 4][e % 4] = i + e < n ? (tail ? x[e] : v.x[e / 4][e % 4]) : 0.0f;
        return r;
    }
}

template <typename T>
__device__ __forceinline__ Act<T> load_at(const T *base, uint32_t at)
{
    return load_wide<16>(reinterpret_cast<const T *>(reinterpret_cast<const uint8_t *>(base) + at));
}

// A thread's share of a tile of 64 rows of C8 8-element units, N threads: unit c8 of the rows row + step u.
template <int C8, int N>
struct Share {
    int row, c8;
    __device__ __forceinline__ Share(int tid) : row(tid / C8), c8(tid % C8) {}
    static constexpr int step = N / C8, units = kC / step;

    // unit u of the `len` rows from `base` on; past the last row that one is read (valid() tells)
    template <bool VEC, typename T>
    __device__ __forceinline__ Act<T> load(const T *base, int64_t stride, int u, int n, int len) const
    {
        int r = row;
        asm volatile("" : "+v"(r));          // the offset is formed at the load, not kept in registers from chunk to chunk
        return load8<VEC>(row_of(base, min(r + step * u, len - 1), stride), 8 * c8, n);
    }
    __device__ __forceinline__ Share again() const
    {
        Share s = *this;
        asm volatile("" : "+v"(s.row));
        return s;
    }
    __device__ __forceinline__ bool valid(int u, int n, int len) const { return row + step * u < len && 8 * c8 < n; }
};

// Four outputs of a lane in their type.
template <typename T>
struct Out4;
template <>
struct Out4<float> {
    f32x4 x;
    __device__ __forceinline__ void set(const f32x4 &v) { x = v; }
    __device__ __forceinline__ float at(int r) const { return x[r]; }
};
template <>
struct Out4<bf16_t> {
    uint32_t x[2];
    __device__ __forceinline__ void set(const f32x4 &v)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            x[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2));
    }
    __device__ __forceinline__ bf16_t at(int r) const { return static_cast<bf16_t>(r % 2 ? x[r / 2] >> 16 : x[r / 2]); }
};

template <typename T>
__device__ __forceinline__ Act<T> zero_unless(bool keep, const Act<T> &v)
{
    Act<T> r;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.x[i] = keep ? v.x[i] : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.x[i / 4][i % 4] = keep ? v.x[i / 4][i % 4] : 0.0f;
    }
    return r;
}

// |x|'s largest of a thread's N units, as the bits of a float
template <int N>
__device__ __forceinline__ uint32_t max_of(const Act<bf16_t> (&v)[N])
{
    using u16x2 = __attribute__((ext_vector_type(2))) uint16_t;
    u16x2 m = {};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i].x[e] & 0x7fff7fffu));
    return static_cast<uint32_t>(max(m[0], m[1])) << 16;
}
template <int N>
__device__ __forceinline__ uint32_t max_of(const Act<float> (&v)[N])
{
    uint32_t m = 0;                          // as integers, in which a NaN is above all
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(fabsf(v[i].x[e / 4][e % 4])));
    return m;
}
constexpr uint32_t kInfBits = 0x7f800000u;
template <typename T>
__device__ __forceinline__ bool all_finite(const Act<T> &v)
{
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float a;
        if constexpr (sizeof(T) == 2) a = i % 2 ? upper_bf16(v.x[i / 2]) : lower_bf16(v.x[i / 2]);
        else a = v.x[i / 4][i % 4];
        ok &= fabsf(a) < INFINITY;
    }
    return ok;
}
// A tile of keys or queries: 64 rows of DKP elements in bfloat16 planes.  Their
// summation slots are the elements in order (operands are 16-byte reads), so
// the state, their partner, keeps element 32 kb + 8 g + 4 h + r of a column in
// row 4 g + r of its block 2 kb + h.
__device__ __forceinline__ int state_row(int block, int row)
{
    return 32 * (block >> 1) + 8 * (row >> 2) + 4 * (block & 1) + (row & 3);
}

template <typename T, int DKP>
struct RowTile {
    static constexpr int NA = Act<T>::planes, RB = DKP * 2;
    alignas(16) uint8_t b[NA][kC * RB];

    __device__ __forceinline__ void put(int row, int c8, const Act<T> &v)
    {
        uint8_t *at = &b[0][row * RB + ((c8 ^ swizzle<RB>(row)) * 16)];
        if constexpr (NA == 1) {
            *reinterpret_cast<u32x4 *>(at) = v.x;
        } else {
            bf16x8 p[NA];
            split(v.x[0], v.x[1], p);
#pragma unroll
            for (int n = 0; n < NA; ++n) *reinterpret_cast<bf16x8 *>(at + n * kC * RB) = p[n];
        }
    }

    // operand: row 16 rt + n, elements 32 kb .. 32 kb + 31
    __device__ __forceinline__ void rows(int rt, int kb, int g, int n, bf16x8 (&a)[NA]) const
    {
        const int row = 16 * rt + n;
#pragma unroll
        for (int i = 0; i < NA; ++i)
            a[i] = *reinterpret_cast<const bf16x8 *>(&b[i][row * RB + (((4 * kb + g) ^ swizzle<RB>(n)) * 16)]);
    }

    // operand A of the transposed tile: tokens 32 kb .. 32 kb + 31 of state row state_row(dt, n)
    __device__ __forceinline__ void columns(int dt, int kb, int g, int n, bf16x8 (&a)[NA]) const
    {
        const int f = swizzle<RB>(4 * g + (n >> 2));
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            u32x4 w;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = 32 * kb + 16 * h + 4 * g + (n >> 2), slot = 4 * (dt / 2) + (n & 3);
                const u32x2 x = read_columns(&b[i][row * RB + ((slot ^ f) * 16) + 8 * (dt & 1)]);
                w[2 * h] = x[0], w[2 * h + 1] = x[1];
            }
            a[i] = __builtin_bit_cast(bf16x8, w);
        }
    }
};

// A tile of bfloat16 values: 64 rows of W columns.
template <int W>
struct ValueTile {
    static constexpr int RB = 2 * W;
    alignas(16) uint8_t b[kC * RB];

    __device__ __forceinline__ void put(int row, int c8, const Act<bf16_t> &v)
    {
        *reinterpret_cast<u32x4 *>(&b[row * RB + ((c8 ^ swizzle<RB>(row)) * 16)]) = v.x;
    }

    // rows 16 tt + 4 g .. + 3 of column col + n (col a multiple of 16)
    __device__ __forceinline__ f32x4 four(int tt, int col, int g, int n) const
    {
        const int row = 16 * tt + 4 * g + (n >> 2), slot = col / 8 + ((n & 3) >> 1);
        const u32x2 w = read_columns(&b[row * RB + ((slot ^ swizzle<RB>(row)) * 16) + 8 * (n & 1)]);
        return f32x4{lower_bf16(w[0]), upper_bf16(w[0]), lower_bf16(w[1]), upper_bf16(w[1])};
    }
};

// Lower triangles of 64x64 as operand A: blocks 0 .. 5 of 16 rows x 32 columns, (0,0), (1,0), (2,0), (2,1), (3,0), (3,1)
__device__ __forceinline__ constexpr int triangle_row(int b) { return b < 2 ? b : b < 4 ? 2 : 3; }
__device__ __forceinline__ constexpr int triangle_block(int b) { return b < 2 ? 0 : b & 1; }

struct TriangleTile {
    alignas(16) uint8_t b[3][6 * 1024];
    __device__ __forceinline__ void put(int block, int lane, const f32x4 &lo, const f32x4 &hi)
    {
        bf16x8 p[3];
        split(lo, hi, p);
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<bf16x8 *>(&b[i][block * 1024 + lane * 16]) = p[i];
    }
    __device__ __forceinline__ void rows(int rb, int kb, int lane, bf16x8 (&a)[3]) const
    {
        const int block = rb < 2 ? rb : 2 * rb - 2 + kb;
#pragma unroll
        for (int i = 0; i < 3; ++i) a[i] = *reinterpret_cast<const bf16x8 *>(&b[i][block * 1024 + lane * 16]);
    }
};

__device__ __forceinline__ float decay(double from, double to) { return __builtin_amdgcn_exp2f(static_cast<float>(to - from)); }

// log2 of a gate; 0 becomes a finite value whose powers are 0
__device__ __forceinline__ double log2_gate(float a) { return a == 0.0f ? -1000.0 : log2(static_cast<double>(a)); }

// The gates' products of a chunk of n tokens from t0 on, lane i token i: log2 G_i.
__device__ __forceinline__ double scan_gates(const PromptArgs &a, int t0, int n, int h, int lane, float *beta, bool *fine)
{
    double lg = 0.0;
    *beta = 0.0f;
    *fine = true;
    if (lane < n) {
        const size_t at = static_cast<size_t>(t0 + lane) * a.Hv + h;
        const float al = a.alpha.at(at);
        *beta = a.beta.p ? a.beta.at(at) : 1.0f;
        lg = log2_gate(al);
        *fine = al >= 0.0f && al < INFINITY && fabsf(*beta) < INFINITY;      // no logarithm below 0
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double up = __shfl_up(lg, d);
        if (lane >= d) lg += up;
    }
    return lg;
}

__device__ __forceinline__ void put_gates(ChunkGates *r, int lane, double lg, float beta)
{
    const double last = __shfl(lg, 63);
    r->lg[lane] = lg;
    r->g[lane] = decay(0.0, lg);
    r->w[lane] = decay(lg, last);
    r->b[lane] = beta;
}

// A wave puts sequence s in its place among the sequences, longest first.
__device__ __forceinline__ void put_order(const ChunkArgs &a, int s, int lane)
{
    const int2 be = seq_bounds(a.p, s);
    const int len = be.y - be.x;
    int before = 0;
    for (int t = lane; t < a.p.n_seq; t += 64) {
        const int2 other = seq_bounds(a.p, t);
        const int d = other.y - other.x - len;
        before += d > 0 || (d == 0 && t < s);
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) before += __shfl_xor(before, m);
    if (lane == 0) a.order[before] = make_int4(s, be.x, be.y, initial_index(a.p, s));
}

// First launch, decay rule: a wave per (chunk, head).  Bound by the latency of
// its scan: 512 chunks x 32 heads in 16 us.
__global__ __launch_bounds__(256) void prompt_gates_kernel(ChunkArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const int x = static_cast<int>(id / a.p.Hv), h = static_cast<int>(id - static_cast<int64_t>(x) * a.p.Hv);
    if (x >= a.slots) return;
    if (a.order && x < a.p.n_seq && h == 0) put_order(a, x, lane);       // there are at least as many slots
    const int s = owner(a.p, x, lane);
    const int2 be = seq_bounds(a.p, s);
    const int c = x - first_slot(a.p, s), t0 = be.x + c * kC, n = min(kC, be.y - t0);
    if (c < 0 || n <= 0) return;
    float beta;
    bool fine;
    const double lg = scan_gates(a.p, t0, n, h, lane, &beta, &fine);
    put_gates(reinterpret_cast<ChunkGates *>(a.ws + id * a.record), lane, lg, beta);
}

// First launch, Delta rule: a workgroup per (chunk, head) forms T'.  Wave w owns
// the 16 rows of row block w: k_i . k_j on the matrix cores, the 16x16 diagonal
// block's inverse by substitution, then the blocks left of it from
//   T_wc = -T_ww sum_{c <= l < w} M_wl T_lc
// in fp32 products, the blocks at equal distance from the diagonal together.
// M is 4 % of a chunk's products; what counts is the chain of 16 substitution
// steps and 3 rounds of blocks, so that 4 waves a SIMD (128 registers; the
// inverse takes the keys' place in LDS) beat 3 with more registers: 32 sequences
// 174 -> 139 us.  8 sequences of 1088 tokens x 32 heads: 53 us, 2.4 TB/s of keys
// read and T' written.  T' goes to the workspace in fp32, 4 bytes an entry where
// its three planes are 6.
//   With beta |k|^2 beyond 2 the recurrence grows, and rows of T' may pass fp32:
// their tokens and those after them are lost, and 0 stands in their place, so
// that no product takes them to a row before.
template <typename T, int DKP, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 4 : DKP == 64 ? 3 : 2) void prompt_solve_kernel(ChunkArgs a)
{
    constexpr int NA = Act<T>::planes, U = DKP / 32, LD = 68;
    // the keys are not needed once M is formed: the inverse takes their place
    __shared__ union Place {
        RowTile<T, DKP> K;
        alignas(16) float X[kC][LD];
    } place;
    __shared__ alignas(16) float M[kC][LD];
    RowTile<T, DKP> &K = place.K;
    auto &X = place.X;
    __shared__ double lgs[kC];
    __shared__ float bs[kC];
    __shared__ int bad_s;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, n = lane & 15;
    const Share<DKP / 8, 256> sh(tid);
    const int x = blockIdx.x / a.p.Hv, h = blockIdx.x - x * a.p.Hv, hq = h / (a.p.Hv / a.p.Hqk);
    if (a.order && x < a.p.n_seq && h == 0 && w == 0) put_order(a, x, lane);     // there are at least as many slots
    const int s = owner(a.p, x, lane);
    const int2 be = seq_bounds(a.p, s);
    const int chunk = x - first_slot(a.p, s);
    const int64_t t0 = be.x + chunk * kC;
    const int len = min(kC, be.y - static_cast<int>(t0));
    if (chunk < 0 || len <= 0) return;
    if (tid == 0) bad_s = kC;
    Act<T> v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        v[i] = sh.template load<VEC>(static_cast<const T *>(a.p.k) + t0 * a.p.sk + hq * a.p.dk, a.p.sk, i, a.p.dk, len);
    }
    // the gates' products: one wave's work
    float beta = 0.0f;
    bool fine = true;
    double lg = 0.0;
    if (w == 0) lg = scan_gates(a.p, t0, len, h, lane, &beta, &fine);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if constexpr (!VEC) v[i] = settle(v[i], 8 * sh.c8, a.p.dk);
        v[i] = zero_unless(sh.valid(i, a.p.dk, len), v[i]);
    }
    const bool keys_fine = max_of(v) < kInfBits;
    __syncthreads();
    if (!fine) atomicMin(&bad_s, lane);
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const int row = sh.row + sh.step * i;
        if (!keys_fine && !all_finite(v[i])) atomicMin(&bad_s, row);
        K.put(row, sh.c8, v[i]);
    }
    if (w == 0) lgs[lane] = lg, bs[lane] = beta;
    __syncthreads();
    const int bad = bad_s;
    uint8_t *rec = a.ws + (static_cast<size_t>(x) * a.p.Hv + h) * a.record;
    if (w == 0) put_gates(reinterpret_cast<ChunkGates *>(rec), lane, lg, beta);
    // M: lane (g, n) holds row i = 16 w + n, columns 16 tt + 4 g .. + 3
    bf16x8 mine[DKP / 32][NA];
#pragma unroll
    for (int kb = 0; kb < DKP / 32; ++kb) K.rows(w, kb, g, n, mine[kb]);
    const int row_i = 16 * w + n;
    const double lgi = lgs[row_i];
    const float bi = bs[row_i];
    const auto finite_or_lost = [&](float y, int row) {
        if (fabsf(y) < INFINITY) return y;
        atomicMin(&bad_s, row);
        return 0.0f;
    };
    for (int tt = 0; tt <= w; ++tt) {
        f32x4 c = {};
#pragma unroll
        for (int kb = 0; kb < DKP / 32; ++kb) {
            bf16x8 k[NA];
            K.rows(tt, kb, g, n, k);
            mma(c, k, mine[kb]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * tt + 4 * g + r;
            c[r] = j < row_i && row_i < bad ? finite_or_lost(bi * decay(lgs[j], lgi) * c[r], row_i) : 0.0f;
        }
        *reinterpret_cast<f32x4 *>(&M[row_i][16 * tt + 4 * g]) = c;
    }
    __syncthreads();
    {
        // column n of the diagonal block's inverse (every group of 16 lanes forms it)
        float t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i % 8 == 0) __builtin_amdgcn_sched_barrier(0);     // half of the rows of M in registers at a time
            float y = i == n ? 1.0f : 0.0f;
#pragma unroll
            for (int l = 0; l < i; ++l) y = fmaf(-M[16 * w + i][16 * w + l], t[l], y);
            t[i] = y;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if ((i >> 2) == g) X[16 * w + i][16 * w + n] = t[i];
    }
    for (int d = 1; d < 4; ++d) {
        __syncthreads();
        if (w >= d) {
            const int c = w - d;
            f32x4 y = {};
            for (int l = c; l < w; ++l) {
                const f32x4 m = *reinterpret_cast<const f32x4 *>(&M[16 * w + n][16 * l + 4 * g]);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    y = __builtin_amdgcn_mfma_f32_16x16x4f32(m[r], X[16 * l + 4 * g + r][16 * c + n], y, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = finite_or_lost(y[r], 16 * w + 4 * g + r);
            const f32x4 tw = *reinterpret_cast<const f32x4 *>(&X[16 * w + n][16 * w + 4 * g]);
            f32x4 z = {};
#pragma unroll
            for (int r = 0; r < 4; ++r) z = __builtin_amdgcn_mfma_f32_16x16x4f32(tw[r], y[r], z, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) X[16 * w + 4 * g + r][16 * c + n] = -finite_or_lost(z[r], 16 * w + 4 * g + r);
        }
    }
    __syncthreads();
    // beta into the columns, then block by block to the record
    for (int tt = 0; tt <= w; ++tt) {
        f32x4 *at = reinterpret_cast<f32x4 *>(&X[row_i][16 * tt + 4 * g]);
        f32x4 y = *at;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * tt + 4 * g + r;
            y[r] = j < bad ? finite_or_lost(y[r] * bs[j], row_i) : 0.0f;
        }
        *at = y;
    }
    __syncthreads();
    if (tid == 0) reinterpret_cast<ChunkGates *>(rec)->bad = bad_s;
    for (int b = w; b < 6; b += 4) {
        const int rb = triangle_row(b), kb = triangle_block(b);
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(&X[16 * rb + n][32 * kb + 4 * g]);
        const f32x4 hi = 2 * kb + 1 <= rb ? *reinterpret_cast<const f32x4 *>(&X[16 * rb + n][32 * kb + 16 + 4 * g]) : f32x4{};
        f32x4 *to = reinterpret_cast<f32x4 *>(rec + sizeof(ChunkGates) + b * 2048) + 2 * lane;
        to[0] = lo, to[1] = hi;
    }
}

// f(address, rt, r) for the rows of a state that a lane holds, column n of `base`.
template <int DKP, typename F, typename P>
__device__ __forceinline__ void each_state_row(P *base, int dk, int dv, int g, int n, const F &f)
{
    int first = 8 * g;
    asm volatile("" : "+v"(first));          // addresses and masks are formed here, not kept for the other call
    const uint32_t at = static_cast<uint32_t>(first) * dv + n;
#pragma unroll
    for (int rt = 0; rt < DKP / 16; ++rt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int up = state_row(rt, r);
            if (dk == DKP || first + up < dk) f(base + static_cast<int64_t>(up) * dv + at, rt, r);
        }
}

// The state sequence s starts from; NULL: zeros.
__device__ __forceinline__ const float *initial_state(const PromptArgs &a, int src, int h)
{
    return src >= 0 ? a.state_in + (static_cast<size_t>(src) * a.Hv + h) * a.dk * a.dv : nullptr;
}

// Long sequences with too few heads to fill the chip are cut into segments of
// whole chunks.  A segment takes a state S to A S + B (decay rule: A = gamma I),
// whatever S is, so that: a launch forms B of every segment by walking it from
// a zero state, and for the Delta rule A by walking it from the identity with
// all values zero; one applies them in order (prompt_join kernels), leaving the
// state after each segment in B's place (the last one has no B: there, the state
// before the first); and then all segments are walked at once.
constexpr int kSegmentHead = 64;         // floats; [0] = gamma

// Second launch: a workgroup of NW waves walks the chunks of one (sequence, head)
// or of a segment of it (OUT false: for B and A, without outputs) for 16 NW value
// columns, a wave holds 16 columns of the state in registers (result layout: lane
// n column n).  Every product with the state, and every one after it, keeps the
// columns in their lanes, so that the waves share only what is read.  fp32 values
// come straight into that layout (their tile, beside keys and queries in three
// planes, would not fit the LDS).
//   Bound by the chain of a chunk: R needs S, U needs R, the next S needs U, and
// 2 waves a SIMD (their state, R, O and the next chunk's tiles: 184 registers)
// cover its waits only in part.  8 sequences of 1088 tokens x 32 heads, a
// workgroup for every CU: 141 us, 8.3 us a chunk, in which the vector units issue
// half of the time (splitting into planes above all) and the matrix cores work
// 43 %; 1.9 TB/s.  Without outputs bfloat16 takes 128 registers, two workgroups a
// CU.  Measured with the operands in two binary16 planes, for 32 sequences: 32
// columns a wave spill; 128 registers and two workgroups a CU spill too (826 us
// against 618 then); two workgroups of 64 columns form K, Q and P twice (492 ->
// 564); opposite orders of P and K S in the two waves of a SIMD 570 -> 603; values
// asked for a whole chunk ahead 488 -> 498.
//   VEC: rows of 16-byte pieces that start at 16 bytes.  The other form reads
// them at any alignment and cuts the last one; taken for all, 570 -> 628 us.
template <typename T, int DKP, int NW, bool DELTA, bool VEC, bool OUT>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 || NW == 8 ? 2 : 1) void prompt_chunks_kernel(ChunkArgs a)
{
    constexpr int NA = Act<T>::planes, KB = DKP / 32, W = 16 * NW;
    using ShareQ = Share<DKP / 8, 64 * NW>;
    using ShareV = Share<W / 8, 64 * NW>;
    constexpr int UQ = ShareQ::units, UV = ShareV::units;
    __shared__ RowTile<T, DKP> K;
    __shared__ std::conditional_t<OUT, RowTile<T, DKP>, char> Q;
    __shared__ std::conditional_t<sizeof(T) == 2, ValueTile<W>, char> V;
    __shared__ std::conditional_t<OUT, TriangleTile, char> P;
    __shared__ std::conditional_t<DELTA, TriangleTile, char> Tt;
    __shared__ struct alignas(16) {
        double lg[kC];
        float g[kC], w[kC], b[kC];
        int32_t bad;
    } ga;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    // Addresses in LDS follow from the lane: formed again in each phase, they do not hold registers from chunk to chunk.
    const auto again = [&] {
        asm volatile("" : "+v"(lane));
        g = lane >> 4, n = lane & 15;
    };
    const ShareQ sh(threadIdx.x);
    const ShareV sv(threadIdx.x);
    const int value_blocks = a.p.dv / W, blocks = value_blocks + (OUT || !DELTA ? 0 : (DKP + W - 1) / W);
    const int cb = blockIdx.x % blocks, h = blockIdx.x / blocks % a.p.Hv, item = blockIdx.x / blocks / a.p.Hv;
    const int hq = h / (a.p.Hv / a.p.Hqk);
    const bool values = OUT || !DELTA || cb < value_blocks;      // B; else A
    const int col0 = (values ? cb : cb - value_blocks) * W, mycol = wv * 16;
    int s, start;
    int2 be;
    if (!a.seg && a.order) {
        const int4 e = a.order[item];            // one load deep
        s = e.x, be = make_int2(e.y, e.z), start = e.w;
    } else {
        s = a.seg ? owner(a.p, item, lane, kC * a.seg) : item;
        be = seq_bounds(a.p, s);
        start = initial_index(a.p, s);
    }
    const int total = (be.y - be.x + kC - 1) / kC, part = a.seg ? item - first_slot(a.p, s, kC * a.seg) : 0;
    const int first = part * a.seg, chunks = a.seg ? min(total, first + a.seg) : total;
    if (part < 0 || (part > 0 && first >= total)) return;        // tokens before the first sequence, or a slot that none has
    if (!OUT && chunks == total) return;         // nothing follows it
    float *rec = a.seg ? a.segs + (static_cast<size_t>(item) * a.p.Hv + h) * a.seg_floats : nullptr;
    const uint8_t *records = a.ws + (static_cast<size_t>(be.x / kC + s) * a.p.Hv + h) * a.record;

    f32x4 S[DKP / 16];
#pragma unroll
    for (int rt = 0; rt < DKP / 16; ++rt) S[rt] = f32x4{};
    if constexpr (OUT) {
        // the first of several segments has its state from the last one's record: state_out may be state_in
        const int64_t back = part == 0 && a.seg ? (total + a.seg - 1) / a.seg - 1 : -1;
        const float *from = part == 0 && back <= 0 ? initial_state(a.p, start, h)
                                                   : rec + back * a.p.Hv * static_cast<int64_t>(a.seg_floats) + kSegmentHead;
        if (from)
            each_state_row<DKP>(from + col0 + mycol, a.p.dk, a.p.dv, g, n,
                                [&](const float *at, int rt, int r) { S[rt][r] = *at; });
    } else if (!values) {
#pragma unroll
        for (int rt = 0; rt < DKP / 16; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[rt][r] = state_row(rt, 4 * g + r) == col0 + mycol + n ? 1.0f : 0.0f;
    }
    float gamma = 1.0f;

    // What the next chunk needs is on its way while this one is computed, each
    // part in registers for as short as its latency allows: keys and queries
    // from the second barrier on, values and gates from the state's update on;
    // T' from the chunk's own first barrier to its third.
    Act<T> kx[UQ], qx[OUT ? UQ : 1];
    Act<bf16_t> vx[sizeof(T) == 2 ? UV : 1] = {};
    f32x4 vf[sizeof(T) == 4 ? 4 : 1] = {};           // fp32 values: rows 16 rb + 4 g .. + 3 of the lane's column
    constexpr int NT = (6 + NW - 1) / NW;            // blocks of T' per wave
    f32x4 tx[NT][2];
    constexpr int NG = (kGateWords + 64 * NW - 1) / (64 * NW);
    uint32_t gx[NG];
    const auto record = [&](int c) { return records + static_cast<size_t>(c) * a.p.Hv * a.record; };
    // Whole chunks whose rows lie within 32-bit offsets: one lane offset per
    // array for all chunks, the rest in scalar registers.
    const bool near = VEC && a.near && a.p.dk == DKP;
    const uint32_t at_k = (sh.row * static_cast<uint32_t>(a.p.sk) + 8 * sh.c8) * static_cast<uint32_t>(sizeof(T));
    const uint32_t at_q = (sh.row * static_cast<uint32_t>(a.p.sq) + 8 * sh.c8) * static_cast<uint32_t>(sizeof(T));
    const uint32_t at_v = sizeof(T) == 2 ? (sv.row * static_cast<uint32_t>(a.p.sv) + 8 * sv.c8) * 2u
                                         : (4 * g * static_cast<uint32_t>(a.p.sv) + n) * 4u;
    const auto fetch = [&](int c) {
        const int64_t t0 = be.x + c * kC;
        const int len = min(kC, be.y - static_cast<int>(t0));
        if (near && len == kC) {
#pragma unroll
            for (int i = 0; i < UQ; ++i) {
                kx[i] = load_at(static_cast<const T *>(a.p.k) + (t0 + i * sh.step) * a.p.sk + hq * a.p.dk, at_k);
                if constexpr (OUT) qx[i] = load_at(static_cast<const T *>(a.p.q) + (t0 + i * sh.step) * a.p.sq + hq * a.p.dk, at_q);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < UQ; ++i) {
            kx[i] = sh.template load<VEC>(static_cast<const T *>(a.p.k) + t0 * a.p.sk + hq * a.p.dk, a.p.sk, i, a.p.dk, len);
            if constexpr (OUT)
                qx[i] = sh.template load<VEC>(static_cast<const T *>(a.p.q) + t0 * a.p.sq + hq * a.p.dk, a.p.sq, i, a.p.dk, len);
        }
    };
    // bfloat16 values past the last token repeat it, fp32 ones are 0: their rows of U are 0 (beta is 0 there)
    const auto fetch_values = [&](int c) {
        const int64_t t0 = be.x + c * kC;
        const int len = min(kC, be.y - static_cast<int>(t0));
        const T *from = static_cast<const T *>(a.p.v) + t0 * a.p.sv + h * a.p.dv + col0;
        if constexpr (sizeof(T) == 2) {
            if (values && near && len == kC) {
#pragma unroll
                for (int i = 0; i < UV; ++i) vx[i] = load_at(from + i * sv.step * a.p.sv, at_v);
            } else if (values)
#pragma unroll
            for (int i = 0; i < UV; ++i) vx[i] = sv.template load<VEC>(from, a.p.sv, i, W, len);
        } else if (values) {
            const auto load = [&](int m) {
                const T *row = from + mycol;
#pragma unroll
                for (int rb = 0; rb < 4; ++rb, row += 12 * a.p.sv)
#pragma unroll
                    for (int r = 0; r < 4; ++r, row += a.p.sv)
                        vf[rb][r] = 16 * rb + 4 * g + r < m
                                        ? *reinterpret_cast<const T *>(reinterpret_cast<const uint8_t *>(row) + at_v) : 0.0f;
            };
            len == kC ? load(kC) : load(len);
        }
        const uint32_t *words = reinterpret_cast<const uint32_t *>(record(c));
#pragma unroll
        for (int i = 0; i < NG; ++i) gx[i] = words[min(static_cast<int>(threadIdx.x) + 64 * NW * i, kGateWords - 1)];
    };
    if (chunks > first) fetch(first), fetch_values(first);

    for (int c = first; c < chunks; ++c) {
        const int64_t t0 = be.x + c * kC;
        const int len = min(kC, be.y - static_cast<int>(t0));
        if (len < kC || a.p.dk < DKP) {
#pragma unroll
            for (int i = 0; i < UQ; ++i) {
                const bool keep = sh.valid(i, a.p.dk, len);
                if constexpr (!VEC) {
                    kx[i] = settle(kx[i], 8 * sh.c8, a.p.dk);
                    if constexpr (OUT) qx[i] = settle(qx[i], 8 * sh.c8, a.p.dk);
                }
                kx[i] = zero_unless(keep, kx[i]);
                if constexpr (OUT) qx[i] = zero_unless(keep, qx[i]);
            }
        }
        again();
        lds_barrier();
        const ChunkGates *cg = reinterpret_cast<const ChunkGates *>(record(c));
        if constexpr (DELTA) {
            const f32x4 *from = reinterpret_cast<const f32x4 *>(cg + 1) + 2 * lane;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int b = min(wv + NW * i, 5) * 128;
                tx[i][0] = from[b], tx[i][1] = from[b + 1];
            }
        }
        const auto at = sh.again();
#pragma unroll
        for (int i = 0; i < UQ; ++i) {
            K.put(at.row + at.step * i, at.c8, kx[i]);
            if constexpr (OUT) Q.put(at.row + at.step * i, at.c8, qx[i]);
        }
        if constexpr (sizeof(T) == 2) {
            const auto av = sv.again();
#pragma unroll
            for (int i = 0; i < UV; ++i) V.put(av.row + av.step * i, av.c8, vx[i]);
        }
#pragma unroll
        for (int i = 0; i < NG; ++i)
            reinterpret_cast<uint32_t *>(&ga)[min(static_cast<int>(threadIdx.x) + 64 * NW * i, kGateWords - 1)] = gx[i];
        lds_barrier();
        if (c + 1 < chunks) fetch(c + 1);
        const int bad = DELTA ? __builtin_amdgcn_readfirstlane(ga.bad) : kC;

        again();
        // P, a block of 16 rows x 32 columns to a wave: lane (g, n) forms row i = 16 rb + n, columns 16 tt + 4 g .. + 3
        if constexpr (OUT)
#pragma unroll
        for (int b = wv; b < 6; b += NW) {
            const int rb = triangle_row(b), pb = triangle_block(b);
            bf16x8 q[KB][NA];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) Q.rows(rb, kb, g, n, q[kb]);
            const double lgi = ga.lg[16 * rb + n];
            f32x4 y[2] = {};
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int tt = 2 * pb + hh;
                if (tt <= rb) {
                    f32x4 x = {};
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        bf16x8 k[NA];
                        K.rows(tt, kb, g, n, k);
                        mma(x, k, q[kb]);
                    }
                    float d[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) d[r] = x[r] * decay(ga.lg[16 * tt + 4 * g + r], lgi);
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[hh][r] = ((tt < rb) | (4 * g + r <= n)) ? d[r] : 0.0f;
                }
            }
            P.put(b, lane, y[0], y[1]);
        }
        again();
        // K S and Q S
        f32x4 ks[4], o[4];
#pragma unroll
        for (int rb = 0; rb < 4; ++rb) ks[rb] = o[rb] = f32x4{};
#pragma unroll
        for (int kb = 0; kb < (OUT || DELTA ? KB : 0); ++kb) {
            bf16x8 sp[3];
            split(S[2 * kb], S[2 * kb + 1], sp);
#pragma unroll
            for (int rb = 0; rb < 4; ++rb) {
                if constexpr (OUT) {
                    bf16x8 q[NA];
                    Q.rows(rb, kb, g, n, q);
                    mma(o[rb], q, sp);
                }
                if constexpr (DELTA) {
                    bf16x8 k[NA];
                    K.rows(rb, kb, g, n, k);
                    mma(ks[rb], k, sp);
                }
            }
        }
        // 3 steps' operands ahead (32 sequences, in two binary16 planes: 537 -> 530 us); the update of S the same way is
        // slower (541)
        if constexpr (OUT && DELTA && sizeof(T) == 2) reads_ahead<4 * KB, 2, 6, 3>();
        again();
        // R (Delta) or U (decay); O's part from the state
#pragma unroll
        for (int rb = 0; rb < 4; ++rb) {
            const f32x4 gg = *reinterpret_cast<const f32x4 *>(&ga.g[16 * rb + 4 * g]);
            f32x4 bb = {};
            if (!DELTA) bb = *reinterpret_cast<const f32x4 *>(&ga.b[16 * rb + 4 * g]);
            f32x4 v;
            if constexpr (sizeof(T) == 2) v = V.four(rb, mycol, g, n);
            else v = vf[rb];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (DELTA) ks[rb][r] = fmaf(-gg[r], ks[rb][r], v[r]);
                else ks[rb][r] = v[r] * bb[r];
                if (OUT) o[rb][r] *= gg[r];
            }
        }
        // Tokens from `from` on are lost in their column: what is not finite there may not reach the others
        // through products with zeros, so it is taken out of an operand and put in its place at the end.  A
        // product of the operand with zeros tells (the final state needs no care: it has all tokens).
        bool lost = false;
        int from = bad;
        const auto operand = [&](bf16x8 (&p)[2][3], bool cut) {
            const auto form = [&] {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) split(ks[2 * kb], ks[2 * kb + 1], p[kb]);
            };
            form();
            if constexpr (OUT) {
                f32x4 z = {};
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16x8{}, p[kb][0], z, 0, 0, 0);
                cut |= __any(z[0] != 0.0f);
            }
            if (!cut) return;
            lost = true;
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!(fabsf(ks[rb][r]) < INFINITY)) from = min(from, 16 * rb + 4 * g + r);
            from = kC - static_cast<int>(column_max(kC - from));
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * rb + 4 * g + r >= from) ks[rb][r] = 0.0f;
            form();
        };
        if constexpr (DELTA)
#pragma unroll
            for (int i = 0; i < NT; ++i)
                if (wv + NW * i < 6) Tt.put(wv + NW * i, lane, tx[i][0], tx[i][1]);
        lds_barrier();
        again();
        // U = T' R
        if constexpr (DELTA) {
            bf16x8 rp[2][3];
            operand(rp, bad < kC);
#pragma unroll
            for (int rb = 0; rb < 4; ++rb) {
                ks[rb] = f32x4{};
#pragma unroll
                for (int kb = 0; kb <= rb / 2; ++kb) {
                    bf16x8 t[3];
                    Tt.rows(rb, kb, lane, t);
                    mma(ks[rb], t, rp[kb]);
                }
            }
        }
        again();
        // O += P U
        if constexpr (OUT) {
            bf16x8 up[2][3];
            operand(up, false);              // U may pass fp32 where R did not
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
#pragma unroll
                for (int kb = 0; kb <= rb / 2; ++kb) {
                    bf16x8 p[3];
                    P.rows(rb, kb, lane, p);
                    mma(o[rb], p, up[kb]);
                }
        }
        if (OUT && lost)
#pragma unroll
            for (int rb = 0; rb < 4; ++rb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * rb + 4 * g + r >= from) o[rb][r] = NAN;
        Out4<T> y[4];
#pragma unroll
        for (int rb = 0; rb < 4; ++rb) y[rb].set(o[rb]);
        const auto store = [&](int m) {
            // each row's address is the wave's own (scalar) plus this lane's fixed part
            uint8_t *out = reinterpret_cast<uint8_t *>(static_cast<T *>(a.p.o) + t0 * a.p.so + h * a.p.dv + col0 + mycol);
            const uint32_t at = (4 * g * static_cast<uint32_t>(a.p.so) + n) * static_cast<uint32_t>(sizeof(T));
            const int64_t step = a.p.so * static_cast<int64_t>(sizeof(T));
#pragma unroll
            for (int rb = 0; rb < 4; ++rb, out += 12 * step)
#pragma unroll
                for (int r = 0; r < 4; ++r, out += step)
                    if (16 * rb + 4 * g + r < m) *reinterpret_cast<T *>(out + at) = y[rb].at(r);
        };
        // bfloat16 outputs wait in half the registers, so that what the next chunk needs is asked for first
        if constexpr (OUT && sizeof(T) == 4) again(), len == kC ? store(kC) : store(len);
        if (c + 1 < chunks) fetch_values(c + 1);
        again();
        // S <- G_last S + K^T (w U)
        {
            const float glast = ga.g[kC - 1];
            if (!OUT) gamma *= glast;
            bf16x8 up[2][3];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const f32x4 w0 = *reinterpret_cast<const f32x4 *>(&ga.w[32 * kb + 4 * g]);
                const f32x4 w1 = *reinterpret_cast<const f32x4 *>(&ga.w[32 * kb + 16 + 4 * g]);
                split(ks[2 * kb] * w0, ks[2 * kb + 1] * w1, up[kb]);
            }
#pragma unroll
            for (int rt = 0; rt < DKP / 16; ++rt) {
                S[rt] *= glast;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    bf16x8 k[NA];
                    K.columns(rt, kb, g, n, k);
                    mma(S[rt], k, up[kb]);
                }
            }
        }
        if (lost && from < kC)
#pragma unroll
            for (int rt = 0; rt < DKP / 16; ++rt) S[rt] = f32x4{NAN, NAN, NAN, NAN};
        if constexpr (OUT && sizeof(T) == 2) again(), len == kC ? store(kC) : store(len);
    }

    const auto put = [&](float *at, int rt, int r) { *at = S[rt][r]; };
    if constexpr (OUT) {
        if (chunks == total)
            each_state_row<DKP>(a.p.state_out + (static_cast<size_t>(s) * a.p.Hv + h) * a.p.dk * a.p.dv + col0 + mycol, a.p.dk,
                                a.p.dv, g, n, put);
    } else {
        if (cb == 0 && threadIdx.x == 0) rec[0] = gamma;
        float *to = rec + kSegmentHead + col0 + mycol;
        if (values) each_state_row<DKP>(to, a.p.dk, a.p.dv, g, n, put);
        else if (col0 + mycol < DKP) each_state_row<DKP>(to + a.p.dk * a.p.dv, DKP, DKP, g, n, put);
    }
}

// The states after the segments of a sequence, in order, decay rule: 4 elements
// a thread.  Bound by memory: the records of 8 segments x 32 heads of 128 x 128
// read and written, 34 MB in 8.5 us, 3.9 TB/s; of 24, 100 MB in 21 us, 4.7.
__global__ __launch_bounds__(256) void prompt_join_decay_kernel(ChunkArgs a)
{
    const int quads = a.p.dk * a.p.dv / 4, blocks = (quads + 255) / 256;
    const int h = blockIdx.x / blocks % a.p.Hv, s = blockIdx.x / blocks / a.p.Hv, e = blockIdx.x % blocks * 256 + threadIdx.x;
    const int2 be = seq_bounds(a.p, s);
    const int total = (be.y - be.x + kC - 1) / kC, parts = (total + a.seg - 1) / a.seg;
    if (e >= quads || parts < 2) return;
    const float *from = initial_state(a.p, initial_index(a.p, s), h);
    f32x4 S = {};
    if (from)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[i] = from[4 * e + i];
    float *rec = a.segs + (static_cast<size_t>(first_slot(a.p, s, kC * a.seg)) * a.p.Hv + h) * a.seg_floats;
    reinterpret_cast<f32x4 *>(rec + (parts - 1) * (a.p.Hv * a.seg_floats) + kSegmentHead)[e] = S;
    for (int j = 0; j + 1 < parts; ++j, rec += a.p.Hv * a.seg_floats) {
        f32x4 *B = reinterpret_cast<f32x4 *>(rec + kSegmentHead) + e;
        S = *B + S * rec[0];
        *B = S;
    }
}

// The same for the Delta rule, S <- A S + B in fp32 products: a workgroup 16
// columns of the state, a wave a quarter of its rows.  The state goes around
// through LDS; A does not depend on it and is asked for one segment ahead.
// Bound by the chain of segments: 8 of them x 32 heads of 128 x 128 in 27 us (97
// us with a workgroup for all columns of a head; 32 with a head's column blocks
// on 8 XCDs, each of which read A for itself).
template <int DKP>
__global__ __launch_bounds__(256) void prompt_join_delta_kernel(ChunkArgs a)
{
    constexpr int KT = DKP / 16, RT = KT / 4, LD = DKP + 4;
    __shared__ alignas(16) float st[2][16 * LD];      // [column][row]
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    // the column blocks of a head go to one XCD (every 8th workgroup), which then reads its A once
    const int blocks = a.p.dv / 16, pair = blockIdx.x / (8 * blocks) * 8 + blockIdx.x % 8;
    if (pair >= a.p.n_seq * a.p.Hv) return;
    const int h = pair % a.p.Hv, s = pair / a.p.Hv;
    const int col = blockIdx.x / 8 % blocks * 16 + n, row0 = 16 * RT * wv + 4 * g;     // + 16 rt + r
    const int2 be = seq_bounds(a.p, s);
    const int total = (be.y - be.x + kC - 1) / kC, parts = (total + a.seg - 1) / a.seg;
    if (parts < 2) return;
    const size_t step = a.p.Hv * a.seg_floats;
    float *rec = a.segs + (static_cast<size_t>(first_slot(a.p, s, kC * a.seg)) * a.p.Hv + h) * a.seg_floats;
    const float *from = initial_state(a.p, initial_index(a.p, s), h);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = row0 + 16 * rt + r;
            x[r] = from && i < a.p.dk ? from[i * a.p.dv + col] : 0.0f;
            if (i < a.p.dk) rec[(parts - 1) * step + kSegmentHead + i * a.p.dv + col] = x[r];
        }
        *reinterpret_cast<f32x4 *>(&st[0][n * LD + row0 + 16 * rt]) = x;
    }
    f32x4 x[RT][KT], y[RT];
    const auto fetch = [&](const float *at) {
        const f32x4 *A = reinterpret_cast<const f32x4 *>(at + kSegmentHead + a.p.dk * a.p.dv) + (16 * RT * wv + n) * (DKP / 4) + g;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) x[rt][kt] = A[rt * 16 * (DKP / 4) + 4 * kt];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = row0 + 16 * rt + r;
                y[rt][r] = i < a.p.dk ? at[kSegmentHead + i * a.p.dv + col] : 0.0f;
            }
        }
    };
    fetch(rec);
    for (int j = 0; j + 1 < parts; ++j, rec += step) {
        __syncthreads();
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const f32x4 S = *reinterpret_cast<const f32x4 *>(&st[j & 1][n * LD + 16 * kt + 4 * g]);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int r = 0; r < 4; ++r) y[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[rt][kt][r], S[r], y[rt], 0, 0, 0);
        }
        f32x4 z[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            z[rt] = y[rt];
            *reinterpret_cast<f32x4 *>(&st[~j & 1][n * LD + row0 + 16 * rt]) = z[rt];
        }
        if (j + 2 < parts) fetch(rec + step);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (row0 + 16 * rt + r < a.p.dk) rec[kSegmentHead + (row0 + 16 * rt + r) * a.p.dv + col] = z[rt][r];
    }
}

template <typename T, int DKP, bool DELTA, bool VEC>
void launch_rule(const ChunkArgs &a, hipStream_t s)
{
    const int64_t items = static_cast<int64_t>(a.slots) * a.p.Hv;
    if constexpr (DELTA) prompt_solve_kernel<T, DKP, VEC><<<dim3(static_cast<unsigned>(items)), 256, 0, s>>>(a);
    else prompt_gates_kernel<<<dim3(static_cast<unsigned>((items + 3) / 4)), 256, 0, s>>>(a);
    const unsigned pairs = static_cast<unsigned>(a.p.n_seq) * a.p.Hv, walks = static_cast<unsigned>(a.seg ? a.seg_slots : a.p.n_seq) * a.p.Hv;
    if (a.seg) {
        const unsigned blocks = 1 + (DELTA ? (DKP + a.p.dv - 1) / a.p.dv : 0);
        if (a.p.dv == 128) prompt_chunks_kernel<T, DKP, 8, DELTA, VEC, false><<<dim3(walks * blocks), 512, 0, s>>>(a);
        else prompt_chunks_kernel<T, DKP, 4, DELTA, VEC, false><<<dim3(walks * blocks), 256, 0, s>>>(a);
        if constexpr (DELTA) prompt_join_delta_kernel<DKP><<<dim3((pairs + 7) / 8 * 8 * (a.p.dv / 16)), 256, 0, s>>>(a);
        else prompt_join_decay_kernel<<<dim3(pairs * ((a.p.dk * a.p.dv / 4 + 255) / 256)), 256, 0, s>>>(a);
    }
    if (a.p.dv == 128) prompt_chunks_kernel<T, DKP, 8, DELTA, VEC, true><<<dim3(walks), 512, 0, s>>>(a);
    else prompt_chunks_kernel<T, DKP, 4, DELTA, VEC, true><<<dim3(walks), 256, 0, s>>>(a);
}

template <typename T, int DKP>
void launch(const ChunkArgs &a, bool delta, bool vec, hipStream_t s)
{
    if (delta) {
        if (vec) launch_rule<T, DKP, true, true>(a, s);
        else launch_rule<T, DKP, true, false>(a, s);
    } else {
        if (vec) launch_rule<T, DKP, false, true>(a, s);
        else launch_rule<T, DKP, false, false>(a, s);
    }
}

// Sequence s has its chunks from slot cu[s] / 64 + s on: enough for any lengths
// that add up to n_tokens, and known without reading cu_seqlens on the host.
int64_t slots(const stepq_prompt_desc *d) { return d->n_tokens / kC + d->n_seq; }

stepq_status check(const stepq_prompt_desc *d)
{
    if (!d) return bad("desc is NULL");
    if (d->n_v_heads < 1 || d->n_qk_heads < 1 || d->n_v_heads % d->n_qk_heads)
        return bad("head counts must be >= 1 and n_v_heads a multiple of n_qk_heads");
    if (d->d_k < 1 || d->d_k > 128 || (d->d_v != 64 && d->d_v != 128))
        return set_error(STEPQ_E_UNSUPPORTED, "d_k must be 1 .. 128 and d_v 64 or 128");
    if (!known_dtype(d->act_dtype) || !known_dtype(d->gate_dtype)) return bad("unknown activation or gate dtype");
    if (d->rule != STEPQ_RULE_DECAY && d->rule != STEPQ_RULE_DELTA) return bad("unknown rule");
    if (d->n_tokens < 0 || d->n_seq < 0 || d->n_states_in < 0) return bad("negative count");
    if (d->n_tokens >= (int64_t(1) << 31))
        return set_error(STEPQ_E_UNSUPPORTED, "2^31 tokens or more in one call: split the batch");
    if (static_cast<int64_t>(d->n_seq) * d->n_v_heads > (int64_t(1) << 24))
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^24 (sequence, head) pairs in one call: split the batch");
    const int64_t qk = int64_t(d->n_qk_heads) * d->d_k, vo = int64_t(d->n_v_heads) * d->d_v;
    if ((d->q_stride && d->q_stride < qk) || (d->k_stride && d->k_stride < qk) || (d->v_stride && d->v_stride < vo) ||
        (d->o_stride && d->o_stride < vo))
        return bad("a token stride is smaller than a token");
    // the kernels' offsets within a wave's rows are 32-bit
    if (std::max({d->q_stride, d->k_stride, d->v_stride, d->o_stride, qk, vo}) > (int64_t(1) << 26))
        return set_error(STEPQ_E_UNSUPPORTED, "tokens more than 2^26 elements apart");
    // (a launch has less than 2^32 threads)
    if (slots(d) * d->n_v_heads >= (int64_t(1) << 23))
        return set_error(STEPQ_E_UNSUPPORTED, "2^23 (chunk, head) pairs or more in one call: split the batch");
    return STEPQ_OK;
}

// Chunks per segment; 0: sequences are walked whole.  Lengths are not known
// here: the average decides, and of several sequences the longest is taken to be
// half as long again.  Segments pay where whole sequences leave CUs idle: they
// cost a walk of their own for B (Delta rule: and one for A), and a step of the
// join each, of which more than about the root of the chunks' number are not
// worth it.  Whole against segments, heads of 128 x 128, us:
//   Delta, 32 heads: 6 chunks 54 / 55 (6 segments), 8 chunks 67 / 58 (6), 16
//     chunks 121 / 87 (8), 32 chunks 228 / 120, 128 chunks 882 / 319; 64 heads, 8
//     chunks 69 / 74 (4), 16 chunks 125 / 117 (4); 8 heads, 64 chunks 431 / 118
//     (16); 96 heads, 64 chunks 495 / 449 (2), 16 chunks 135 / 149; 128 heads, 16
//     chunks 139 / 157 (2), 32 chunks 265 / 270 (2); 5 ragged fp32 sequences of 6
//     heads, 12 chunks each on the average, 167 / 88 (12);
//   decay, 32 heads: 8 chunks 50 / 38 (8), 32 chunks 174 / 62, 128 chunks 671 /
//     155, 256 chunks 1366 / 281 (8; 16: 304, 24: 329), 512 chunks 2717 / 548 (8;
//     24: 606); 4 chunks 29 / 35 (4); 8 heads, 512 chunks 2674 / 159 (32); 64 heads,
//     16 chunks 92 / 63 (4), 256 chunks 1380 / 532 (4; 12: 600); 128 heads, 64
//     chunks 368 / 287 (4), 16 chunks 94 / 106; 152 heads, 32 chunks 181 / 187 (3).
int32_t segment_chunks(const stepq_prompt_desc *d)
{
    const int64_t pairs = int64_t(d->n_seq) * d->n_v_heads, each = d->n_seq ? slots(d) / d->n_seq : 0;
    const int64_t longest = d->n_seq > 1 ? each * 3 / 2 : each, root = std::lround(std::sqrt(static_cast<double>(each)));
    const bool delta = d->rule == STEPQ_RULE_DELTA;
    if (pairs < 1 || pairs >= (delta ? 100 : 160)) return 0;
    int64_t parts;
    if (delta) {
        parts = std::min(256 / pairs, 2 * root);
        if (parts < 2 || (longest + 4) * parts < 72) return 0;
    } else {
        parts = std::min({(pairs <= 64 ? 256 : 512) / pairs, 4 * root, each});
        if (parts < 2 || longest < (pairs <= 64 ? 8 : 32)) return 0;
    }
    return static_cast<int32_t>((each + parts - 1) / parts);
}

size_t record_bytes(const stepq_prompt_desc *d)
{
    return sizeof(ChunkGates) + (d->rule == STEPQ_RULE_DELTA ? kTBytes : 0);
}

struct Layout {              // of the workspace
    size_t record, chunks;   // bytes per (chunk, head), of all
    int32_t seg, seg_slots;
    size_t seg_floats, order, bytes;   // order: its place, 0 without one
};

Layout layout_of(const stepq_prompt_desc *d)
{
    Layout l{};
    l.record = record_bytes(d);
    l.chunks = (static_cast<size_t>(slots(d)) * d->n_v_heads * l.record + 255) / 256 * 256;
    l.seg = segment_chunks(d);
    if (l.seg) {
        l.seg_slots = static_cast<int32_t>(d->n_tokens / (kC * int64_t(l.seg)) + d->n_seq);
        const size_t dkp = d->d_k > 64 ? 128 : 64;
        l.seg_floats = kSegmentHead + (size_t(d->d_k) * d->d_v + (d->rule == STEPQ_RULE_DELTA ? dkp * dkp : 0) + 63) / 64 * 64;
    }
    l.bytes = l.chunks + static_cast<size_t>(l.seg_slots) * d->n_v_heads * l.seg_floats * sizeof(float);
    // More walks than CUs are begun longest first, or the chip waits for long ones that were begun late.  Of very
    // many sequences the last ones are a small part, and counting who is longer is not.
    if (!l.seg && d->n_seq > 1 && d->n_seq <= 4096 && int64_t(d->n_seq) * d->n_v_heads > 256) {
        l.order = l.bytes;
        l.bytes += (static_cast<size_t>(d->n_seq) * sizeof(int4) + 255) / 256 * 256;
    }
    return l;
}


}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_prompt_workspace(const stepq_prompt_desc *d, size_t *bytes)
{
    if (const stepq_status st = check(d)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = layout_of(d).bytes;
    return STEPQ_OK;
}

extern "C" stepq_status stepq_prompt(const stepq_prompt_desc *d, const int32_t *cu_seqlens, const void *q,
                                     const void *k, const void *v, const void *alpha, const void *beta, void *o,
                                     const float *state_in, const int32_t *in_ids, float *state_out, void *workspace,
                                     size_t workspace_bytes, void *stream)
{
    if (const stepq_status st = check(d)) return st;
    if (d->n_seq == 0) return STEPQ_OK;
    if (!cu_seqlens && d->n_seq > 1) return bad("NULL cu_seqlens with more than one sequence");
    if (!state_out) return bad("state_out is NULL");
    if (d->n_tokens && (!q || !k || !v || !alpha || !o)) return bad("NULL activation or output pointer");
    if (!state_in && in_ids) return bad("in_ids without state_in");
    if (state_in && !in_ids && d->n_states_in < d->n_seq) return bad("fewer states in state_in than sequences");
    if (state_in == state_out && in_ids) return bad("state_out must not be state_in where in_ids chooses the states");
    const Layout l = layout_of(d);
    if (!workspace || workspace_bytes < l.bytes) return bad("workspace is smaller than stepq_prompt_workspace()");
    if (!aligned(workspace, 256) || !aligned(state_out, 4)) return bad("workspace must be 256-byte aligned");
    const int64_t qk = int64_t(d->n_qk_heads) * d->d_k, vo = int64_t(d->n_v_heads) * d->d_v;
    const int32_t gf = d->gate_dtype == STEPQ_F32;
    ChunkArgs a{};
    a.p = PromptArgs{cu_seqlens, q, k, v, {alpha, gf}, {beta, gf}, o, state_in, in_ids, state_out,
                     d->q_stride ? d->q_stride : qk, d->k_stride ? d->k_stride : qk, d->v_stride ? d->v_stride : vo,
                     d->o_stride ? d->o_stride : vo, static_cast<int32_t>(d->n_tokens), d->n_seq, d->n_v_heads,
                     d->n_qk_heads, d->d_k, d->d_v, d->n_states_in};
    a.ws = static_cast<uint8_t *>(workspace);
    a.record = l.record;
    a.slots = static_cast<int32_t>(slots(d));
    a.near = std::max({a.p.sq, a.p.sk, a.p.sv}) <= (int64_t(1) << 23);
    a.seg = l.seg, a.seg_slots = l.seg_slots, a.seg_floats = l.seg_floats;
    a.segs = reinterpret_cast<float *>(a.ws + l.chunks);
    a.order = l.order ? reinterpret_cast<int4 *>(a.ws + l.order) : nullptr;
    const int e = d->act_dtype == STEPQ_BF16 ? 8 : 4;   // elements in 16 bytes
    const bool vec = d->d_k % 8 == 0 && (a.p.sq | a.p.sk | a.p.sv) % e == 0 && aligned(q, 16) && aligned(k, 16) && aligned(v, 16);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool delta = d->rule == STEPQ_RULE_DELTA;
    if (d->act_dtype == STEPQ_BF16) {
        if (d->d_k > 64) launch<bf16_t, 128>(a, delta, vec, s);
        else launch<bf16_t, 64>(a, delta, vec, s);
    } else {
        if (d->d_k > 64) launch<float, 128>(a, delta, vec, s);
        else launch<float, 64>(a, delta, vec, s);
    }
    return launched("prompt launch");
}
