// Attention of single tokens over a shared prefix and each request's own pages.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "stepq_softmax.h"

namespace stepq {
namespace {

using f32x16 = __attribute__((ext_vector_type(16))) float;

struct AttnArgs {
    const void *q, *k, *v;
    const int32_t *prefix_pages, *table, *lengths;
    void *o;
    float *lse;
    float2 *ml;              // [parts][batch * Hq]: a part's maximum (in powers of two) and sum
    float *acc;              // [parts][batch * Hq][D]: its unnormalised output
    int64_t prefix;
    int32_t batch, Hq, Hkv, G, n_pages, page, max_pages;
    int32_t prefix_parts, own_parts;   // parts 0 .. prefix_parts - 1 of the prefix, then the requests' own
    int32_t prefix_items;    // workgroups of attn_rows_kernel that read the prefix (0: attn_prefix_kernel does)
    FastDiv div_page;
    float scale;             // times log2 e: scores are kept in powers of two
};

// Row of the caches ([n_pages * Hkv * page][D]) of token t of `pages`; -1: none.
__device__ __forceinline__ int token_row(const AttnArgs &a, const int32_t *pages, int t, int hk, bool valid)
{
    if (!valid) return -1;
    const int p = fdiv(t, a.div_page), id = pages[p];
    return id >= 0 && id < a.n_pages ? (id * a.Hkv + hk) * a.page + (t - p * a.page) : -1;
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

// ---------------------------------------------------------------------------
// Few queries per key: a workgroup takes 16 query rows (the group's heads of
// one request over a range of its own tokens, or 16 rows of all requests over a
// range of the prefix) and its waves take key tiles in turn.  Scores are formed
// transposed, keys x queries, so that a query's weights lie in one lane group
// and go into the second product as they are; values pass through LDS of the
// wave's own to be read by columns.  Bound by the bytes of the caches: 64
// requests x 8 key/value heads x 1-1024 tokens of 128 bfloat16 (134 MB) in 28.5 us,
// 4.7 TB/s.  512 x 2 x 1-256 tokens of 256 (134 MB) take 50 us, 2.7 TB/s: a wave
// has one tile or two there, and its registers (400) leave 4 waves a CU to wait
// with; at 256 registers they spill.  4 requests over 512 + 64 tokens: 6.6 us, latency.
template <typename T>
struct Tile;
template <>
struct Tile<bf16_t> {
    static constexpr int keys = 32;
};
template <>
struct Tile<float> {
    static constexpr int keys = 16;
};

template <typename T, int D>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void attn_rows_kernel(AttnArgs a)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KT = Tile<T>::keys, RB = D * static_cast<int>(sizeof(T)), SL = RB / 16;   // bytes and 16-byte slots of a row
    constexpr int RT = KT / 16;                       // row blocks of keys
    constexpr int QF = RB / 64;                       // 16-byte pieces of a row per lane group: operand reads
    constexpr int VL = KT * SL / 64;                  // 16-byte loads of values per lane
    constexpr int SW = SL < 16 ? 128 : 256;
    __shared__ alignas(16) uint8_t vs[4][KT * RB];
    __shared__ float sm[4][16], sl[4][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    int x = blockIdx.x, part, hk, row0, rows, from, to;
    const int32_t *pages;
    if (x < a.prefix_items) {
        const int blocks = (a.batch * a.G + 15) / 16;
        hk = x % a.Hkv, x /= a.Hkv;
        row0 = x % blocks * 16, part = x / blocks;
        rows = a.batch * a.G;
        pages = a.prefix_pages;
        const int len = static_cast<int>(a.prefix), step = ((len + a.prefix_parts - 1) / a.prefix_parts + KT - 1) / KT * KT;
        from = min(len, part * step), to = min(len, from + step);
    } else {
        x -= a.prefix_items;
        const int blocks = (a.G + 15) / 16;
        part = x % a.own_parts, x /= a.own_parts;
        row0 = x % blocks * 16, x /= blocks;
        hk = x % a.Hkv;
        const int b = x / a.Hkv;
        rows = a.G;
        pages = a.table + static_cast<size_t>(b) * a.max_pages;
        const int len = min(max(a.lengths[b], 0), a.max_pages * a.page);
        const int step = ((len + a.own_parts - 1) / a.own_parts + KT - 1) / KT * KT;
        from = min(len, part * step), to = min(len, from + step);
        row0 += b * a.G;
        rows += b * a.G;
        part += a.prefix_parts;
    }
    // row r of (all requests, group) is request r / G, head r % G of the group
    const bool live = row0 + n < rows;
    const int rr = live ? row0 + n : row0, rb = rr / a.G;
    const size_t qrow = static_cast<size_t>(rb) * a.Hq + hk * a.G + (rr - rb * a.G);
    using Piece = std::conditional_t<BF, bf16x8, f32x4>;
    Piece q[QF];
#pragma unroll
    for (int i = 0; i < QF; ++i)
        q[i] = __builtin_bit_cast(Piece, with_sign(reinterpret_cast<const u32x4 *>(static_cast<const T *>(a.q) + qrow * D)[4 * i + g],
                                                   a.scale, BF ? 0x80008000u : 0x80000000u));
    const float scale = scale_of(a.scale);

    const uint8_t *K = static_cast<const uint8_t *>(a.k), *V = static_cast<const uint8_t *>(a.v);
    Running run;
    f32x4 acc[D / 16] = {};
    Piece kx[RT][QF];
    int at = -1;                 // lane l < KT: the cache row of key l of the tile whose keys are in kx
    const auto rows_of = [&](int t0) { return token_row(a, pages, t0 + lane, hk, lane < KT && t0 + lane < to); };
    const auto fetch_keys = [&] {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int r = max(__shfl(at, 16 * rt + n), 0);
#pragma unroll
            for (int i = 0; i < QF; ++i)
                kx[rt][i] = reinterpret_cast<const Piece *>(K + static_cast<size_t>(r) * RB)[4 * i + g];
        }
    };
    int t0 = from + wave * KT;
    int next_at = t0 < to ? rows_of(t0) : -1;
    if (t0 < to) at = next_at, fetch_keys();
    for (; t0 < to; t0 += 4 * KT) {
        // the tile's values, and the rows of the next tile
        u32x4 vx[VL];
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int piece = i * 64 + lane, row = piece / SL, r = __shfl(at, row);
            const u32x4 y = *reinterpret_cast<const u32x4 *>(V + static_cast<size_t>(max(r, 0)) * RB + piece % SL * 16);
            vx[i] = r >= 0 ? y : u32x4{};
        }
        const bool more = t0 + 4 * KT < to;
        if (more) next_at = rows_of(t0 + 4 * KT);
        // scores: lane (g, n) holds keys 16 rt + 4 g .. + 3 of query n
        f32x4 s[RT];
        float top = -INFINITY;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            s[rt] = f32x4{};
#pragma unroll
            for (int i = 0; i < QF; ++i) {
                if constexpr (BF) {
                    s[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kx[rt][i], q[i], s[rt], 0, 0, 0);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kx[rt][i][r], q[i][r], s[rt], 0, 0, 0);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool none = __shfl(at, 16 * rt + 4 * g + r) < 0;
                if (none) s[rt][r] = -INFINITY;
                top = fmaxf(top, s[rt][r]);
            }
        }
        if (more) at = next_at, fetch_keys();
        const float f = run.next(swap_max32(swap_max16(top)) * scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[rt][r] = __builtin_amdgcn_exp2f(fmaf(s[rt][r], scale, -run.base));
                run.l += s[rt][r];
            }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int piece = i * 64 + lane, row = piece / SL, slot = piece % SL;
            *reinterpret_cast<u32x4 *>(&vs[wave][row * RB + ((slot ^ (BF ? swizzle<SW>(row) : row & 3)) * 16)]) = vx[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        if constexpr (BF) {
            // the weights in two bfloat16 planes (16 bits): their rounding is then far below the output's
            bf16x8 p[2];
            {
                float y[8] = {s[0][0], s[0][1], s[0][2], s[0][3], s[RT - 1][0], s[RT - 1][1], s[RT - 1][2], s[RT - 1][3]};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[0][i] = static_cast<__bf16>(y[i]);
                    p[1][i] = static_cast<__bf16>(y[i] - static_cast<float>(p[0][i]));
                }
            }
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                u32x4 w;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = 16 * h + 4 * g + (n >> 2), slot = 2 * dt + ((n & 3) >> 1);
                    const u32x2 y = read_columns(&vs[wave][row * RB + ((slot ^ swizzle<SW>(row)) * 16) + 8 * (n & 1)]);
                    w[2 * h] = y[0], w[2 * h + 1] = y[1];
                }
                const bf16x8 v = __builtin_bit_cast(bf16x8, w);
                acc[dt] *= f;
#pragma unroll
                for (int i = 1; i >= 0; --i) acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[i], acc[dt], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                acc[dt] *= f;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int row = 4 * g + r, slot = 4 * dt + (n >> 2);
                    const float v = *reinterpret_cast<const float *>(&vs[wave][row * RB + ((slot ^ (row & 3)) * 16) + (n & 3) * 4]);
                    acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[0][r], acc[dt], 0, 0, 0);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    // the four waves' parts: lane (g, n) holds dimensions 16 dt + 4 g .. + 3 of query n
    run.l = swap_add32(swap_add16(run.l));
    if (g == 0) sm[wave][n] = run.m, sl[wave][n] = run.l;
    __syncthreads();
    float top = -INFINITY, z = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][n]);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < 4; ++w) z += sl[w][n] * __builtin_amdgcn_exp2f(sm[w][n] - base);
    const float mine = __builtin_amdgcn_exp2f(run.m - base);
    constexpr int LD = D + 4;
    static_assert(16 * LD * 4 <= static_cast<int>(sizeof(vs)), "the sum fits the values' place");
    float *sum = reinterpret_cast<float *>(vs);
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
        if (wave == w)
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) {
                f32x4 *to4 = reinterpret_cast<f32x4 *>(sum + n * LD + 16 * dt + 4 * g);
                const f32x4 y = acc[dt] * mine;
                *to4 = w == 0 ? y : *to4 + y;
            }
        __syncthreads();
    }
    const size_t total = static_cast<size_t>(a.batch) * a.Hq;
    for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
        const int r = e / (D / 4), c = e % (D / 4);
        if (row0 + r < rows) {
            const int b = (row0 + r) / a.G;
            const size_t at_row = part * total + static_cast<size_t>(b) * a.Hq + hk * a.G + (row0 + r - b * a.G);
            reinterpret_cast<f32x4 *>(a.acc + at_row * D)[c] = *reinterpret_cast<const f32x4 *>(sum + r * LD + 4 * c);
        }
    }
    if (wave == 0 && g == 0 && live) a.ml[part * total + qrow] = make_float2(top, z);
}

// ---------------------------------------------------------------------------
// Many queries per key: the prefix of a large batch, a matrix product.  A
// workgroup takes 256 query rows (32 to a wave, their queries in registers) and
// a range of the prefix, 64 (D = 256: 32) keys at a time, in two LDS buffers by
// turns, so that a tile costs one barrier and waves may be a tile's phase apart;
// the tile after the next is on its way in registers, with the page ids of the
// one after that: nothing waits for a load of its own tile.  Rows in LDS are
// padded, which makes every address a lane's base and a constant.  Scores
// transposed as above, in 32x32 blocks.  The running maximum follows only when
// it is passed by 2^6, so that the outputs are rescaled a few times in all.  The
// weights go into the second product in two bfloat16 planes (16 bits), as in
// attn_rows_kernel: a request gets the same precision in any batch.  In one plane
// (8 bits) 512 requests over 16384 tokens of 256 took 212 us in all, not 262, and
// the error of o was 2.2e-3, not the 1.7e-3 of its own rounding.
//   Bound by the matrix cores and the LDS reads that feed them (D = 256: the
// queries and the output fill the registers, so a key block read from LDS serves
// 32 queries only, and both take the same time at their best).  4096 rows a head
// x 16384 tokens x 256, 2 heads: 137 GFLOP in 193 us, 0.71 PFLOP/s, 0.57 of a
// large library product's rate (a half more with the weights' second plane, which
// the matrix cores compute too); 256 rows x 4096 x 128, 8 heads (the queries of 64
// requests): 21 us.
template <int D>
__global__ __launch_bounds__(512, 2) void attn_prefix_kernel(AttnArgs a)
{
    constexpr int KT = D == 256 ? 32 : 64;            // as many as the registers of 2 waves per SIMD allow
    constexpr int KK = KT / 32, RB = 2 * D, SL = RB / 16, L = KT * SL / 512, KB = D / 16, DT = D / 32;
    // rows in LDS: 16 keys one 16-byte slot apart, and 4 rows of values read by columns 64 bytes apart, fill the banks
    constexpr int KR = RB + 16, VR = RB + 64;
    __shared__ alignas(16) uint8_t ks[2][KT * KR], vs[2][KT * VR];
    __shared__ uint8_t missing[3][KT];                // of tile t in t % 3: written two tiles ahead
    int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int lane = tid & 63, h = lane >> 5, n = lane & 31;
    // Addresses in LDS are formed again for each use, not kept in registers.
    const auto again = [&] {
        asm volatile("" : "+v"(lane), "+v"(tid));
        h = lane >> 5, n = lane & 31;
    };
    const int rows = a.batch * a.G, tiles = (rows + 255) / 256, pieces = a.Hkv * a.prefix_parts;
    // pieces of the prefix stay on one XCD, whose cache then serves all query tiles that read them
    int piece, tile;
    if (pieces % 8 == 0) piece = blockIdx.x % 8 + 8 * (blockIdx.x / 8 / tiles), tile = blockIdx.x / 8 % tiles;
    else piece = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int hk = piece % a.Hkv, part = piece / a.Hkv;
    const int len = static_cast<int>(a.prefix), step = ((len + a.prefix_parts - 1) / a.prefix_parts + KT - 1) / KT * KT;
    const int from = min(len, part * step), to = min(len, from + step);
    const auto query_row = [&](int row) {
        const int b = row / a.G;
        return static_cast<size_t>(b) * a.Hq + hk * a.G + (row - b * a.G);
    };
    const size_t qrow = query_row(min(tile * 256 + wave * 32 + n, rows - 1));
    // operand B: query n, elements 16 kb + 8 h .. + 7
    bf16x8 q[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
        q[kb] = reinterpret_cast<const bf16x8 *>(static_cast<const bf16_t *>(a.q) + qrow * D)[2 * kb + h];
    const float scale = scale_of(a.scale);
    if (!(a.scale > 0.0f))
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
            q[kb] = __builtin_bit_cast(bf16x8, with_sign(__builtin_bit_cast(u32x4, q[kb]), a.scale, 0x80008000u));
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) asm volatile("" : "+v"(q[kb]));   // there before the loop: nothing in it waits for them
    const uint8_t *K = static_cast<const uint8_t *>(a.k), *V = static_cast<const uint8_t *>(a.v);
    // a thread's 16-byte pieces of the next tile, on their way with the page ids of the tile after it
    u32x4 kx[L], vx[L];
    int id[L];
    uint64_t gone[L];            // lanes whose key there is not: their values are made 0
    const auto token = [&](int i) { return (i * 512 + tid) / SL; };
    const auto ids_of = [&](int t0) {
#pragma unroll
        for (int i = 0; i < L; ++i) id[i] = a.prefix_pages[fdiv(min(t0 + token(i), to - 1), a.div_page)];
    };
    const auto fetch = [&](int t0, int ring) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int t = t0 + token(i), slot = (i * 512 + tid) % SL;
            const bool there = t < to && id[i] >= 0 && id[i] < a.n_pages;
            const int row = there ? (id[i] * a.Hkv + hk) * a.page + t - fdiv(t, a.div_page) * a.page : 0;
            const size_t from_byte = static_cast<size_t>(row) * RB + slot * 16;
            kx[i] = *reinterpret_cast<const u32x4 *>(K + from_byte);
            vx[i] = *reinterpret_cast<const u32x4 *>(V + from_byte);
            gone[i] = __ballot(!there);
            if (slot == 0) missing[ring][token(i)] = !there;
        }
    };
    const auto store = [&](int buf) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (gone[i] && (gone[i] >> lane & 1)) vx[i] = u32x4{};
            const int kr = token(i), slot = (i * 512 + tid) % SL;
            *reinterpret_cast<u32x4 *>(ks[buf] + kr * KR + slot * 16) = kx[i];
            *reinterpret_cast<u32x4 *>(vs[buf] + kr * VR + slot * 16) = vx[i];
        }
    };
    f32x16 acc[DT] = {};
    float m = -INFINITY, base = 0.0f, l = 0.0f;
    if (from < to) {
        ids_of(from);
        fetch(from, 0);
        ids_of(from + KT);
        store(0);
        if (from + KT < to) {
            fetch(from + KT, 1);
            ids_of(from + 2 * KT);
        }
    }
    int buf = 0, ring = 0;
    for (int t0 = from; t0 < to; t0 += KT, buf ^= 1, ring = ring == 2 ? 0 : ring + 1) {
        lds_barrier();
        again();
        const uint8_t *kb0 = ks[buf] + n * KR + h * 16;
        // scores: lane (h, n) holds keys 32 kt + 8 (r / 4) + 4 h + r % 4 of query n
        f32x16 s[KK];
#pragma unroll
        for (int kt = 0; kt < KK; ++kt) {
            s[kt] = f32x16{};
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const bf16x8 k = *reinterpret_cast<const bf16x8 *>(kb0 + 32 * kt * KR + kb * 32);
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[kb], s[kt], 0, 0, 0);
            }
        }
        reads_ahead<KK * KB, 1, 1, 3>();
        float top = -INFINITY;
        const uint64_t none = __ballot(missing[ring][lane % KT] != 0);
        if (none) {
#pragma unroll
            for (int kt = 0; kt < KK; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (none >> (32 * kt + 8 * (r / 4) + 4 * h + r % 4) & 1) s[kt][r] = -INFINITY;
        }
#pragma unroll
        for (int kt = 0; kt < KK; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kt][r]);
        top = swap_max32(top) * scale;
        if (__any(!(top <= base + 6.0f)) || m == -INFINITY) {
            const float to_m = fmaxf(m, top), nb = to_m == -INFINITY ? 0.0f : to_m, f = __builtin_amdgcn_exp2f(m == -INFINITY ? m : base - nb);
            l *= f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[dt] *= f;
            base = nb;
        }
        m = fmaxf(m, top);
        bf16x8 p[2][2 * KK];
#pragma unroll
        for (int kt = 0; kt < KK; ++kt)
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                const f32x2 e = {__builtin_amdgcn_exp2f(fmaf(s[kt][r], scale, -base)),
                                 __builtin_amdgcn_exp2f(fmaf(s[kt][r + 1], scale, -base))};
                l += e[0] + e[1];
                const bf16x2 w = __builtin_convertvector(e, bf16x2);
                const bf16x2 x = __builtin_convertvector((f32x2{e[0] - static_cast<float>(w[0]), e[1] - static_cast<float>(w[1])}), bf16x2);
                const int i = 2 * kt + r / 8;
                p[0][i][r % 8] = w[0], p[0][i][r % 8 + 1] = w[1];
                p[1][i][r % 8] = x[0], p[1][i][r % 8 + 1] = x[1];
            }
#pragma unroll
        for (int i = 0; i < 2 * KK; ++i) asm volatile("" : "+v"(p[0][i]), "+v"(p[1][i]));   // formed here, not after the next tile's loads
        if (t0 + KT < to) {
            again();
            store(buf ^ 1);
            if (t0 + 2 * KT < to) {
                again();
                fetch(t0 + 2 * KT, ring == 0 ? 2 : ring - 1);
                ids_of(t0 + 3 * KT);
            }
        }
        again();
        const uint8_t *vb0 = vs[buf] + (4 * h + (lane & 15) / 4) * VR + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
        // O^T += V^T P: summation slot 8 h + 4 u + j of a block of 16 keys is key 8 u + 4 h + j
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int kb = 0; kb < 2 * KK; ++kb) {
                u32x4 w;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const u32x2 y = read_columns(vb0 + (16 * kb + 8 * u) * VR + dt * 64);
                    w[2 * u] = y[0], w[2 * u + 1] = y[1];
                }
#pragma unroll
                for (int i = 1; i >= 0; --i)
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), p[i][kb], acc[dt], 0, 0, 0);
            }
        reads_ahead<DT * 2 * KK, 2, 2, 2>();
    }
    l = swap_add32(l);
    again();
    const int row = tile * 256 + wave * 32 + n;
    if (row < rows) {
        const size_t at = part * (static_cast<size_t>(a.batch) * a.Hq) + query_row(row);
        if (h == 0) a.ml[at] = make_float2(m == -INFINITY ? m : base, l);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4 *>(a.acc + at * D + 32 * dt + 2 * r + 4 * h) =
                    f32x4{acc[dt][r], acc[dt][r + 1], acc[dt][r + 2], acc[dt][r + 3]};
    }
}

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
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    constexpr int E = D / 64, U = 4;
    using Piece = __attribute__((ext_vector_type(E))) float;
    __shared__ alignas(16) float sum[4][D];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = w % W, lane = threadIdx.x & 63;
    const size_t total = static_cast<size_t>(a.batch) * a.Hq, row = static_cast<size_t>(blockIdx.x) * (4 / W) + w / W;
    if (W == 1 && row >= total) return;
    const int parts = a.prefix_parts + a.own_parts;
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

stepq_status check(const stepq_attn_desc *d)
{
    if (!d) return bad("desc is NULL");
    if (d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads)
        return bad("head counts must be >= 1 and n_q_heads a multiple of n_kv_heads");
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
        return set_error(STEPQ_E_UNSUPPORTED, "head_dim must be 64, 128 or 256");
    if (!known_dtype(d->act_dtype)) return bad("unknown activation dtype");
    if (d->batch < 0 || d->n_pages < 0 || d->max_pages < 0 || d->prefix_len < 0) return bad("negative count");
    if (d->page_size < 1) return bad("page_size must be >= 1");
    if (!std::isfinite(d->scale)) return bad("scale must be finite");
    if (d->prefix_len >= (int64_t(1) << 30) || static_cast<int64_t>(d->max_pages) * d->page_size >= (int64_t(1) << 30))
        return set_error(STEPQ_E_UNSUPPORTED, "2^30 tokens or more in the prefix or a request's pages");
    if (static_cast<int64_t>(d->batch) * d->n_q_heads > (int64_t(1) << 23))      // a launch has less than 2^32 threads
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^23 (request, head) rows in one call: split the batch");
    if (static_cast<double>(d->n_pages) * d->n_kv_heads * d->page_size >= 2147483648.0)
        return set_error(STEPQ_E_UNSUPPORTED, "2^31 rows or more in a cache");
    return STEPQ_OK;
}

// How the keys are split over workgroups.
struct Split {
    int prefix_parts, own_parts, prefix_items;
    bool product;            // the prefix by attn_prefix_kernel
};

Split split_of(const stepq_attn_desc *d)
{
    Split s{};
    if (d->batch == 0) return s;
    const int64_t G = d->n_q_heads / d->n_kv_heads, rows = d->batch * G;
    const auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    // attn_rows_kernel: two workgroups a CU, of ranges of 128 keys or more (a tile per wave), 256 where there would be
    // more than 16, whose join costs more than the shorter ranges save: 4 requests over 512 + 64 tokens 10.9 us at 256, 9.6
    // at 128; one over 4096 + 1024 11.8 and 13.1, over 16384 20 and 28; 64 is slower than 128 from 1024 tokens on
    const auto ranges = [&](int64_t blocks, int64_t len) {
        const int64_t want = std::clamp<int64_t>(ceil_div(512, blocks), 1, std::max<int64_t>(1, ceil_div(len, 128)));
        return want <= 16 ? want : std::max<int64_t>(16, std::min(want, ceil_div(len, 256)));
    };
    if (d->prefix_len) {
        // attn_rows_kernel reads the prefix once for every 16 rows; the product reads it once for 256 and computes
        // 256 however few there are.  It pays where more than 130 MB are read again, and from 33 rows on at D = 256
        // (whose rows take most registers in the other kernel), 65 otherwise.  Whole calls, rows / product, us:
        //   D = 256, 2 heads, 134 MB of prefix: 4 rows 47 / 62, 32 65 / 63, 48 93 / 65, 128 121 / 72, 512 385 / 129;
        //     8 heads, 67 MB: 32 37 / 41, 48 45 / 42 (134 MB again), 64 51 / 43; 17 MB: 128 42 / 43 (119 MB), 256 57 / 54
        //   D = 128, 8 heads, 268 MB: 4 52 / 108, 32 58 / 114, 64 95 / 115, 128 169 / 120; 17 MB: 128 25 / 29, 256 35 /
        //     32; 1 head, 134 MB: 48 74 / 70, 64 92 / 70, 128 167 / 73
        //   D = 64, 2 heads, 134 MB: 4 37 / 90, 48 71 / 82, 64 86 / 82, 128 106 / 83; 17 MB: 128 22 / 29, 256 32 / 31
        const double again = static_cast<double>(ceil_div(rows, 16) - 1) * d->prefix_len * d->n_kv_heads * d->head_dim * 4;
        s.product = d->act_dtype == STEPQ_BF16 && again > 130e6 && rows > (d->head_dim == 256 ? 32 : 64);
        const int64_t blocks = d->n_kv_heads * ceil_div(rows, s.product ? 256 : 16), most = ceil_div(d->prefix_len, 256);
        int64_t parts = s.product ? std::clamp<int64_t>(ceil_div(256, blocks), 1, most) : ranges(blocks, d->prefix_len);
        // whole rounds of the 8 XCDs where that costs few parts
        if (s.product)
            while (parts < most && d->n_kv_heads * parts % 8 != 0 && parts < 2 * ceil_div(256, blocks)) ++parts;
        s.prefix_parts = static_cast<int>(parts);
        if (!s.product) s.prefix_items = static_cast<int>(blocks * parts);
    }
    s.own_parts = static_cast<int>(ranges(d->batch * static_cast<int64_t>(d->n_kv_heads) * ceil_div(G, 16),
                                          static_cast<int64_t>(d->max_pages) * d->page_size));
    return s;
}

size_t part_bytes(const stepq_attn_desc *d)
{
    return static_cast<size_t>(d->batch) * d->n_q_heads * (d->head_dim * sizeof(float) + sizeof(float2));
}

template <typename T, int D>
void launch(AttnArgs a, const Split &s, hipStream_t st)
{
    const int blocks = (a.G + 15) / 16;
    const int64_t own = static_cast<int64_t>(a.batch) * a.Hkv * blocks * a.own_parts;
    if constexpr (sizeof(T) == 2)
        if (s.product) {
            const int64_t grid = static_cast<int64_t>((a.batch * a.G + 255) / 256) * a.Hkv * a.prefix_parts;
            attn_prefix_kernel<D><<<dim3(static_cast<unsigned>(grid)), 512, 0, st>>>(a);
        }
    attn_rows_kernel<T, D><<<dim3(static_cast<unsigned>(a.prefix_items + own)), 256, 0, st>>>(a);
    const unsigned rows = static_cast<unsigned>(a.batch) * a.Hq;
    if (rows <= 1024) attn_join_kernel<T, D, 4><<<dim3(rows), 256, 0, st>>>(a);
    else attn_join_kernel<T, D, 1><<<dim3((rows + 3) / 4), 256, 0, st>>>(a);
}

template <typename T>
void launch(const AttnArgs &a, const Split &s, int D, hipStream_t st)
{
    if (D == 64) launch<T, 64>(a, s, st);
    else if (D == 128) launch<T, 128>(a, s, st);
    else launch<T, 256>(a, s, st);
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_prefix_attention_workspace(const stepq_attn_desc *d, size_t *bytes)
{
    if (const stepq_status st = check(d)) return st;
    if (!bytes) return bad("bytes is NULL");
    const Split s = split_of(d);
    *bytes = d->batch ? part_bytes(d) * (s.prefix_parts + s.own_parts) : 0;
    return STEPQ_OK;
}

extern "C" stepq_status stepq_prefix_attention(const stepq_attn_desc *d, const void *q, const void *k_cache,
                                               const void *v_cache, const int32_t *prefix_pages,
                                               const int32_t *page_table, const int32_t *lengths, void *o, float *lse,
                                               void *workspace, size_t workspace_bytes, void *stream)
{
    if (const stepq_status st = check(d)) return st;
    if (d->batch == 0) return STEPQ_OK;
    if (!q || !o || !lengths) return bad("NULL q, o or lengths");
    if (d->n_pages && (!k_cache || !v_cache)) return bad("NULL cache");
    if (d->prefix_len && !prefix_pages) return bad("prefix_pages is NULL");
    if (d->max_pages && !page_table) return bad("page_table is NULL");
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16))
        return bad("q and the caches must be 16-byte aligned");
    const Split sp = split_of(d);
    const size_t need = part_bytes(d) * (sp.prefix_parts + sp.own_parts);
    if (!workspace || workspace_bytes < need) return bad("workspace is smaller than stepq_prefix_attention_workspace()");
    if (!aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
    const size_t rows = static_cast<size_t>(d->batch) * d->n_q_heads;
    AttnArgs a{};
    a.q = q, a.k = k_cache, a.v = v_cache;
    // what is not there is read as row 0 and left out; without a page, the queries stand in for that row
    if (d->n_pages == 0) a.k = a.v = q;
    a.prefix_pages = prefix_pages, a.table = page_table, a.lengths = lengths;
    a.o = o, a.lse = lse;
    a.acc = static_cast<float *>(workspace);
    a.ml = reinterpret_cast<float2 *>(a.acc + rows * d->head_dim * (sp.prefix_parts + sp.own_parts));
    a.prefix = d->prefix_len;
    a.batch = d->batch, a.Hq = d->n_q_heads, a.Hkv = d->n_kv_heads, a.G = d->n_q_heads / d->n_kv_heads;
    a.n_pages = d->n_pages, a.page = d->page_size, a.max_pages = d->max_pages;
    a.prefix_parts = sp.prefix_parts, a.own_parts = sp.own_parts, a.prefix_items = sp.prefix_items;
    a.div_page = fast_div(static_cast<uint32_t>(d->page_size));
    a.scale = d->scale * 1.4426950408889634f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->act_dtype == STEPQ_BF16) launch<bf16_t>(a, sp, d->head_dim, s);
    else launch<float>(a, sp, d->head_dim, s);
    return launched("prefix attention launch");
}
