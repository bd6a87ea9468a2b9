// Attention of single tokens over pages of quantized keys and values.
#include <algorithm>
#include <cmath>

#include "stepq_cache.h"
#include "stepq_softmax.h"

namespace stepq {
namespace {

struct CacheAttnArgs {
    CacheView c;
    const void *q;
    const int32_t *table, *lengths, *selected;   // selected NULL: all of a request's pages
    void *o;
    float *lse;
    float2 *ml;              // [parts][batch * Hq]: a part's maximum (in powers of two) and sum
    float *acc;              // [parts][batch * Hq][D]: its unnormalised output
    int32_t batch, Hq, G, max_pages, n_select, parts, chunk;
    float scale;             // times log2 e: scores are kept in powers of two
};

#ifndef CUT_WGS
#define CUT_WGS 2048
#endif
#ifndef CUT_MIN
#define CUT_MIN 256
#endif
constexpr int kTile = 32;    // keys of a wave's turn
constexpr int kMaxChunk = 2048;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
// Bytes i and j of a word as bfloat16 (exact).
__device__ __forceinline__ uint32_t bytes_of(uint32_t w, int i, int j)
{
    return pack_bf16(static_cast<float>(static_cast<int8_t>(w >> (8 * i))), static_cast<float>(static_cast<int8_t>(w >> (8 * j))));
}
// The low nibble of byte B as a sixteenth of its code (exact), and nibble j of both halves of a word so.
template <int B>
__device__ __forceinline__ float sixteenth(uint32_t w)
{
    float y;
    if constexpr (B == 0) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(y) : "v"(w));
    if constexpr (B == 1) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(y) : "v"(w));
    if constexpr (B == 2) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(y) : "v"(w));
    if constexpr (B == 3) asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(y) : "v"(w));
    return y;
}
__device__ __forceinline__ uint32_t nibbles_of(uint32_t w, int j)
{
    const uint32_t u = j % 2 ? w >> 4 : w;
    return j / 2 ? pack_bf16(sixteenth<1>(u), sixteenth<3>(u)) : pack_bf16(sixteenth<0>(u), sixteenth<2>(u));
}
// The same as bfloat16 1.5 + code / 16, put into the upper bits of a 1's mantissa with the sign turned: two
// instructions in place of 3 1/4.  Only for sums that 1.5 times the other operand may be taken off.
__device__ __forceinline__ uint32_t raised_nibbles_of(uint32_t w, int j)
{
    return ((j ? w >> (4 * j - 3) : w << 3) & 0x00780078u) ^ 0x3fc03fc0u;
}
constexpr uint32_t kRaised = 0x3fc03fc0u;           // 1.5 twice

// One of a request's key heads, 16 of its query heads, `chunk` of its tokens
// (all of them, or those of its selected pages): the waves take tiles of 32 keys
// in turn.  Scores are formed transposed, keys x queries, from codes as bfloat16
// (exact), each group's sum times its scale; values pass through LDS of the wave's
// own as codes, to be read by columns of 16 bits, 2 or 4 dimensions at once, and
// their scales go into the weights.  The next tile's codes and scales are on their way
// meanwhile, into the registers that the tile's codes have left.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(256, (sizeof(T) == 4 || (D == 256 && BITS == 4) ? (D == 256 ? 1 : 2) : D == 256 ? 2 : 3)) void cache_attn_kernel(CacheAttnArgs a)
{
    constexpr bool BF = sizeof(T) == 2;
    using Row = RowOf<D, BITS>;
    constexpr int RB = Row::bytes, NG = Row::scales, RT = kTile / 16;
    constexpr int LB = RB / 4, PB = LB < 16 ? LB : 16, PIECES = LB / PB;     // bytes of a row per lane group, in loads of PB
    constexpr int STEPS = D / 32, QP = BF ? 1 : 3, PP = BF ? 2 : 3;          // products over D; planes of queries and weights
    constexpr int VS = 32 * (RB / 32 | 1);            // a row of values in LDS: 16 rows' 32 bytes fall on all banks
    constexpr int LD = D + 4, VB = 4 * kTile * VS, SB = 16 * LD * 4;
    __shared__ alignas(16) uint8_t vs[VB > SB ? VB : SB];
    __shared__ alignas(16) float sc[4][2][NG][kTile];
    __shared__ float sm[4][16], sl[4][16];
    __shared__ int2 pages[kMaxChunk + 1];             // the chunk's pages: record (-1: none), tokens that count
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const int blocks = (a.G + 15) / 16, Hkv = a.c.Hkv, page = a.c.page;
    int x = blockIdx.x;
    const int part = x % a.parts;
    x /= a.parts;
    const int row0 = x % blocks * 16;
    x /= blocks;
    const int hk = x % Hkv, b = x / Hkv, rows = min(16, a.G - row0);
    const int len = min(max(a.lengths[b], 0), a.max_pages * page);
    const int total = a.selected ? a.n_select * page : len;
    const int from = part * a.chunk, to = min(total, from + a.chunk);
    if (part && from >= total) return;
    const int32_t *table = a.table + static_cast<size_t>(b) * a.max_pages;
    const int32_t *chosen = a.selected ? a.selected + (static_cast<size_t>(b) * Hkv + hk) * a.n_select : nullptr;
    const int first_page = page_of(from, a.c.div_page);
    if (from < to)
        for (int p = first_page + threadIdx.x, last = page_of(to - 1, a.c.div_page); p <= last; p += 256) {
            const int pos = chosen ? chosen[p] : p;
            int2 e = make_int2(-1, 0);
            if (pos >= 0 && pos < a.max_pages && pos * page < len) {
                const int id = table[pos];
                if (id >= 0 && id < a.c.n_pages) e = make_int2(id * Hkv + hk, len - pos * page);
            }
            pages[p - first_page] = e;
        }

    // queries, operand B: query n, the 8 dimensions of each step that the codes of a lane group stand for
    const size_t qrow = static_cast<size_t>(b) * a.Hq + hk * a.G + row0 + min(n, rows - 1);
    bf16x8 q[STEPS][QP];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
        // 8 bits: half st % 2 of piece st / 2; 4 bits: nibble st % 4 of piece st / 4 (D = 64: two nibbles of 4 words)
        int d0, d1;
        if constexpr (BITS == 8) d0 = st / 2 * 64 + g * 16 + st % 2 * 8, d1 = d0 + 4;
        else if constexpr (D == 64) d0 = 32 * st + 4 * g, d1 = d0 + 16;
        else d0 = st % 4 * (D / 4) + st / 4 * 32 + 8 * g, d1 = d0 + 4;
        const T *from_q = static_cast<const T *>(a.q) + qrow * D;
        if constexpr (BF) {
            const u32x2 lo = *reinterpret_cast<const u32x2 *>(from_q + d0), hi = *reinterpret_cast<const u32x2 *>(from_q + d1);
            q[st][0] = __builtin_bit_cast(bf16x8, with_sign(u32x4{lo[0], lo[1], hi[0], hi[1]}, a.scale, 0x80008000u));
        } else {
            const auto take = [&](int d) {
                return __builtin_bit_cast(f32x4, with_sign(*reinterpret_cast<const u32x4 *>(from_q + d), a.scale, 0x80000000u));
            };
            bf16x8 p[3];
            split(take(d0), take(d1), p);
#pragma unroll
            for (int i = 0; i < 3; ++i) q[st][i] = p[i];
        }
    }
    // the group that a step's dimensions lie in
    const auto group_of = [](int st) { return NG == 1 ? 0 : st % 4 * (D / 4) / kGroup4; };
    // raised codes: what 1.5 adds to each query's sums is taken off where they begin
    constexpr bool RAISED = BITS == 4 && BF;
    f32x4 qz[NG] = {};
    if constexpr (RAISED) {
        const bf16x8 zero[1] = {__builtin_bit_cast(bf16x8, (u32x4{kRaised, kRaised, kRaised, kRaised}))};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) mma(qz[group_of(st)], zero, q[st]);
#pragma unroll
        for (int m = 0; m < NG; ++m) qz[m] = -qz[m];
    }
    const auto key_nibbles = [](uint32_t w, int j) { return RAISED ? raised_nibbles_of(w, j) : nibbles_of(w, j); };
    const float scale = scale_of(a.scale);
    const auto wave_sync = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    __syncthreads();

    uint8_t *mine = vs + wave * kTile * VS;
    // a tile's key: lane l has key l % 32's record, row and whether it is there
    int64_t at = 0;
    int row = 0;
    uint32_t none = ~0u;
    const auto locate = [&](int t0) {
        const int t = t0 + lane % kTile;
        at = 0, row = 0;
        bool there = false;
        if (t < to) {
            const int p = page_of(t, a.c.div_page), r = t - p * page;
            const int2 e = pages[p - first_page];
            there = e.x >= 0 && r < e.y;
            if (there) at = static_cast<int64_t>(e.x) * a.c.record, row = r;
        }
        none = ~static_cast<uint32_t>(__ballot(there));
    };
    uint32_t kx[RT][LB / 4], vx[RT][LB / 4], sx[(NG + 1) / 2];
    const uint8_t *base[RT];
    const auto bases = [&] {
        const int64_t off = at + row * RB;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const uint32_t lo = __shfl(static_cast<int>(off), 16 * rt + n), hi = __shfl(static_cast<int>(off >> 32), 16 * rt + n);
            base[rt] = a.c.mem + static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo) + g * PB;
        }
    };
    const auto fetch = [&](uint32_t (&y)[RT][LB / 4], int behind) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int w = 0; w < PB / 4; ++w)
                    y[rt][i * (PB / 4) + w] = reinterpret_cast<const uint32_t *>(base[rt] + behind + 4 * i * PB)[w];
    };
    // lanes 0 .. 31: their key's scales; 32 .. 63: those of its value
    const auto fetch_scales = [&] {
        const uint8_t *s = a.c.mem + at + Row::scale(page, lane >= kTile, row);
        if constexpr (NG == 1) sx[0] = *reinterpret_cast<const bf16_t *>(s);
        else
#pragma unroll
            for (int m = 0; m < NG / 2; ++m) sx[m] = reinterpret_cast<const uint32_t *>(s)[m];
    };
    float m = -INFINITY, low = 0.0f, l = 0.0f;        // the maximum, what is taken off the scores, the sum
    f32x4 acc[D / 16] = {};
    const int value_at = page * RB;
    int t0 = from + wave * kTile;
    for (; t0 < to; t0 += 4 * kTile) {                // the first tile with a key
        locate(t0);
        if (none != ~0u) break;
    }
    if (t0 < to) {
        bases();
        fetch_scales();
        fetch(vx, value_at);
        fetch(kx, 0);
    }
    while (t0 < to) {
        const uint32_t gone = none;
        const bool there = !(gone >> (lane % kTile) & 1);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const float y = i % 2 ? upper_bf16(sx[i / 2]) : lower_bf16(sx[i / 2]);
            sc[wave][lane / kTile][i][lane % kTile] = there ? (BITS == 4 ? 16.0f * y : y) : 0.0f;
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                using Piece = __attribute__((ext_vector_type(PB / 4))) uint32_t;
                Piece y;
#pragma unroll
                for (int w = 0; w < PB / 4; ++w) y[w] = vx[rt][i * (PB / 4) + w];
                *reinterpret_cast<Piece *>(mine + (16 * rt + n) * VS + (4 * i + g) * PB) = y;
            }
        wave_sync();
        for (t0 += 4 * kTile; t0 < to; t0 += 4 * kTile) {
            locate(t0);
            if (none != ~0u) break;
        }
        if (t0 < to) {
            bases();
            fetch_scales();
            fetch(vx, value_at);
        }
        // scores: lane (g, n) holds keys 16 rt + 4 g .. + 3 of query n
        f32x4 s[RT];
        float top = -INFINITY;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            f32x4 y[NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) y[i] = qz[i];
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (BITS == 8) w[i] = bytes_of(kx[rt][st * 2 + i / 2], i % 2 * 2, i % 2 * 2 + 1);
                    else if constexpr (D == 64) w[i] = key_nibbles(kx[rt][i % 2], 2 * st + i / 2);
                    else w[i] = key_nibbles(kx[rt][st / 4 * 4 + i], st % 4);
                }
                const bf16x8 k[1] = {__builtin_bit_cast(bf16x8, w)};
                mma(y[group_of(st)], k, q[st]);
            }
            s[rt] = f32x4{};
#pragma unroll
            for (int i = 0; i < NG; ++i) s[rt] += y[i] * *reinterpret_cast<const f32x4 *>(&sc[wave][0][i][16 * rt + 4 * g]);
        }
        if (t0 < to) fetch(kx, 0);
        if (gone) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (gone >> (16 * rt + 4 * g + i) & 1) s[rt][i] = -INFINITY;
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[rt][i]);
        // what is taken off follows the maximum only when that has passed it by 2^6
        top = swap_max32(swap_max16(top)) * scale;
        if (__any(!(top <= low + 6.0f) || m == -INFINITY)) {
            const float to_m = fmaxf(m, top), nb = to_m == -INFINITY ? 0.0f : to_m;
            const float f = __builtin_amdgcn_exp2f(m == -INFINITY ? m : low - nb);
            l *= f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) acc[i] *= f;
            low = nb;
        }
        m = fmaxf(m, top);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[rt][i] = __builtin_amdgcn_exp2f(fmaf(s[rt][i], scale, -low));
                l += s[rt][i];
            }
        // weights times the scales of each group of dimensions, in planes
        bf16x8 p[NG][PP];
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const f32x4 y0 = s[0] * *reinterpret_cast<const f32x4 *>(&sc[wave][1][i][4 * g]);
            const f32x4 y1 = s[1] * *reinterpret_cast<const f32x4 *>(&sc[wave][1][i][16 + 4 * g]);
            if constexpr (BF) {
                const float y[8] = {y0[0], y0[1], y0[2], y0[3], y1[0], y1[1], y1[2], y1[3]};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[i][0][j] = static_cast<__bf16>(y[j]);
                    p[i][1][j] = static_cast<__bf16>(y[j] - static_cast<float>(p[i][0][j]));
                }
            } else {
                split(y0, y1, p[i]);
            }
        }
#pragma unroll
        for (int cb = 0; cb < RB / 32; ++cb) {
            uint32_t w[4];                            // 16 columns of 16 bits: keys 4 g .. + 3, then 16 + 4 g .. + 3
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x2 y = read_columns(mine + (16 * h + 4 * g + (n >> 2)) * VS + cb * 32 + (n & 3) * 8);
                w[2 * h] = y[0], w[2 * h + 1] = y[1];
            }
            constexpr int per = BITS == 8 ? 2 : 4;    // dimensions in a column
#pragma unroll
            for (int j = 0; j < per; ++j) {
                u32x4 u;
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = BITS == 8 ? bytes_of(w[i], j, j + 2) : nibbles_of(w[i], j);
                const bf16x8 v[1] = {__builtin_bit_cast(bf16x8, u)};
                mma(acc[cb * per + j], v, p[NG == 1 ? 0 : j * (D / 4) / kGroup4]);
            }
        }
        wave_sync();
    }
    // the four waves' parts: lane (g, n) holds rows 4 g .. + 3 of each tile of dimensions, of query n
    l = swap_add32(swap_add16(l));
    const float mine_m = m == -INFINITY ? m : low;
    if (g == 0) sm[wave][n] = mine_m, sl[wave][n] = l;
    __syncthreads();
    float top = -INFINITY, z = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][n]);
    const float base_m = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < 4; ++w) z += sl[w][n] * __builtin_amdgcn_exp2f(sm[w][n] - base_m);
    const float own = __builtin_amdgcn_exp2f(mine_m - base_m);
    float *sum = reinterpret_cast<float *>(vs);
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
        if (wave == w) {
#pragma unroll
            for (int tile = 0; tile < D / 16; ++tile)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = BITS == 8 ? tile / 2 * 32 + 2 * (4 * g + i) + tile % 2
                                            : tile % 4 * (D / 4) + tile / 4 * 16 + 4 * g + i;
                    float *to_d = sum + n * LD + d;
                    const float y = acc[tile][i] * own;
                    *to_d = w == 0 ? y : *to_d + y;
                }
        }
        __syncthreads();
    }
    const size_t all = static_cast<size_t>(a.batch) * a.Hq, first = static_cast<size_t>(b) * a.Hq + hk * a.G + row0;
    if (total <= a.chunk) {                           // the only part
        if (wave == 0 && g == 0) {
            sl[0][n] = z;
            if (n < rows && a.lse) a.lse[first + n] = z == 0.0f ? -INFINITY : (base_m + log2f(z)) * kLn2;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < rows * D; e += 256) {
            const float y = sl[0][e / D];
            static_cast<T *>(a.o)[first * D + e] = narrow<T>(y == 0.0f ? 0.0f : sum[e / D * LD + e % D] / y);
        }
        return;
    }
    for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
        const int r = e / (D / 4), c = e % (D / 4);
        reinterpret_cast<f32x4 *>(a.acc + (part * all + first + r) * D)[c] = *reinterpret_cast<const f32x4 *>(sum + r * LD + 4 * c);
    }
    if (wave == 0 && g == 0 && n < rows) a.ml[part * all + first + n] = make_float2(top, z);
}

stepq_status check(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    if (const stepq_status st = check_cache(c)) return st;
    if (!d) return bad("desc is NULL");
    if (d->n_q_heads < 1 || d->n_q_heads % c->n_kv_heads) return bad("n_q_heads must be a multiple of the cache's n_kv_heads, >= 1");
    if (!known_dtype(d->act_dtype)) return bad("unknown activation dtype");
    if (d->batch < 0 || d->max_pages < 0 || d->n_select < 0) return bad("negative count");
    if (!std::isfinite(d->scale)) return bad("scale must be finite");
    if (static_cast<int64_t>(std::max(d->max_pages, d->n_select)) * c->page_size >= (int64_t(1) << 30))
        return set_error(STEPQ_E_UNSUPPORTED, "2^30 tokens or more in a request's pages or in its selected ones");
    if (static_cast<int64_t>(d->batch) * d->n_q_heads > (int64_t(1) << 23))      // a launch has less than 2^32 threads
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^23 (request, head) rows in one call: split the batch");
    return STEPQ_OK;
}

// Tokens of a part (the last of a request's may have fewer), and the most parts that a request takes.
struct Cut {
    int32_t chunk, parts;
};

Cut cut_of(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    const int64_t tokens = static_cast<int64_t>(d->n_select ? d->n_select : d->max_pages) * c->page_size;
    if (d->batch == 0 || tokens == 0) return {kMaxChunk, 1};
    const int64_t G = d->n_q_heads / c->n_kv_heads, blocks = static_cast<int64_t>(d->batch) * c->n_kv_heads * ((G + 15) / 16);
    const int64_t want = std::clamp<int64_t>((blocks * tokens + CUT_WGS - 1) / CUT_WGS, CUT_MIN, kMaxChunk);
    const int64_t chunk = (want + 127) / 128 * 128;
    return {static_cast<int32_t>(chunk), static_cast<int32_t>((tokens + chunk - 1) / chunk)};
}

size_t workspace_of(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    const int parts = cut_of(c, d).parts;
    return parts == 1 ? 0 : static_cast<size_t>(d->batch) * d->n_q_heads * (c->head_dim * sizeof(float) + sizeof(float2)) * parts;
}

template <typename T, int D>
void launch(const CacheAttnArgs &a, int bits, hipStream_t st)
{
    const int64_t grid = static_cast<int64_t>(a.batch) * a.c.Hkv * ((a.G + 15) / 16) * a.parts;
    if (bits == 8) cache_attn_kernel<T, D, 8><<<dim3(static_cast<unsigned>(grid)), 256, 0, st>>>(a);
    else cache_attn_kernel<T, D, 4><<<dim3(static_cast<unsigned>(grid)), 256, 0, st>>>(a);
    if (a.parts > 1) join_parts<T, D>({a.ml, a.acc, a.o, a.lse, static_cast<size_t>(a.batch) * a.Hq, a.parts, a.selected ? nullptr : a.lengths, a.Hq,
                          a.max_pages * a.c.page, a.chunk}, st);
}

template <typename T>
void launch(const CacheAttnArgs &a, int D, int bits, hipStream_t st)
{
    if (D == 64) launch<T, 64>(a, bits, st);
    else if (D == 128) launch<T, 128>(a, bits, st);
    else launch<T, 256>(a, bits, st);
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_cache_attention_workspace(const stepq_cache_desc *c, const stepq_cache_attn_desc *d, size_t *bytes)
{
    if (const stepq_status st = check(c, d)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = workspace_of(c, d);
    return STEPQ_OK;
}

extern "C" stepq_status stepq_cache_attention(const stepq_cache_desc *c, const stepq_cache_attn_desc *d, const void *cache,
                                              const void *q, const int32_t *page_table, const int32_t *lengths,
                                              const int32_t *selected, void *o, float *lse, void *workspace,
                                              size_t workspace_bytes, void *stream)
{
    if (const stepq_status st = check(c, d)) return st;
    if (const stepq_status st = check_paged(c, cache, d->batch, d->max_pages, page_table)) return st;
    if (d->batch == 0) return STEPQ_OK;
    if (!q || !o || !lengths) return bad("NULL q, o or lengths");
    if (!aligned(q, 16) || !aligned(o, d->act_dtype == STEPQ_F32 ? 4 : 2)) return bad("q must be 16-byte aligned, o to its type");
    if (d->n_select && !selected) return bad("selected is NULL");
    const size_t need = workspace_of(c, d);
    if (need && (!workspace || workspace_bytes < need)) return bad("workspace is smaller than stepq_cache_attention_workspace()");
    if (!aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
    const size_t rows = static_cast<size_t>(d->batch) * d->n_q_heads;
    const Cut cut = cut_of(c, d);
    CacheAttnArgs a{};
    a.c = cache_view(c, cache);
    a.q = q, a.table = page_table, a.lengths = lengths, a.selected = d->n_select ? selected : nullptr;
    a.o = o, a.lse = lse;
    a.batch = d->batch, a.Hq = d->n_q_heads, a.G = d->n_q_heads / c->n_kv_heads;
    a.max_pages = d->max_pages, a.n_select = d->n_select, a.parts = cut.parts, a.chunk = cut.chunk;
    a.acc = static_cast<float *>(workspace);
    if (need) a.ml = reinterpret_cast<float2 *>(a.acc + rows * c->head_dim * a.parts);
    a.scale = d->scale * 1.4426950408889634f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->act_dtype == STEPQ_BF16) launch<bf16_t>(a, c->head_dim, c->bits, s);
    else launch<float>(a, c->head_dim, c->bits, s);
    return launched("cache attention launch");
}
