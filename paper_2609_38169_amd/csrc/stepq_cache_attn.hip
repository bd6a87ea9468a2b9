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
    int32_t batch, Hq, G, max_pages, n_select, parts;
    float scale;             // times log2 e: scores are kept in powers of two
};

constexpr int kTile = 32;    // keys of a wave's turn

// Eight codes as bfloat16 (exact).  8 bits: the bytes of two words; 4 bits: nibble j of four pairs of words, where
// the pairs lie 16 bits apart.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ float byte_of(uint32_t w, int i) { return static_cast<float>(static_cast<int8_t>(w >> (8 * i))); }
__device__ __forceinline__ float nibble_of(uint32_t w, int i)
{
    return static_cast<float>(static_cast<int32_t>(w << (28 - 4 * i)) >> 28);
}

// One of a request's key heads, 16 of its query heads, one range of its tokens
// (all of them, or those of its selected pages): the waves take tiles of 32 keys
// in turn.  Scores are formed transposed, keys x queries, from codes as bfloat16
// (exact), each group's sum times its scale; values pass through LDS of the wave's
// own as codes, to be read by columns of 16 bits, 2 or 4 dimensions at once, and
// their scales go into the weights.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(256, 1) void cache_attn_kernel(CacheAttnArgs a)
{
    constexpr bool BF = sizeof(T) == 2;
    using Row = RowOf<D, BITS>;
    constexpr int RB = Row::bytes, NG = Row::scales, RT = kTile / 16;
    constexpr int LB = RB / 4, PB = LB < 16 ? LB : 16, PIECES = LB / PB;     // bytes of a row per lane group, in loads of PB
    constexpr int STEPS = D / 32, QP = BF ? 1 : 3, PP = BF ? 2 : 3;          // products over D; planes of queries and weights
    constexpr int VL = kTile * RB / 16 / 64;          // 16-byte loads of values per lane
    constexpr int VS = 32 * (RB / 32 | 1);            // a row of values in LDS: 16 rows' 32 bytes fall on all banks
    constexpr int LD = D + 4, VB = 4 * kTile * VS, SB = 16 * LD * 4;
    __shared__ alignas(16) uint8_t vs[VB > SB ? VB : SB];
    __shared__ alignas(16) float sc[4][2][NG][kTile];
    __shared__ float sm[4][16], sl[4][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const int blocks = (a.G + 15) / 16, Hkv = a.c.Hkv, page = a.c.page;
    int x = blockIdx.x;
    const int part = x % a.parts;
    x /= a.parts;
    const int row0 = x % blocks * 16;
    x /= blocks;
    const int hk = x % Hkv, b = x / Hkv, rows = min(16, a.G - row0);
    const int32_t *table = a.table + static_cast<size_t>(b) * a.max_pages;
    const int32_t *chosen = a.selected ? a.selected + (static_cast<size_t>(b) * Hkv + hk) * a.n_select : nullptr;
    const int len = min(max(a.lengths[b], 0), a.max_pages * page);
    const int total = chosen ? a.n_select * page : len;
    const int step = ((total + a.parts - 1) / a.parts + kTile - 1) / kTile * kTile;
    const int from = min(total, part * step), to = min(total, from + step);

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
    const float scale = scale_of(a.scale);
    const auto wave_sync = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };

    uint8_t *mine = vs + wave * kTile * VS;
    Running run;
    f32x4 acc[D / 16] = {};
    for (int t0 = from + wave * kTile; t0 < to; t0 += 4 * kTile) {
        // lane l < 32: the record and row of key l; none: row 0 of the cache stands in, its scales 0
        int64_t at = 0;
        int r = 0;
        bool there = false;
        if (lane < kTile && t0 + lane < to) {
            const int t = t0 + lane, p = page_of(t, a.c.div_page);
            r = t - p * page;
            const int pos = chosen ? chosen[p] : p;
            if (pos >= 0 && pos < a.max_pages && pos * page + r < len) {
                const int id = table[pos];
                there = id >= 0 && id < a.c.n_pages;
                if (there) at = (static_cast<int64_t>(id) * Hkv + hk) * a.c.record;
            }
        }
        const uint32_t none = ~static_cast<uint32_t>(__ballot(there));
        if (none == ~0u) continue;
        if (!there) at = 0, r = 0;
        const auto base_of = [&](int key) {
            const uint32_t lo = __shfl(static_cast<int>(at), key), hi = __shfl(static_cast<int>(at >> 32), key);
            return a.c.mem + (static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo));
        };
        wave_sync();
        if (lane < kTile) {
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const bf16_t *s = reinterpret_cast<const bf16_t *>(a.c.mem + at + Row::scale(page, kv, r));
#pragma unroll
                for (int m = 0; m < NG; ++m) sc[wave][kv][m][lane] = there ? widen(s[m]) : 0.0f;
            }
        }
        uint32_t kx[RT][LB / 4];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int key = 16 * rt + n;
            const uint8_t *row = base_of(key) + Row::codes(page, false, __shfl(r, key));
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int w = 0; w < PB / 4; ++w)
                    kx[rt][i * (PB / 4) + w] = reinterpret_cast<const uint32_t *>(row + (4 * i + g) * PB)[w];
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int piece = i * 64 + lane, key = piece / (RB / 16), slot = piece % (RB / 16);
            const uint8_t *row = base_of(key) + Row::codes(page, true, __shfl(r, key));
            *reinterpret_cast<u32x4 *>(mine + key * VS + slot * 16) = *reinterpret_cast<const u32x4 *>(row + slot * 16);
        }
        wave_sync();
        // scores: lane (g, n) holds keys 16 rt + 4 g .. + 3 of query n
        f32x4 s[RT];
        float top = -INFINITY;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            s[rt] = f32x4{};
#pragma unroll
            for (int m = 0; m < NG; ++m) {
                f32x4 y = {};
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    // the group that the step's dimensions lie in
                    constexpr int nib = BITS == 4 && D != 64 ? 4 : 1;
                    const int group = NG == 1 ? 0 : (st % nib) * (D / 4) / kGroup4;
                    if (group != m) continue;
                    u32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (BITS == 8) {
                            const uint32_t u = kx[rt][st * 2 + i / 2];
                            w[i] = pack_bf16(byte_of(u, i % 2 * 2), byte_of(u, i % 2 * 2 + 1));
                        } else if constexpr (D == 64) {
                            const uint32_t u = kx[rt][i % 2];
                            const int j = 2 * st + i / 2;
                            w[i] = pack_bf16(nibble_of(u, j), nibble_of(u, j + 4));
                        } else {
                            const uint32_t u = kx[rt][st / 4 * 4 + i];
                            w[i] = pack_bf16(nibble_of(u, st % 4), nibble_of(u, st % 4 + 4));
                        }
                    }
                    const bf16x8 k[1] = {__builtin_bit_cast(bf16x8, w)};
                    mma(y, k, q[st]);
                }
                s[rt] += y * *reinterpret_cast<const f32x4 *>(&sc[wave][0][m][16 * rt + 4 * g]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (none >> (16 * rt + 4 * g + i) & 1) s[rt][i] = -INFINITY;
                top = fmaxf(top, s[rt][i]);
            }
        }
        const float f = run.next(swap_max32(swap_max16(top)) * scale);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[rt][i] = __builtin_amdgcn_exp2f(fmaf(s[rt][i], scale, -run.base));
                run.l += s[rt][i];
            }
        // weights times the scales of each group of dimensions, in planes; then the values of that group
#pragma unroll
        for (int m = 0; m < NG; ++m) {
            const f32x4 y0 = s[0] * *reinterpret_cast<const f32x4 *>(&sc[wave][1][m][4 * g]);
            const f32x4 y1 = s[1] * *reinterpret_cast<const f32x4 *>(&sc[wave][1][m][16 + 4 * g]);
            bf16x8 p[PP];
            if constexpr (BF) {
                const float y[8] = {y0[0], y0[1], y0[2], y0[3], y1[0], y1[1], y1[2], y1[3]};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[0][i] = static_cast<__bf16>(y[i]);
                    p[1][i] = static_cast<__bf16>(y[i] - static_cast<float>(p[0][i]));
                }
            } else {
                split(y0, y1, p);
            }
#pragma unroll
            for (int cb = 0; cb < RB / 32; ++cb) {
                uint32_t w[4];                        // 16 columns of 16 bits: keys 4 g .. + 3, then 16 + 4 g .. + 3
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x2 y = read_columns(mine + (16 * h + 4 * g + (n >> 2)) * VS + cb * 32 + (n & 3) * 8);
                    w[2 * h] = y[0], w[2 * h + 1] = y[1];
                }
                constexpr int per = BITS == 8 ? 2 : 4;          // dimensions in a column
#pragma unroll
                for (int j = 0; j < per; ++j) {
                    const int group = NG == 1 ? 0 : j * (D / 4) / kGroup4;
                    if (group != m) continue;
                    u32x4 u;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        u[i] = BITS == 8 ? pack_bf16(byte_of(w[i], j), byte_of(w[i], j + 2))
                                         : pack_bf16(nibble_of(w[i], j), nibble_of(w[i], j + 4));
                    const int tile = cb * per + j;
                    acc[tile] *= f;
                    const bf16x8 v[1] = {__builtin_bit_cast(bf16x8, u)};
                    mma(acc[tile], v, p);
                }
            }
        }
    }
    // the four waves' parts: lane (g, n) holds rows 4 g .. + 3 of each tile of dimensions, of query n
    run.l = swap_add32(swap_add16(run.l));
    if (g == 0) sm[wave][n] = run.m, sl[wave][n] = run.l;
    __syncthreads();
    float top = -INFINITY, z = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][n]);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < 4; ++w) z += sl[w][n] * __builtin_amdgcn_exp2f(sm[w][n] - base);
    const float own = __builtin_amdgcn_exp2f(run.m - base);
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
    if (a.parts == 1) {
        if (wave == 0 && g == 0) {
            sl[0][n] = z;
            if (n < rows && a.lse) a.lse[first + n] = z == 0.0f ? -INFINITY : (base + log2f(z)) * kLn2;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < rows * D; e += 256) {
            const float l = sl[0][e / D];
            static_cast<T *>(a.o)[first * D + e] = narrow<T>(l == 0.0f ? 0.0f : sum[e / D * LD + e % D] / l);
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

// Ranges that each request's tokens are cut into.
int parts_of(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    if (d->batch == 0) return 1;
    const int64_t G = d->n_q_heads / c->n_kv_heads, blocks = static_cast<int64_t>(d->batch) * c->n_kv_heads * ((G + 15) / 16);
    const int64_t tokens = static_cast<int64_t>(d->n_select ? d->n_select : d->max_pages) * c->page_size;
    const int64_t want = std::clamp<int64_t>((512 + blocks - 1) / blocks, 1, std::max<int64_t>(1, (tokens + 255) / 256));
    return static_cast<int>(want);
}

size_t workspace_of(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    const int parts = parts_of(c, d);
    return parts == 1 ? 0 : static_cast<size_t>(d->batch) * d->n_q_heads * (c->head_dim * sizeof(float) + sizeof(float2)) * parts;
}

template <typename T, int D>
void launch(const CacheAttnArgs &a, int bits, hipStream_t st)
{
    const int64_t grid = static_cast<int64_t>(a.batch) * a.c.Hkv * ((a.G + 15) / 16) * a.parts;
    if (bits == 8) cache_attn_kernel<T, D, 8><<<dim3(static_cast<unsigned>(grid)), 256, 0, st>>>(a);
    else cache_attn_kernel<T, D, 4><<<dim3(static_cast<unsigned>(grid)), 256, 0, st>>>(a);
    if (a.parts > 1) join_parts<T, D>({a.ml, a.acc, a.o, a.lse, static_cast<size_t>(a.batch) * a.Hq, a.parts}, st);
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
    CacheAttnArgs a{};
    a.c = cache_view(c, cache);
    a.q = q, a.table = page_table, a.lengths = lengths, a.selected = d->n_select ? selected : nullptr;
    a.o = o, a.lse = lse;
    a.batch = d->batch, a.Hq = d->n_q_heads, a.G = d->n_q_heads / c->n_kv_heads;
    a.max_pages = d->max_pages, a.n_select = d->n_select, a.parts = parts_of(c, d);
    a.acc = static_cast<float *>(workspace);
    if (need) a.ml = reinterpret_cast<float2 *>(a.acc + rows * c->head_dim * a.parts);
    a.scale = d->scale * 1.4426950408889634f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->act_dtype == STEPQ_BF16) launch<bf16_t>(a, c->head_dim, c->bits, s);
    else launch<float>(a, c->head_dim, c->bits, s);
    return launched("cache attention launch");
}
