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
    FastDiv div_items, div_blocks, div_hkv;      // by the workgroups of one part, by the blocks of 16 heads, by Hkv
    float scale;             // times log2 e, scores are kept in powers of two; and 16 of 4 bits, whose codes come as sixteenths
    float unit;              // of the values' sums: 1, or 16 of 4 bits
};

constexpr int kMaxChunk = 1024;
constexpr int kTile = 32;    // keys of a wave's turn
constexpr int kFewParts = 8;
// Waves of a SIMD that the registers are for.
template <typename T, int D>
constexpr int waves_of()
{
    if (D == 256) return sizeof(T) == 4 ? 1 : 2;
    return sizeof(T) == 4 ? 2 : 3;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
// Bytes i and j of a word as bfloat16 (exact).
__device__ __forceinline__ uint32_t bytes_of(uint32_t w, int i, int j)
{
    return pack_bf16(static_cast<float>(static_cast<int8_t>(w >> (8 * i))), static_cast<float>(static_cast<int8_t>(w >> (8 * j))));
}
// The nibbles of a word as sixteenths of their codes (exact): byte b's lower one, or of w >> 4 its upper one.
__device__ __forceinline__ float sixteenth(uint32_t w, int b) { return __builtin_amdgcn_cvt_off_f32_i4(w >> (8 * b) & 0xff); }
// Nibble j of both halves of a word so, as bfloat16, for all four.
__device__ __forceinline__ void nibbles_of(uint32_t w, uint32_t (&y)[4])
{
    uint32_t u = w >> 4;
    asm("" : "+v"(u));                   // one shift, and bytes chosen by the conversions
    y[0] = pack_bf16(sixteenth(w, 0), sixteenth(w, 2));
    y[1] = pack_bf16(sixteenth(u, 0), sixteenth(u, 2));
    y[2] = pack_bf16(sixteenth(w, 1), sixteenth(w, 3));
    y[3] = pack_bf16(sixteenth(u, 1), sixteenth(u, 3));
}

// Two floats rounded to bfloat16, and what that leaves of them so.
__device__ __forceinline__ void two_planes(float a, float b, bf16x2 &hi, bf16x2 &lo)
{
    hi = __builtin_convertvector((f32x2{a, b}), bf16x2);
    lo = __builtin_convertvector((f32x2{a - static_cast<float>(hi[0]), b - static_cast<float>(hi[1])}), bf16x2);
}

// One of a request's key heads, 16 of its query heads, `chunk` of its tokens
// (all of them, or those of its selected pages): the waves take tiles of keys in
// turn.  Scores are formed transposed, keys x queries, from codes as bfloat16
// (exact), each group's sum times its scale; values pass through LDS of the wave's
// own as codes, to be read by columns of 16 bits, 2 or 4 dimensions at once, and
// their scales go into the weights.  The next tile's codes and scales are on their way
// meanwhile, into the registers that the tile's codes have left.
//   Rounded are the sums and weights only: bfloat16 weights to two planes (16 bits), so
// that their rounding is far below the output's, fp32 ones and queries to three (24 bits).
//   8 bits: bound by memory, 64 requests x 8 heads x 1-8192 tokens of 128 (550 MB) in 113
// us, 4.9 TB/s (6.0 is what a kernel that only reads reaches here); 1 x 2 x 131072 of 256 (135 MB) in
// 28 us.  4 bits: bound by vector issue, 400 instructions for 32 keys of a head, 104 of them
// for the values' conversion, as many for the keys' and 32 for the weights' planes: 256 x 8 x 1-4096
// of 128 (539 MB) in 154 us, 3.5 TB/s, 67 % of the cycles issue.  Codes put into a bfloat16's mantissa as
// 1.5 + c / 16 convert in 40 fewer for each operand (keys so: 147 us); but 1.5 times the sum of the other operand,
// taken off again, leaves 2^-20 of a row's largest value in dimensions whose codes are 0, and in the scores 2^-24
// of 24 times a query's largest dimension and the key's scale, whatever the codes there.
// Tiles of 64 keys with two waves a SIMD take 7 % more; four waves a SIMD spill (twice the time).
//   4 requests x 640 tokens: 5.8 us, the chain of loads.
//   FOLD: few heads leave most of the matrix cores' columns idle, so each group of a row's scales has
// columns of its own with the same queries: a lane makes the weights of one group, and sums of other groups'
// dimensions in its column are left.  64 requests x 8192 tokens of 4 bits with 4 or 8 query heads each, whole
// calls, us, without and with it: 8 heads of 128, bf16, 144 / 141 and 145 / 139, fp32 180 / 173 and 187 / 176;
// 2 of 256 (4 query heads), bf16, 77 / 74, fp32 124 / 106; 4 requests x 640 9.2 / 8.7 with either.
template <typename T, int D, int BITS, bool FOLD>
__global__ __launch_bounds__(256, (waves_of<T, D>()))
void cache_attn_kernel(CacheAttnArgs a)
{
    constexpr bool BF = sizeof(T) == 2;
    using Row = RowOf<D, BITS>;
    constexpr int RB = Row::bytes, NG = Row::scales, KT = kTile, RT = KT / 16;
    constexpr int LB = RB / 4, PB = LB < 16 ? LB : 16, PIECES = LB / PB;     // bytes of a row per lane group, in loads of PB
    constexpr int STEPS = D / 32, QP = BF ? 1 : 3, PP = BF ? 2 : 3;          // products over D; planes of queries and weights
    constexpr int VS = 32 * (RB / 32 | 1);            // a row of values in LDS: 16 rows' 32 bytes fall on all banks
    constexpr int LD = D + 4, VB = 4 * KT * VS, SB = 4 * 16 * LD * 4;
    constexpr int PAGES = (kMaxChunk + 1) * static_cast<int>(sizeof(int2));
    __shared__ alignas(16) uint8_t vs[VB + PAGES > SB ? VB + PAGES : SB];     // values and pages; in the end the waves' sums
    __shared__ alignas(16) float sc[4][2][NG][KT];
    __shared__ float sm[4][16], sl[4][16];
    int2 *pages = reinterpret_cast<int2 *>(vs + VB);  // the chunk's pages: record (-1: none), tokens that count
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const int Hkv = a.c.Hkv, page = a.c.page;
    const int part = fdiv(blockIdx.x, a.div_items), item = blockIdx.x - part * (a.batch * Hkv * ((a.G + 15) / 16));
    const int bh = fdiv(item, a.div_blocks), row0 = (item - bh * ((a.G + 15) / 16)) * 16;
    // columns of queries: FOLD: the same ones for each group of a row's scales
    constexpr int COLS = FOLD ? 16 / NG : 16, SETS = FOLD ? 1 : NG;          // of weights, that a lane makes
    const int b = fdiv(bh, a.div_hkv), hk = bh - b * Hkv, rows = min(COLS, a.G - row0), r = n % COLS, group = n / COLS;
    const int32_t *table = a.table + static_cast<size_t>(b) * a.max_pages;
    const int32_t *chosen = a.selected ? a.selected + static_cast<size_t>(bh) * a.n_select : nullptr;
    const int from = part * a.chunk, most = (chosen ? a.n_select : a.max_pages) * page;
    const int first_page = fdiv(from, a.c.div_page);
    const int end_page = most ? fdiv(min(most, from + a.chunk) - 1, a.c.div_page) + 1 : 0;
    // page p's position and id; both are looked up before the length is there
    const auto look = [&](int p, int &pos, int &id) {
        pos = chosen ? chosen[p] : p;
        id = pos >= 0 && pos < a.max_pages ? table[pos] : -1;
    };
    int pos0 = 0, id0 = -1;
    if (first_page + static_cast<int>(threadIdx.x) < end_page) look(first_page + threadIdx.x, pos0, id0);

    // queries, operand B: query n, the 8 dimensions of each step that the codes of a lane group stand for
    const size_t qrow = static_cast<size_t>(b) * a.Hq + hk * a.G + row0 + min(r, rows - 1);
    u32x4 raw[STEPS][BF ? 1 : 2];
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
            raw[st][0] = u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            raw[st][0] = *reinterpret_cast<const u32x4 *>(from_q + d0), raw[st][1] = *reinterpret_cast<const u32x4 *>(from_q + d1);
        }
    }
    const int len = min(max(a.lengths[b], 0), a.max_pages * page);
    const int total = chosen ? most : len, to = min(total, from + a.chunk);
    if (part && from >= total) return;
    const auto entry = [&](int pos, int id) {
        return id >= 0 && id < a.c.n_pages && pos * page < len ? make_int2(id * Hkv + hk, len - pos * page) : make_int2(-1, 0);
    };
    if (first_page + static_cast<int>(threadIdx.x) < end_page) pages[threadIdx.x] = entry(pos0, id0);
    for (int p = first_page + 256 + threadIdx.x; p < end_page; p += 256) {
        int pos, id;
        look(p, pos, id);
        pages[p - first_page] = entry(pos, id);
    }
    bf16x8 q[STEPS][QP];
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
        if (!(a.scale > 0.0f))
#pragma unroll
            for (u32x4 &y : raw[st]) y = with_sign(y, a.scale, BF ? 0x80008000u : 0x80000000u);
        if constexpr (BF) {
            q[st][0] = __builtin_bit_cast(bf16x8, raw[st][0]);
        } else {
            bf16x8 p[3];
            split(__builtin_bit_cast(f32x4, raw[st][0]), __builtin_bit_cast(f32x4, raw[st][1]), p);
#pragma unroll
            for (int i = 0; i < 3; ++i) q[st][i] = p[i];
        }
    }
    // the group that a step's dimensions lie in
    const auto group_of = [](int st) { return NG == 1 ? 0 : st % 4 * (D / 4) / kGroup4; };
    const float scale = scale_of(a.scale);
    const auto wave_sync = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    __syncthreads();

    uint8_t *mine = vs + wave * KT * VS;
    // a tile's keys: lane l has the record and row of key l % KT; there: the keys that are (row 0 of the cache stands in)
    int64_t at = 0;
    uint32_t unit = 0;                                // of its row, in 32 bytes
    int row = 0;
    uint32_t there = 0;
    const uint32_t record_units = static_cast<uint32_t>(a.c.record / 32);
    const auto locate = [&](int t0) {
        const int t = t0 + lane % KT;
        at = 0, unit = 0, row = 0;
        bool ok = false;
        if (t < to) {
            const int p = fdiv(t, a.c.div_page), in_page = t - p * page;
            const int2 e = pages[p - first_page];
            ok = e.x >= 0 && in_page < e.y;
            if (ok) at = static_cast<int64_t>(e.x) * a.c.record, row = in_page, unit = e.x * record_units + in_page * (RB / 32);
        }
        there = static_cast<uint32_t>(__ballot(ok));
    };
    uint32_t kx[RT][LB / 4], vx[RT][LB / 4], sx[(NG + 1) / 2];
    const uint8_t *base[RT];
    const auto bases = [&] {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
            base[rt] = a.c.mem + static_cast<uint64_t>(static_cast<uint32_t>(__shfl(static_cast<int>(unit), 16 * rt + n))) * 32 + g * PB;
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
        const uint8_t *s = a.c.mem + at + Row::scale(page, lane >= KT, row);
        if constexpr (NG == 1) sx[0] = *reinterpret_cast<const bf16_t *>(s);
        else
#pragma unroll
            for (int i = 0; i < NG / 2; ++i) sx[i] = reinterpret_cast<const uint32_t *>(s)[i];
    };
    float m = -INFINITY, low = 0.0f, l = 0.0f;        // the maximum, what is taken off the scores, the sum
    f32x4 acc[D / 16] = {};
    const int value_at = page * RB;
    int t0 = from + wave * KT;
    for (; t0 < to; t0 += 4 * KT) {                   // the first tile with a key
        locate(t0);
        if (there) break;
    }
    if (t0 < to) {
        bases();
        fetch_scales();
        fetch(vx, value_at);
        fetch(kx, 0);
    }
    while (t0 < to) {
        const uint32_t have = there;
        const bool mine_there = have >> (lane % KT) & 1;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const float y = i % 2 ? upper_bf16(sx[i / 2]) : lower_bf16(sx[i / 2]);
            sc[wave][lane / KT][i][lane % KT] = mine_there ? y : 0.0f;
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
        for (t0 += 4 * KT; t0 < to; t0 += 4 * KT) {
            locate(t0);
            if (there) break;
        }
        if (t0 < to) {
            bases();
            fetch_scales();
            fetch(vx, value_at);
        }
        // scores: lane (g, n) holds keys 16 rt + 4 g .. + 3 of query n
        f32x4 s[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            f32x4 y[NG] = {};
            const auto step = [&](int st, const u32x4 &w) {
                const bf16x8 k[1] = {__builtin_bit_cast(bf16x8, w)};
                mma(y[group_of(st)], k, q[st]);
            };
            if constexpr (BITS == 8) {
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    const uint32_t u = kx[rt][st * 2], v = kx[rt][st * 2 + 1];
                    step(st, u32x4{bytes_of(u, 0, 1), bytes_of(u, 2, 3), bytes_of(v, 0, 1), bytes_of(v, 2, 3)});
                }
            } else {
                constexpr int W = D == 64 ? 2 : 4;    // words of a piece
#pragma unroll
                for (int i = 0; i < LB / 4 / W; ++i) {
                    uint32_t y4[W][4];
#pragma unroll
                    for (int w = 0; w < W; ++w) nibbles_of(kx[rt][i * W + w], y4[w]);
                    if constexpr (D == 64) {
#pragma unroll
                        for (int st = 0; st < 2; ++st)
                            step(st, u32x4{y4[0][2 * st], y4[1][2 * st], y4[0][2 * st + 1], y4[1][2 * st + 1]});
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) step(4 * i + j, u32x4{y4[0][j], y4[1][j], y4[2][j], y4[3][j]});
                    }
                }
            }
            s[rt] = y[0] * *reinterpret_cast<const f32x4 *>(&sc[wave][0][0][16 * rt + 4 * g]);
#pragma unroll
            for (int i = 1; i < NG; ++i) s[rt] += y[i] * *reinterpret_cast<const f32x4 *>(&sc[wave][0][i][16 * rt + 4 * g]);
        }
        if (t0 < to) fetch(kx, 0);
        if (~have) {                                  // not all of the tile's keys are
            const uint32_t x = have >> (4 * g);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(x >> (16 * rt + i) & 1)) s[rt][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[rt][i]);
        // What is taken off begins 6 above the maximum and follows only when that has passed it: weights are at most 1, so
        // that sums over n values of at most a stay within n a
        top = swap_max32(swap_max16(top)) * scale;
        if (__any(!(top <= low) || m == -INFINITY)) {
            const float to_m = fmaxf(m, top), nb = to_m == -INFINITY ? 0.0f : to_m + 6.0f;
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
        // weights times the scales of a group of dimensions, in planes
        const auto weights = [&](int i, bf16x8 (&p)[PP]) {
            const float *vsc = &sc[wave][1][FOLD ? group : i][4 * g];
            const f32x4 y0 = s[0] * *reinterpret_cast<const f32x4 *>(vsc);
            const f32x4 y1 = s[1] * *reinterpret_cast<const f32x4 *>(vsc + 16);
            if constexpr (BF) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bf16x2 hi, lo;
                    if (j < 2) two_planes(y0[2 * j], y0[2 * j + 1], hi, lo);
                    else two_planes(y1[2 * j - 4], y1[2 * j - 3], hi, lo);
                    p[0][2 * j] = hi[0], p[0][2 * j + 1] = hi[1];
                    p[1][2 * j] = lo[0], p[1][2 * j + 1] = lo[1];
                }
            } else {
                split(y0, y1, p);
            }
        };
        // four groups in two passes over the values, nibbles 0 and 2, then 1 and 3: their weights fill the registers
        constexpr int PASSES = SETS == 4 ? 2 : 1, NP = SETS / PASSES;
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
            bf16x8 p[NP][PP];
#pragma unroll
            for (int i = 0; i < NP; ++i) weights(PASSES * i + pass, p[i]);
#pragma unroll
            for (int cb = 0; cb < RB / 32; ++cb) {
                uint32_t w[4];                        // 16 columns of 16 bits: keys 4 g .. + 3, then 16 + 4 g .. + 3
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x2 y = read_columns(mine + (16 * i + 4 * g + (n >> 2)) * VS + cb * 32 + (n & 3) * 8);
                    w[2 * i] = y[0], w[2 * i + 1] = y[1];
                }
                constexpr int per = BITS == 8 ? 2 : 4;          // dimensions in a column
                u32x4 u[per];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (BITS == 8) {
                        u[0][i] = bytes_of(w[i], 0, 2), u[1][i] = bytes_of(w[i], 1, 3);
                    } else {
                        uint32_t y[4];
                        nibbles_of(w[i], y);
#pragma unroll
                        for (int j = 0; j < 4; ++j) u[j][i] = y[j];
                    }
                }
#pragma unroll
                for (int j = pass; j < per; j += PASSES) {
                    const bf16x8 v[1] = {__builtin_bit_cast(bf16x8, u[j])};
                    mma(acc[cb * per + j], v, p[SETS == 1 ? 0 : j * (D / 4) / kGroup4 / PASSES]);
                }
            }
        }
        wave_sync();
    }
    // the four waves' parts: lane (g, n) holds rows 4 g .. + 3 of each tile of dimensions, of query n
    l = swap_add32(swap_add16(l));
    const float mine_m = m == -INFINITY ? m : low;
    if (g == 0) sm[wave][n] = mine_m, sl[wave][n] = l;
    __syncthreads();                                  // no wave reads its values any more
    float top = -INFINITY, z = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][n]);
    const float base_m = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < 4; ++w) z += sl[w][n] * __builtin_amdgcn_exp2f(sm[w][n] - base_m);
    const float own = __builtin_amdgcn_exp2f(mine_m - base_m);
    float *sum = reinterpret_cast<float *>(vs);       // [wave][row][LD]
    if (r < rows) {
        float *to_row = sum + (wave * 16 + r) * LD;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) acc[i] *= own;
        if constexpr (BITS == 8) {
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb) {
                const f32x4 x = acc[2 * cb], y = acc[2 * cb + 1];
                *reinterpret_cast<f32x4 *>(to_row + 32 * cb + 8 * g) = f32x4{x[0], y[0], x[1], y[1]};
                *reinterpret_cast<f32x4 *>(to_row + 32 * cb + 8 * g + 4) = f32x4{x[2], y[2], x[3], y[3]};
            }
        } else {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                if (!FOLD || i % 4 * (D / 4) / kGroup4 == group)
                    *reinterpret_cast<f32x4 *>(to_row + i % 4 * (D / 4) + i / 4 * 16 + 4 * g) = acc[i];
        }
    }
    const size_t all = static_cast<size_t>(a.batch) * a.Hq, first = static_cast<size_t>(b) * a.Hq + hk * a.G + row0;
    const bool only = total <= a.chunk;               // the only part
    __syncthreads();                                  // sm and sl are read, the sums are there
    if (wave == 0 && g == 0 && n < rows) {
        if (only) {
            sl[0][n] = z;
            if (a.lse) a.lse[first + n] = z == 0.0f ? -INFINITY : (base_m + log2f(z)) * kLn2;
        } else {
            a.ml[part * all + first + n] = make_float2(top, z);
        }
    }
    if (only) __syncthreads();
    for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
        const int x = e / (D / 4), c = e % (D / 4);
        f32x4 y = *reinterpret_cast<const f32x4 *>(sum + x * LD + 4 * c);
#pragma unroll
        for (int w = 1; w < 4; ++w) y += *reinterpret_cast<const f32x4 *>(sum + (w * 16 + x) * LD + 4 * c);
        if (only) {
            const float d = sl[0][x];
            T *o = static_cast<T *>(a.o) + (first + x) * D + 4 * c;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = narrow<T>(d == 0.0f ? 0.0f : y[i] / d * a.unit);
        } else {
            reinterpret_cast<f32x4 *>(a.acc + (part * all + first + x) * D)[c] = y;
        }
    }
}

// The parts that row's tokens take; rows of one or none are there already.
__device__ __forceinline__ int parts_of(const CacheAttnArgs &a, size_t row)
{
    if (a.selected) return a.parts;
    const int len = min(a.lengths[row / a.Hq], a.max_pages * a.c.page);
    return len <= a.chunk ? 0 : (len + a.chunk - 1) / a.chunk;
}

// The parts of each row joined where there are few: 4 dimensions a lane, every part's share in its registers.
// 8192 rows of 128 in 1 to 4 parts: 6.0 us (9.0 with a wave's lane groups a part each, and their sums exchanged), 2048 in 1
// to 8: 5.0.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_join_few_kernel(CacheAttnArgs a)
{
    const uint32_t x = blockIdx.x * 256 + threadIdx.x;
    const size_t row = x / (D / 4), all = static_cast<size_t>(a.batch) * a.Hq;
    const int d = x % (D / 4) * 4;
    if (row >= all) return;
    const int parts = parts_of(a, row);
    if (!parts) return;
    f32x4 y[kFewParts];
    float2 ml[kFewParts];
#pragma unroll
    for (int p = 0; p < kFewParts; ++p) {             // past the end: the last again
        const size_t at = min(p, parts - 1) * all + row;
        ml[p] = a.ml[at];
        y[p] = *reinterpret_cast<const f32x4 *>(a.acc + at * D + d);
    }
    float top = ml[0].x;
#pragma unroll
    for (int p = 1; p < kFewParts; ++p) top = fmaxf(top, ml[p].x);
    const float base = top == -INFINITY ? 0.0f : top;
    f32x4 sum = {};
    float z = 0.0f;
#pragma unroll
    for (int p = 0; p < kFewParts; ++p)
        if (p < parts) {
            const float f = __builtin_amdgcn_exp2f(ml[p].x - base);
            z = fmaf(ml[p].y, f, z);
            sum += y[p] * f;
        }
    T *o = static_cast<T *>(a.o) + row * D + d;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = narrow<T>(z == 0.0f ? 0.0f : sum[i] / z * a.unit);
    if (d == 0 && a.lse) a.lse[row] = z == 0.0f ? -INFINITY : (base + log2f(z)) * kLn2;
}

// The same where there are many: a workgroup takes 64 dimensions of a row by 16 lanes, 16 such
// lane groups its parts in turn, four at a time so that their loads overlap.
// 16 rows of 256 in 128 parts: 5.1 us.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a)
{
    constexpr int U = 4, SLOTS = 16;
    __shared__ float tops[4];
    __shared__ alignas(16) f32x4 sums[4][16];
    __shared__ float zs[4];
    const int lane = threadIdx.x & 15, slot = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const size_t row = blockIdx.x / (D / 64), all = static_cast<size_t>(a.batch) * a.Hq;
    const int d = blockIdx.x % (D / 64) * 64 + lane * 4;
    const int parts = parts_of(a, row);
    if (!parts) return;
    float top = -INFINITY;
    for (int p = threadIdx.x; p < parts; p += 256) top = fmaxf(top, a.ml[p * all + row].x);
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    top = swap_max32(swap_max16(top));
    if ((threadIdx.x & 63) == 0) tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float base = top == -INFINITY ? 0.0f : top;
    f32x4 y = {};
    float z = 0.0f;
    for (int p0 = slot; p0 < parts; p0 += SLOTS * U) {
        f32x4 x[U];
        float2 ml[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const size_t at = static_cast<size_t>(min(p0 + u * SLOTS, parts - 1)) * all + row;
            ml[u] = a.ml[at];
            x[u] = *reinterpret_cast<const f32x4 *>(a.acc + at * D + d);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (p0 + u * SLOTS < parts) {
                const float f = __builtin_amdgcn_exp2f(ml[u].x - base);
                z = fmaf(ml[u].y, f, z);
                y += x[u] * f;
            }
    }
    z = swap_add32(swap_add16(z));
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = swap_add32(swap_add16(y[i]));
    if ((threadIdx.x & 63) < 16) sums[wave][lane] = y;
    if ((threadIdx.x & 63) == 0) zs[wave] = z;
    __syncthreads();
    if (threadIdx.x >= 16) return;
    y = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
    z = zs[0] + zs[1] + zs[2] + zs[3];
    T *o = static_cast<T *>(a.o) + row * D + d;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = narrow<T>(z == 0.0f ? 0.0f : y[i] / z * a.unit);
    if (d == 0 && a.lse) a.lse[row] = z == 0.0f ? -INFINITY : (base + log2f(z)) * kLn2;
}

// Tokens of a part (the last of a request's may have fewer), and the most parts that a request takes.
struct Cut {
    int32_t chunk, parts;
};

Cut cut_of(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    const int64_t tokens = static_cast<int64_t>(d->n_select ? d->n_select : d->max_pages) * c->page_size;
    if (d->batch == 0 || tokens == 0) return {kMaxChunk, 1};
    // Ranges of 256 to 1024 tokens, so many that there are two for a CU, or one of D = 256 (registers let three or two run at
    // once, in fp32 two or one); whole calls, us, at 256 / 512 / 768 / 1024 under tables as wide as the longest request:
    //   8 heads of 128, 8 bits, bf16: 1 request x 32768 tokens 21.0 / 19.1 / 21.4 / 24; 16 x 1024 13.4 / 13.4 / 15.8 / 18;
    //     64 x 4096 122 / 110 / 106 / 105; 64 x 1-8192 138 / 125 / - / 117; 2 heads, 2 x 4096 9.6 / 11.9 / 15.0 / 16
    //   2 heads of 256, 8 bits: 1 x 131072 51 / 39 / - / 33; 64 x 8192 125 / 116 / 113 / 105
    // A join, a second launch, takes 3 us more, which a workgroup spends on 768 tokens (512 in fp32): 4 requests x 640 6.2
    // in one part, 9.3 in three; 23 x 1333 in fp32 14.8 in two, 10.6 in six.
    // Lengths are on the device: what is cut is the table.  Ranges past a request's length end at once, but are launched;
    // under a table for 131072 tokens 4 x 1-640 take 7.6 us for 5.9, 64 x 1-8192 145 for 116, 256 x 1-4096 of 4 bits 301 for 156.
    const int64_t G = d->n_q_heads / c->n_kv_heads, blocks = static_cast<int64_t>(d->batch) * c->n_kv_heads * ((G + 15) / 16);
    const int64_t fill = c->head_dim == 256 ? 256 : 512, one = d->act_dtype == STEPQ_BF16 ? 768 : 512;
    const int64_t want = std::clamp<int64_t>((blocks * tokens + fill - 1) / fill, 256, kMaxChunk);
    const int64_t chunk = tokens <= one ? one : (want + 127) / 128 * 128;
    return {static_cast<int32_t>(chunk), static_cast<int32_t>((tokens + chunk - 1) / chunk)};
}

stepq_status check(const stepq_cache_desc *c, const stepq_cache_attn_desc *d)
{
    if (const stepq_status st = check_cache(c)) return st;
    if (!d) return bad("desc is NULL");
    if (d->n_q_heads < 1 || d->n_q_heads % c->n_kv_heads) return bad("n_q_heads must be a multiple of the cache's n_kv_heads, >= 1");
    if (!known_dtype(d->act_dtype)) return bad("unknown activation dtype");
    if (d->batch < 0 || d->max_pages < 0 || d->n_select < 0) return bad("negative count");
    if (!std::isfinite(d->scale)) return bad("scale must be finite");
    if (std::fabs(d->scale) > 0x1p120f)               // times log2 e and a code's unit it has to be finite too
        return set_error(STEPQ_E_UNSUPPORTED, "a scale past 2^120");
    if (static_cast<int64_t>(std::max(d->max_pages, d->n_select)) * c->page_size >= (int64_t(1) << 30))
        return set_error(STEPQ_E_UNSUPPORTED, "2^30 tokens or more in a request's pages or in its selected ones");
    if (static_cast<int64_t>(d->batch) * d->n_q_heads > (int64_t(1) << 23))      // a launch has less than 2^32 threads
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^23 (request, head) rows in one call: split the batch");
    const Cut cut = cut_of(c, d);
    const int64_t rows = static_cast<int64_t>(d->batch) * d->n_q_heads, G = d->n_q_heads / c->n_kv_heads;
    if (static_cast<int64_t>(d->batch) * c->n_kv_heads * ((G + 15) / 16) * cut.parts >= (int64_t(1) << 24) ||
        (cut.parts > kFewParts && rows * (c->head_dim / 64) >= (int64_t(1) << 24)))
        return set_error(STEPQ_E_UNSUPPORTED, "2^24 or more workgroups for these requests and pages: split the batch");
    return STEPQ_OK;
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
    const auto run = [&](auto kernel) { kernel<<<dim3(static_cast<unsigned>(grid)), 256, 0, st>>>(a); };
    constexpr int groups = RowOf<D, 4>::scales;
    if (bits == 8) run(cache_attn_kernel<T, D, 8, false>);
    else if (groups > 1 && a.G <= 16 / groups) run(cache_attn_kernel<T, D, 4, (groups > 1)>);
    else run(cache_attn_kernel<T, D, 4, false>);
    if (a.parts == 1) return;
    const unsigned units = static_cast<unsigned>(a.batch) * a.Hq * (D / 64);     // 16 lanes each
    if (a.parts > kFewParts) cache_join_kernel<T, D><<<dim3(units), 256, 0, st>>>(a);
    else cache_join_few_kernel<T, D><<<dim3((units + 15) / 16), 256, 0, st>>>(a);
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
    const uint32_t blocks = static_cast<uint32_t>((a.G + 15) / 16);
    a.div_items = fast_div(static_cast<uint32_t>(a.batch) * a.c.Hkv * blocks);
    a.div_blocks = fast_div(blocks), a.div_hkv = fast_div(static_cast<uint32_t>(a.c.Hkv));
    a.acc = static_cast<float *>(workspace);
    if (need) a.ml = reinterpret_cast<float2 *>(a.acc + rows * c->head_dim * a.parts);
    a.unit = c->bits == 4 ? 16.0f : 1.0f;
    a.scale = d->scale * 1.4426950408889634f * a.unit;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->act_dtype == STEPQ_BF16) launch<bf16_t>(a, c->head_dim, c->bits, s);
    else launch<float>(a, c->head_dim, c->bits, s);
    return launched("cache attention launch");
}
