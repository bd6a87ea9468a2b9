// Quantized key/value caches: rows quantized as they are written, read back, and the bounds of a page's keys.
#include <algorithm>

#include "stepq_cache.h"
#include "stepq_device.h"

namespace stepq {

stepq_status check_cache(const stepq_cache_desc *d)
{
    if (!d) return bad("cache desc is NULL");
    if (d->n_pages < 0) return bad("negative count of pages");
    if (d->n_kv_heads < 1 || d->page_size < 1) return bad("n_kv_heads and page_size must be >= 1");
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
        return set_error(STEPQ_E_UNSUPPORTED, "head_dim must be 64, 128 or 256");
    if (d->bits != 4 && d->bits != 8) return set_error(STEPQ_E_UNSUPPORTED, "bits must be 4 or 8");
    if (d->page_size > (1 << 20)) return set_error(STEPQ_E_UNSUPPORTED, "more than 2^20 tokens in a page");
    if (static_cast<int64_t>(d->n_pages) * d->n_kv_heads >= (int64_t(1) << 31))
        return set_error(STEPQ_E_UNSUPPORTED, "2^31 or more (page, head) records in a cache");
    if (static_cast<double>(d->n_pages) * d->n_kv_heads * cache_shape(d).record >= 0x1p37)      // offsets in 32 bytes have 32 bits
        return set_error(STEPQ_E_UNSUPPORTED, "2^37 bytes or more in a cache");
    return STEPQ_OK;
}

stepq_status check_paged(const stepq_cache_desc *d, const void *cache, int32_t n, int32_t max_pages, const int32_t *page_table)
{
    if (max_pages < 0) return bad("negative count of pages");
    if (static_cast<int64_t>(max_pages) * d->page_size >= (int64_t(1) << 30))
        return set_error(STEPQ_E_UNSUPPORTED, "2^30 tokens or more in a request's pages");
    if (d->n_pages && !cache) return bad("NULL cache");
    if (!aligned(cache, 128)) return bad("the cache must be 128-byte aligned");
    if (n && max_pages && !page_table) return bad("page_table is NULL");
    return STEPQ_OK;
}

namespace {

struct RowsArgs {
    CacheView c;
    const int32_t *table, *starts, *cu;  // cu NULL: token i is sequence i's only one
    const void *k, *v;                   // write: the tokens' rows; read: where they go
    int64_t sk, sv;                      // elements from one token to the next
    int32_t n_tokens, n_seq, max_pages, slices;      // workgroups that share a token's 2 Hkv rows
    FastDiv div_slices;
};

// The sequence that token t belongs to, the last one that begins at or before it (-1: none), and where it begins.
// A wave's lanes hold 64 of the bounds, spread over all of them; where that does not tell, the rest is looked up.
// 64 (n_seq / 64 + 1), the largest index and one step, is below 2^31.
__device__ __forceinline__ int sequence_of(const RowsArgs &a, int t, int *begin)
{
    *begin = t;
    if (!a.cu) return t;
    const int lane = threadIdx.x & 63, apart = a.n_seq / 64 + 1, held = a.cu[min(lane * apart, a.n_seq)];
    int at = 0, first = __shfl(held, 0);
    if (first > t) at = -1;
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
        const int next = __shfl(held, max(at, 0) + m);
        if (at >= 0 && next <= t) at += m, first = next;
    }
    if (at < 0) return -1;
    int lo = min(at * apart, a.n_seq), hi = min(lo + apart, a.n_seq + 1);      // begins at or before t; does not, or was not asked
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1, y = a.cu[mid];
        if (y <= t) lo = mid, first = y;
        else hi = mid;
    }
    *begin = first;
    return lo < a.n_seq ? lo : -1;
}

// Where token t's rows are: the record of head 0 (NULL: nowhere) and the row.
// held: whether t lies in a sequence at all.  All lanes of a wave take part.
__device__ __forceinline__ uint8_t *place_of(const RowsArgs &a, int t, int *row, bool *held)
{
    int begin;
    const int s = sequence_of(a, t, &begin);
    *held = s >= 0;
    if (s < 0) return nullptr;
    const int start = a.starts[s];
    const int64_t pos = static_cast<int64_t>(start) + (static_cast<int64_t>(t) - begin);
    if (start < 0 || pos >= static_cast<int64_t>(a.max_pages) * a.c.page) return nullptr;
    const int p = fdiv(static_cast<int>(pos), a.c.div_page);
    *row = static_cast<int>(pos) - p * a.c.page;
    return record_of(a.c, a.table[static_cast<size_t>(s) * a.max_pages + p], 0);
}

// A thread's 16 elements of a row in RUNS runs of neighbours: 8-bit codes one
// run of 16; 4-bit codes 4 of 4 (nibble j of its words), a quarter of the row apart.
template <int D, int BITS>
struct Share {
    static constexpr int lanes = D / 16, runs = BITS == 8 ? 1 : 4, run = 16 / runs;
    static __device__ __forceinline__ int dim(int lane, int j) { return j * (D / 4) + lane * run; }
};

template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Raw {     // N elements at an element's alignment, one access
    T x[N];
};

constexpr int kThreads = 256;

// The largest of N neighbouring lanes, 4, 8 or 16; a group takes part as one.
template <int N>
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t x)
{
    x = max(x, dpp_bits<0xB1, 0xF>(x));                               // quad_perm [1,0,3,2]
    x = max(x, dpp_bits<0x4E, 0xF>(x));                               // quad_perm [2,3,0,1]
    if constexpr (N > 4) x = max(x, dpp_bits<0x141, 0xF>(x));         // row_half_mirror: 8 lanes
    if constexpr (N > 8) x = max(x, dpp_bits<0x140, 0xF>(x));         // row_mirror: 16 lanes
    return x;
}

// rint(x / s) in the low bits of the result, in two's complement: of |x / s| < 128, s a bfloat16 and r = 1 / s
// within 2^-22 of it.  Rounded to a whole number by adding 3 2^22, whose last bit counts ones.
//   bfloat16: with s' and x' of 8 bits a quotient off a tie is at least 1 / 1020 off it (|x' 2^a - (c + 1/2) s'| >= 1/4,
// and a > -3 there), while x r is within 2^-14 of it.  So x r, rounded first to a multiple of 2^-11, is on a tie only if
// x / s is, and on the same side of it otherwise.
//   float: x r corrected by its remainder is within 2^-43 of x / s before its last rounding.  x and a tie times s (16 bits)
// are multiples of x's last bit, so that off a tie x / s is 2^-24 of itself off it.  Ties above 1/2 are 1.5 times a power of
// two or more, and a rounding moves what lies beside them by 2^-24 / 1.5 of them; just below 1/2 by 2^-25.
template <typename T>
__device__ __forceinline__ uint32_t rounded_quotient(float x, float s, float r)
{
    constexpr float ones = 0x1.8p23f, steps = 0x1.8p12f;
    if constexpr (std::is_same_v<T, float>) {
        const float y = x * r;
        return __float_as_uint(__builtin_fmaf(__builtin_fmaf(-y, s, x), r, y) + ones);
    } else {
        return __float_as_uint(__builtin_fmaf(x, r, steps) + (ones - steps));
    }
}

// Quantizes rows: scale s, the smallest bfloat16 with top s >= the group's largest magnitude (rounded
// up, so that no code is past the top); codes rint(x / s), those of the exact quotient.
//   A workgroup takes 32 tokens (D = 128) whose places it looks up once, and a share
// of their 2 Hkv rows: found again for every row, 50 us where 42 did.  Bound by memory: 25497
// tokens of 8 heads of 128 bfloat16 out of a projection's output, 8 bits, 104 MB in 256-byte pieces
// and 53 MB out, in 38 us, 4.1 TB/s, the vector units busy half of it (41 us with divisions and
// conversions, 18.8 M vector instructions for 9.6, which filled them).  The next one or three
// rows' loads ahead gain nothing (70 us with the read for 69, 18 for 16 of fp32).  4 tokens: 2.4 us, a launch.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(RowsArgs a)
{
    using S = Share<D, BITS>;
    using Row = RowOf<D, BITS>;
    constexpr int rows = kThreads / S::lanes, per = S::runs / Row::scales;    // runs of one group: all (8 bits, D = 64), 2 or 1
    constexpr float q = BITS == 8 ? 127.0f : 7.0f, below = (1.0f - 0x1p-22f) / q;
    const int lane = threadIdx.x % S::lanes;
    const int block = fdiv(blockIdx.x, a.div_slices), slice = blockIdx.x - block * a.slices;
    const int64_t t64 = static_cast<int64_t>(block) * rows + threadIdx.x / S::lanes;
    const int t = static_cast<int>(min(t64, static_cast<int64_t>(a.n_tokens - 1)));
    int row = 0;
    bool held;
    uint8_t *const rec0 = place_of(a, t, &row, &held);
    if (!rec0 || t64 >= a.n_tokens) return;           // a row's lanes together
    for (int x = slice; x < 2 * a.c.Hkv; x += a.slices) {
        const bool value = x & 1;
        const int hk = x >> 1;
        uint8_t *const rec = rec0 + hk * a.c.record;
        const T *from = static_cast<const T *>(value ? a.v : a.k) + static_cast<size_t>(t) * (value ? a.sv : a.sk) +
                        static_cast<size_t>(hk) * D;
        float e[16];
        uint32_t top[S::runs] = {};
#pragma unroll
        for (int j = 0; j < S::runs; ++j) {
            const auto r = *reinterpret_cast<const Raw<T, S::run> *>(from + S::dim(lane, j));
#pragma unroll
            for (int i = 0; i < S::run; ++i) {
                const float y = widen(r.x[i]);
                e[j * S::run + i] = y;
                top[j] = max(top[j], __float_as_uint(y) & 0x7fffffffu);     // what is not finite is largest
            }
        }
        bf16_t mine = 0;
        float s[Row::scales];
#pragma unroll
        for (int n = 0; n < Row::scales; ++n) {
            uint32_t g = top[n * per];
#pragma unroll
            for (int j = 1; j < per; ++j) g = max(g, top[n * per + j]);
            g = max_of_lanes<S::lanes>(g);
            const float big = __uint_as_float(g);
            uint32_t u = (__float_as_uint(big * below) + 0xffffu) & 0xffff0000u;     // less than two of its last bits too low
            if (__uint_as_float(u) * q < big) u += 0x10000u;                         // the product is exact
            if (big < 0x1p-100f) u = 0;
            if (g >= 0x7f800000u) u = 0x7fc00000u;
            if (lane == n) mine = static_cast<bf16_t>(u >> 16);
            s[n] = __uint_as_float(u);
        }
        uint32_t word[BITS == 8 ? 4 : 2] = {};
#pragma unroll
        for (int j = 0; j < S::runs; ++j) {
            const float sc = s[j / per], inv = __builtin_amdgcn_rcpf(sc);
            const uint32_t keep = sc > 0.0f ? ~0u : 0u;                   // no scale, no codes: whatever came of them
            uint32_t c[S::run];
#pragma unroll
            for (int i = 0; i < S::run; ++i) c[i] = rounded_quotient<T>(e[j * S::run + i], sc, inv);
            if constexpr (BITS == 8) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    word[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[4 * i + 3], c[4 * i + 2], 0x0c0c0400),
                                                    __builtin_amdgcn_perm(c[4 * i + 1], c[4 * i], 0x0c0c0400), 0x05040100) & keep;
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    word[i] |= (__builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100) & 0x000f000fu & keep) << 4 * j;
            }
        }
        uint8_t *to = rec + Row::codes(a.c.page, value, row) + lane * (BITS * 2);
        if constexpr (BITS == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(word[0], word[1], word[2], word[3]);
        else *reinterpret_cast<uint2 *>(to) = make_uint2(word[0], word[1]);
        if (lane < Row::scales) reinterpret_cast<bf16_t *>(rec + Row::scale(a.c.page, value, row))[lane] = mine;
    }
}

// Read back: a thread takes 8 neighbouring dimensions, so that a row's values are written in one piece (16 bytes a
// lane): 8 bytes of codes, or one nibble of 8 words.  Four rows are under way at once; places are looked up as above (75 us
// without, 39 with).  Bound by memory: 32048 tokens of 8 heads of 128 in 4 bits, 35 MB into 131 MB of bfloat16, in 39 us,
// 4.3 TB/s.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(RowsArgs a)
{
    using Row = RowOf<D, BITS>;
    constexpr int lanes = D / 8, rows = kThreads / lanes, U = 4;
    const int lane = threadIdx.x % lanes, d0 = lane * 8;
    const int block = fdiv(blockIdx.x, a.div_slices), slice = blockIdx.x - block * a.slices;
    const int64_t t64 = static_cast<int64_t>(block) * rows + threadIdx.x / lanes;
    const int t = static_cast<int>(min(t64, static_cast<int64_t>(a.n_tokens - 1)));
    int row = 0;
    bool held;
    const uint8_t *rec0 = place_of(a, t, &row, &held);
    if (!held || t64 >= a.n_tokens) return;
    const int nibble = d0 / (D / 4);
    for (int x0 = slice; x0 < 2 * a.c.Hkv; x0 += U * a.slices) {
        uint32_t w[U][BITS == 8 ? 2 : 4];
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * a.slices;
            const bool value = x & 1;
            s[u] = 0.0f;
#pragma unroll
            for (uint32_t &y : w[u]) y = 0;
            if (rec0 && x < 2 * a.c.Hkv) {
                const uint8_t *rec = rec0 + (x >> 1) * a.c.record, *codes = rec + Row::codes(a.c.page, value, row);
                s[u] = widen(reinterpret_cast<const bf16_t *>(rec + Row::scale(a.c.page, value, row))[BITS == 8 ? 0 : d0 / kGroup4]);
                if constexpr (BITS == 8) {
                    const uint2 y = reinterpret_cast<const uint2 *>(codes)[lane];
                    w[u][0] = y.x, w[u][1] = y.y;
                } else {
                    const uint4 y = *reinterpret_cast<const uint4 *>(codes + d0 % (D / 4) * 2);
                    w[u][0] = y.x, w[u][1] = y.y, w[u][2] = y.z, w[u][3] = y.w;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * a.slices;
            if (x >= 2 * a.c.Hkv) break;
            const bool value = x & 1;
            Raw<T, 8> r;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = BITS == 8 ? static_cast<int8_t>(w[u][i / 4] >> (8 * (i % 4)))
                                        : static_cast<int32_t>(w[u][i / 2] << (28 - 16 * (i % 2) - 4 * nibble)) >> 28;
                r.x[i] = narrow<T>(s[u] * static_cast<float>(c));
            }
            T *to = static_cast<T *>(const_cast<void *>(value ? a.v : a.k)) + static_cast<size_t>(t) * (value ? a.sv : a.sk) +
                    static_cast<size_t>(x >> 1) * D + d0;
            *reinterpret_cast<Raw<T, 8> *>(to) = r;
        }
    }
}

struct BoundsArgs {
    CacheView c;
    const int32_t *table, *starts, *lengths;
    bf16_t *bounds;                      // [n_pages][Hkv][2][D]
    int32_t max_pages, turns;            // workgroups that take the pages of one (request, head) in turn
};

// Towards -inf to bfloat16.
__device__ __forceinline__ bf16_t bf16_below(float x)
{
    const uint32_t u = __float_as_uint(x);
    return static_cast<bf16_t>((u >> 31 ? u + 0xffffu : u) >> 16);
}

// A thread takes 4 bytes of every row of its group: 4 dimensions of 8-bit codes,
// nibbles 0 .. 3 of 2 words of 4-bit ones; the groups of rows join in LDS.  Minimum
// and maximum leave out what is not a number, which its scale tells.  Bound by its chain
// of loads (length, page, codes): 64 requests x 8 heads, a page of 64 tokens each, 5.2 us
// (25 with 16 elements a thread and the joins by exchanges between lanes).
template <int D, int BITS>
__global__ __launch_bounds__(kThreads) void cache_bounds_kernel(BoundsArgs a)
{
    using Row = RowOf<D, BITS>;
    constexpr int cols = Row::bytes / 4, groups = kThreads / cols, E = 32 / BITS, NG = Row::scales, U = 4;
    __shared__ float part[2][groups][D];
    __shared__ uint32_t nans;                         // of each group of dimensions
    const int col = threadIdx.x % cols, group = threadIdx.x / cols;
    const auto dim = [&](int i) { return BITS == 8 ? 4 * col + i : i % 4 * (D / 4) + 2 * col + i / 4; };
    const auto scale_of = [](int i) { return NG == 1 ? 0 : i % 4 * (D / 4) / kGroup4; };
    int x = blockIdx.x;
    const int turn = x % a.turns;
    x /= a.turns;
    const int hk = x % a.c.Hkv, b = x / a.c.Hkv;
    const int len = static_cast<int>(min(static_cast<int64_t>(max(a.lengths[b], 0)), static_cast<int64_t>(a.max_pages) * a.c.page));
    const int start = a.starts[b];
    if (start < 0 || start >= len) return;
    const int last = fdiv(len - 1, a.c.div_page);
    for (int p = fdiv(start, a.c.div_page) + turn; p <= last; p += a.turns) {
        const int id = a.table[static_cast<size_t>(b) * a.max_pages + p];
        const uint8_t *rec = record_of(a.c, id, hk);
        if (!rec) continue;
        const int n = min(a.c.page, len - p * a.c.page);
        if (threadIdx.x == 0) nans = 0;
        float lo[E], hi[E];
        uint32_t nan = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
        for (int r0 = group; r0 < n; r0 += groups * U) {
            uint32_t w[U];
            float s[U][NG];
#pragma unroll
            for (int u = 0; u < U; ++u) {             // past the end: the last row again
                const int r = min(r0 + u * groups, n - 1);
                w[u] = reinterpret_cast<const uint32_t *>(rec + Row::codes(a.c.page, false, r))[col];
                const bf16_t *sc = reinterpret_cast<const bf16_t *>(rec + Row::scale(a.c.page, false, r));
#pragma unroll
                for (int m = 0; m < NG; ++m) s[u][m] = widen(sc[m]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int m = 0; m < NG; ++m) nan |= (s[u][m] != s[u][m]) << m;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int c = BITS == 8 ? static_cast<int8_t>(w[u] >> (8 * i))
                                            : static_cast<int32_t>(w[u] << (28 - 16 * (i / 4) - 4 * (i % 4))) >> 28;
                    const float y = s[u][scale_of(i)] * static_cast<float>(c);
                    lo[i] = fminf(lo[i], y), hi[i] = fmaxf(hi[i], y);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < E; ++i) part[0][group][dim(i)] = lo[i], part[1][group][dim(i)] = hi[i];
        __syncthreads();
        if (nan) atomicOr(&nans, nan);
        __syncthreads();
        bf16_t *to = a.bounds + (static_cast<size_t>(id) * a.c.Hkv + hk) * 2 * D;
        for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
            const int d = i % D;
            float y = part[i / D][0][d];
#pragma unroll
            for (int j = 1; j < groups; ++j) y = i < D ? fminf(y, part[0][j][d]) : fmaxf(y, part[1][j][d]);
            const bf16_t v = i < D ? bf16_below(y) : bf16_below(-y) ^ 0x8000u;
            to[i] = nans >> (NG == 1 ? 0 : d / kGroup4) & 1 ? 0x7fc0 : v;
        }
        __syncthreads();
    }
}

template <typename F>
void by_shape(const stepq_cache_desc *d, F &&f)
{
    const auto bits = [&](auto D) {
        if (d->bits == 8) f(D, std::integral_constant<int, 8>());
        else f(D, std::integral_constant<int, 4>());
    };
    if (d->head_dim == 64) bits(std::integral_constant<int, 64>());
    else if (d->head_dim == 128) bits(std::integral_constant<int, 128>());
    else bits(std::integral_constant<int, 256>());
}

stepq_status check_tokens(const stepq_cache_desc *d, const stepq_cache_tokens *t, const void *cache, const int32_t *table,
                          const int32_t *starts, const int32_t *cu, const void *k, const void *v)
{
    if (const stepq_status st = check_cache(d)) return st;
    if (!t) return bad("tokens desc is NULL");
    if (!known_dtype(t->act_dtype)) return bad("unknown activation dtype");
    if (t->n_tokens < 0 || t->n_seq < 0) return bad("negative count");
    if (!cu && t->n_tokens != t->n_seq) return bad("without cu_seqlens every sequence has one token");
    const int64_t heads = static_cast<int64_t>(d->n_kv_heads) * d->head_dim;
    for (const int64_t s : {t->k_stride, t->v_stride}) {
        if (s < 0 || (s && s < heads)) return bad("tokens must not overlap");
        if (s > (int64_t(1) << 26)) return set_error(STEPQ_E_UNSUPPORTED, "a token stride past 2^26 elements");
    }
    // a launch has less than 2^32 threads, 8 elements each of keys and values
    if (t->n_tokens >= (int64_t(1) << 31) || static_cast<double>(t->n_tokens) * heads >= 0x1p33)
        return set_error(STEPQ_E_UNSUPPORTED, "2^31 tokens or 2^33 elements or more in one call: split it");
    if (t->n_seq > INT32_MAX - 64) return set_error(STEPQ_E_UNSUPPORTED, "2^31 - 64 sequences or more");     // see sequence_of
    if (const stepq_status st = check_paged(d, cache, t->n_seq, t->max_pages, table)) return st;
    if (t->n_tokens && t->n_seq && (!starts || !k || !v)) return bad("NULL starts or token rows");
    const int el = t->act_dtype == STEPQ_F32 ? 4 : 2;
    if (!aligned(k, el) || !aligned(v, el)) return bad("token rows must be aligned to their type");
    return STEPQ_OK;
}

RowsArgs rows_args(const stepq_cache_desc *d, const stepq_cache_tokens *t, const void *cache, const int32_t *table,
                   const int32_t *starts, const int32_t *cu, const void *k, const void *v)
{
    const int64_t heads = static_cast<int64_t>(d->n_kv_heads) * d->head_dim;
    return {cache_view(d, cache), table, starts, cu, k, v, t->k_stride ? t->k_stride : heads, t->v_stride ? t->v_stride : heads,
            static_cast<int32_t>(t->n_tokens), t->n_seq, t->max_pages, 1, {}};
}

// EACH elements a thread; a token's rows go to as many workgroups as there are with fewer tokens: written and read
// back, 25497 tokens take 71, 70 and 69 us with 2048, 4096 and 8192 of them to write and 2048 to read, 32048 of 4 bits 45
// with each; with 4096 to read 2 more.
template <int D, int EACH>
unsigned rows_grid(RowsArgs &a, int64_t workgroups)
{
    constexpr int rows = kThreads / (D / EACH);
    const int64_t blocks = (static_cast<int64_t>(a.n_tokens) + rows - 1) / rows;
    const int64_t all = 2 * int64_t(a.c.Hkv), most = std::clamp<int64_t>(workgroups / blocks, 1, all), each = (all + most - 1) / most;
    a.slices = static_cast<int32_t>((all + each - 1) / each);
    a.div_slices = fast_div(static_cast<uint32_t>(a.slices));
    return static_cast<unsigned>(blocks * a.slices);
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_cache_bytes(const stepq_cache_desc *d, size_t *cache_bytes, size_t *record_bytes)
{
    if (const stepq_status st = check_cache(d)) return st;
    if (!cache_bytes) return bad("cache_bytes is NULL");
    const int64_t record = cache_shape(d).record;
    if (record_bytes) *record_bytes = static_cast<size_t>(record);
    *cache_bytes = static_cast<size_t>(record) * d->n_pages * d->n_kv_heads;
    return STEPQ_OK;
}

extern "C" stepq_status stepq_cache_write(const stepq_cache_desc *d, const stepq_cache_tokens *t, void *cache,
                                          const int32_t *page_table, const int32_t *starts, const int32_t *cu_seqlens,
                                          const void *k, const void *v, void *stream)
{
    if (const stepq_status st = check_tokens(d, t, cache, page_table, starts, cu_seqlens, k, v)) return st;
    if (t->n_tokens == 0 || t->n_seq == 0) return STEPQ_OK;
    RowsArgs a = rows_args(d, t, cache, page_table, starts, cu_seqlens, k, v);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(d, [&](auto D, auto B) {
        const dim3 grid(rows_grid<D, 16>(a, 8192));
        if (t->act_dtype == STEPQ_BF16) cache_write_kernel<bf16_t, D, B><<<grid, kThreads, 0, s>>>(a);
        else cache_write_kernel<float, D, B><<<grid, kThreads, 0, s>>>(a);
    });
    return launched("cache write launch");
}

extern "C" stepq_status stepq_cache_read(const stepq_cache_desc *d, const stepq_cache_tokens *t, const void *cache,
                                         const int32_t *page_table, const int32_t *starts, const int32_t *cu_seqlens,
                                         void *k, void *v, void *stream)
{
    if (const stepq_status st = check_tokens(d, t, cache, page_table, starts, cu_seqlens, k, v)) return st;
    if (t->n_tokens == 0 || t->n_seq == 0) return STEPQ_OK;
    RowsArgs a = rows_args(d, t, cache, page_table, starts, cu_seqlens, k, v);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(d, [&](auto D, auto B) {
        const dim3 grid(rows_grid<D, 8>(a, 2048));
        if (t->act_dtype == STEPQ_BF16) cache_read_kernel<bf16_t, D, B><<<grid, kThreads, 0, s>>>(a);
        else cache_read_kernel<float, D, B><<<grid, kThreads, 0, s>>>(a);
    });
    return launched("cache read launch");
}

extern "C" stepq_status stepq_cache_bounds(const stepq_cache_desc *d, const void *cache, int32_t batch, int32_t max_pages,
                                           const int32_t *page_table, const int32_t *starts, const int32_t *lengths,
                                           void *bounds, void *stream)
{
    if (const stepq_status st = check_cache(d)) return st;
    if (batch < 0) return bad("negative count");
    if (static_cast<int64_t>(batch) * d->n_kv_heads > (int64_t(1) << 23))
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^23 (request, key/value head) pairs in one call: split the batch");
    if (const stepq_status st = check_paged(d, cache, batch, max_pages, page_table)) return st;
    if (batch == 0 || max_pages == 0 || d->n_pages == 0) return STEPQ_OK;
    if (!starts || !lengths || !bounds) return bad("NULL starts, lengths or bounds");
    if (!aligned(bounds, 16)) return bad("bounds must be 16-byte aligned");
    const int64_t pairs = static_cast<int64_t>(batch) * d->n_kv_heads;
    const int32_t turns = static_cast<int32_t>(std::clamp<int64_t>(1024 / pairs, 1, max_pages));
    const BoundsArgs a{cache_view(d, cache), page_table, starts, lengths, static_cast<bf16_t *>(bounds), max_pages, turns};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(d, [&](auto D, auto B) {
        cache_bounds_kernel<D, B><<<dim3(static_cast<unsigned>(pairs * turns)), kThreads, 0, s>>>(a);
    });
    return launched("cache bounds launch");
}
