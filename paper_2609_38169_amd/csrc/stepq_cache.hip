// Quantized key/value caches: rows quantized as they are written, read back, and the bounds of a page's keys.
#include <algorithm>

#include "stepq_cache.h"

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
    int32_t n_tokens, n_seq, max_pages;
};

// The sequence that token t belongs to, the last one that begins at or before it; -1: none.
__device__ __forceinline__ int sequence_of(const RowsArgs &a, int t)
{
    if (!a.cu) return t;
    int lo = 0, hi = a.n_seq + 1;        // the first entry beyond t lies in [lo, hi]
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo == 0 || lo > a.n_seq ? -1 : lo - 1;
}

// Where token t's rows of head hk are: the record (NULL: nowhere) and the row.
// held: whether t lies in a sequence at all.
__device__ __forceinline__ uint8_t *place_of(const RowsArgs &a, int t, int hk, int *row, bool *held)
{
    const int s = sequence_of(a, t);
    *held = s >= 0;
    if (s < 0) return nullptr;
    const int start = a.starts[s];
    const int64_t pos = static_cast<int64_t>(start) + (a.cu ? static_cast<int64_t>(t) - a.cu[s] : 0);
    if (start < 0 || pos >= static_cast<int64_t>(a.max_pages) * a.c.page) return nullptr;
    const int p = page_of(static_cast<int>(pos), a.c.div_page);
    *row = static_cast<int>(pos) - p * a.c.page;
    return record_of(a.c, a.table[static_cast<size_t>(s) * a.max_pages + p], hk);
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

// Quantizes rows: scale s, the smallest bfloat16 with top s >= the group's
// largest magnitude; codes rint(x / s).  The quotient is rounded once before rint:
// s has 8 bits and a tie 8 more, so that no fp32 value but the tie itself rounds
// to it, and the codes are those of the exact quotient.
template <typename T, int D, int BITS>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(RowsArgs a)
{
    using S = Share<D, BITS>;
    using Row = RowOf<D, BITS>;
    constexpr int rows = kThreads / S::lanes;
    const int lane = threadIdx.x % S::lanes;
    int x = blockIdx.x;
    const bool value = x & 1;
    x >>= 1;
    const int hk = x % a.c.Hkv;
    const int64_t t64 = static_cast<int64_t>(x / a.c.Hkv) * rows + threadIdx.x / S::lanes;
    const int t = static_cast<int>(min(t64, static_cast<int64_t>(a.n_tokens - 1)));
    int row = 0;
    bool held;
    uint8_t *rec = t64 < a.n_tokens ? place_of(a, t, hk, &row, &held) : nullptr;
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
    // runs of one group: all (8 bits, D = 64), two and two (128), each its own (256)
    constexpr int per = S::runs / Row::scales;
    uint32_t g[Row::scales];
    bf16_t s16[Row::scales];
    float s[Row::scales];
    constexpr float q = BITS == 8 ? 127.0f : 7.0f;
#pragma unroll
    for (int n = 0; n < Row::scales; ++n) {
        g[n] = top[n * per];
#pragma unroll
        for (int j = 1; j < per; ++j) g[n] = max(g[n], top[n * per + j]);
#pragma unroll
        for (int m = 1; m < S::lanes; m <<= 1) g[n] = max(g[n], static_cast<uint32_t>(__shfl_xor(static_cast<int>(g[n]), m)));
        const float big = __uint_as_float(g[n]);
        uint32_t u = (__float_as_uint(big / q) + 0xffffu) & 0xffff0000u;
        if (__uint_as_float(u) * q < big) u += 0x10000u;
        if (big < 0x1p-100f) u = 0;
        if (g[n] >= 0x7f800000u) u = 0x7fc00000u;
        s16[n] = static_cast<bf16_t>(u >> 16);
        s[n] = __uint_as_float(u);
    }
    uint32_t word[BITS == 8 ? 4 : 2] = {};
#pragma unroll
    for (int j = 0; j < S::runs; ++j)
#pragma unroll
        for (int i = 0; i < S::run; ++i) {
            const float sc = s[j / per];
            const int c = sc > 0.0f ? static_cast<int>(rintf(e[j * S::run + i] / sc)) : 0;
            if constexpr (BITS == 8) word[i / 4] |= (static_cast<uint32_t>(c) & 0xffu) << (8 * (i % 4));
            else word[i / 2] |= (static_cast<uint32_t>(c) & 0xfu) << (16 * (i % 2) + 4 * j);
        }
    if (!rec) return;
    uint8_t *to = rec + Row::codes(a.c.page, value, row) + lane * (BITS * 2);
    if constexpr (BITS == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(word[0], word[1], word[2], word[3]);
    else *reinterpret_cast<uint2 *>(to) = make_uint2(word[0], word[1]);
    if (lane < Row::scales) {
        bf16_t mine = s16[0];
#pragma unroll
        for (int n = 1; n < Row::scales; ++n) mine = lane == n ? s16[n] : mine;
        reinterpret_cast<bf16_t *>(rec + Row::scale(a.c.page, value, row))[lane] = mine;
    }
}

// A thread's 16 values of a row.
template <int D, int BITS>
__device__ __forceinline__ void values_of(const uint8_t *rec, int page, bool value, int row, int lane, float (&e)[16])
{
    using S = Share<D, BITS>;
    using Row = RowOf<D, BITS>;
    constexpr int per = S::runs / Row::scales;
    const uint8_t *from = rec + Row::codes(page, value, row) + lane * (BITS * 2);
    const bf16_t *sc = reinterpret_cast<const bf16_t *>(rec + Row::scale(page, value, row));
    float s[Row::scales];
#pragma unroll
    for (int n = 0; n < Row::scales; ++n) s[n] = widen(sc[n]);
    if constexpr (BITS == 8) {
        const uint4 w = *reinterpret_cast<const uint4 *>(from);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = s[0] * static_cast<float>(static_cast<int8_t>(u[i / 4] >> (8 * (i % 4))));
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(from);
        const uint32_t u[2] = {w.x, w.y};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                e[4 * j + i] = s[j / per] * static_cast<float>(static_cast<int32_t>(u[i / 2] << (28 - 16 * (i % 2) - 4 * j)) >> 28);
    }
}

template <typename T, int D, int BITS>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(RowsArgs a)
{
    using S = Share<D, BITS>;
    constexpr int rows = kThreads / S::lanes;
    const int lane = threadIdx.x % S::lanes;
    int x = blockIdx.x;
    const bool value = x & 1;
    x >>= 1;
    const int hk = x % a.c.Hkv;
    const int64_t t64 = static_cast<int64_t>(x / a.c.Hkv) * rows + threadIdx.x / S::lanes;
    if (t64 >= a.n_tokens) return;
    const int t = static_cast<int>(t64);
    int row = 0;
    bool held;
    const uint8_t *rec = place_of(a, t, hk, &row, &held);
    if (!held) return;
    float e[16] = {};
    if (rec) values_of<D, BITS>(rec, a.c.page, value, row, lane, e);
    T *to = static_cast<T *>(const_cast<void *>(value ? a.v : a.k)) + static_cast<size_t>(t) * (value ? a.sv : a.sk) +
            static_cast<size_t>(hk) * D;
#pragma unroll
    for (int j = 0; j < S::runs; ++j) {
        Raw<T, S::run> r;
#pragma unroll
        for (int i = 0; i < S::run; ++i) r.x[i] = narrow<T>(e[j * S::run + i]);
        *reinterpret_cast<Raw<T, S::run> *>(to + S::dim(lane, j)) = r;
    }
}

struct BoundsArgs {
    CacheView c;
    const int32_t *table, *starts, *lengths;
    bf16_t *bounds;                      // [n_pages][Hkv][2][D]
    int32_t batch, max_pages, turns;     // workgroups that take the pages of one (request, head) in turn
};

// Towards -inf to bfloat16.
__device__ __forceinline__ bf16_t bf16_below(float x)
{
    const uint32_t u = __float_as_uint(x);
    return static_cast<bf16_t>((u >> 31 ? u + 0xffffu : u) >> 16);
}

// A thread takes 4 bytes of every row of its group: 4 dimensions of 8-bit codes,
// nibbles 0 .. 3 of 2 words of 4-bit ones; the groups of rows join in LDS.
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
    const int last = page_of(len - 1, a.c.div_page);
    for (int p = page_of(start, a.c.div_page) + turn; p <= last; p += a.turns) {
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
    // a launch has less than 2^32 threads, 16 elements each
    if (t->n_tokens >= (int64_t(1) << 31) || static_cast<double>(t->n_tokens) * heads >= 0x1p34)
        return set_error(STEPQ_E_UNSUPPORTED, "2^31 tokens or 2^34 elements or more in one call: split it");
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
            static_cast<int32_t>(t->n_tokens), t->n_seq, t->max_pages};
}

template <int D>
unsigned rows_grid(const RowsArgs &a)
{
    constexpr int rows = kThreads / (D / 16);
    return static_cast<unsigned>((static_cast<int64_t>(a.n_tokens) + rows - 1) / rows * a.c.Hkv * 2);
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
    const RowsArgs a = rows_args(d, t, cache, page_table, starts, cu_seqlens, k, v);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(d, [&](auto D, auto B) {
        if (t->act_dtype == STEPQ_BF16) cache_write_kernel<bf16_t, D, B><<<dim3(rows_grid<D>(a)), kThreads, 0, s>>>(a);
        else cache_write_kernel<float, D, B><<<dim3(rows_grid<D>(a)), kThreads, 0, s>>>(a);
    });
    return launched("cache write launch");
}

extern "C" stepq_status stepq_cache_read(const stepq_cache_desc *d, const stepq_cache_tokens *t, const void *cache,
                                         const int32_t *page_table, const int32_t *starts, const int32_t *cu_seqlens,
                                         void *k, void *v, void *stream)
{
    if (const stepq_status st = check_tokens(d, t, cache, page_table, starts, cu_seqlens, k, v)) return st;
    if (t->n_tokens == 0 || t->n_seq == 0) return STEPQ_OK;
    const RowsArgs a = rows_args(d, t, cache, page_table, starts, cu_seqlens, k, v);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(d, [&](auto D, auto B) {
        if (t->act_dtype == STEPQ_BF16) cache_read_kernel<bf16_t, D, B><<<dim3(rows_grid<D>(a)), kThreads, 0, s>>>(a);
        else cache_read_kernel<float, D, B><<<dim3(rows_grid<D>(a)), kThreads, 0, s>>>(a);
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
    const BoundsArgs a{cache_view(d, cache), page_table, starts, lengths, static_cast<bf16_t *>(bounds), batch, max_pages, turns};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(d, [&](auto D, auto B) {
        cache_bounds_kernel<D, B><<<dim3(static_cast<unsigned>(pairs * turns)), kThreads, 0, s>>>(a);
    });
    return launched("cache bounds launch");
}
