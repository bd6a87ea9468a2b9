// The pages of a quantized cache that a request's query may need most, by the bounds of their keys.
#include <algorithm>

#include "stepq_cache.h"
#include "stepq_device.h"

namespace stepq {
namespace {

struct SelectArgs {
    const void *q;
    const bf16_t *bounds;    // [n_pages][Hkv][2][D]
    const int32_t *table, *lengths;
    uint32_t *keys;          // [batch][Hkv][max_pages]: scores, in an order of whole numbers
    int32_t *selected;       // [batch][Hkv][n_select]
    int32_t batch, Hkv, G, n_pages, page, max_pages, n_select, n_first, n_last, turns;
    FastDiv div_page;
};

// The pages that a request's tokens take.
__device__ __forceinline__ int pages_of(const SelectArgs &a, int b)
{
    const int len = static_cast<int>(min(static_cast<int64_t>(max(a.lengths[b], 0)), static_cast<int64_t>(a.max_pages) * a.page));
    return len ? fdiv(len - 1, a.div_page) + 1 : 0;
}

// Scores as whole numbers that order as they do; NaN above all (and 0, below -inf, for a page that there is not).
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    return x != x ? 0xffffffffu : u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// Another lane's number, by the lane exchange that CTRL encodes.
template <int CTRL>
__device__ __forceinline__ double exchanged(double x)
{
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x));
    const uint64_t lo = dpp_bits<CTRL, 0xF>(static_cast<uint32_t>(u)), hi = dpp_bits<CTRL, 0xF>(static_cast<uint32_t>(u >> 32));
    return __longlong_as_double(static_cast<long long>(hi << 32 | lo));
}

// score = sum_d hi_d sum_h max(q_hd, 0) + lo_d sum_h min(q_hd, 0): the workgroup adds
// up the heads, a lane takes 8 dimensions of one bound of page after page, four at a
// time; D/4 lanes make a page's score.  Summed in 64 bits and rounded once: an error
// of 2^-45 of the terms, so that the order of summation hardly ever tells.
// Bound by vector issue (58 % of the cycles: conversions, products, the lanes' sums) and
// latency: 64 requests x 8 heads x 217 pages of 128 dimensions (57 MB) in 16.7 us, 8192
// pages of one request (34 MB) in 9.1; 18.9 and 11.6 with the heads added up by every lane for itself,
// 18.5 and 10.7 with the next pages' bounds on their way before that.  Eight pages at a time, or half as many
// workgroups, are no faster; twice as many 2 us slower where there are many requests.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_score_kernel(SelectArgs a)
{
    constexpr int lanes = D / 4, at_once = 256 / lanes, U = 4;
    __shared__ alignas(16) double sums[2 * D];        // over the heads: of the negative parts, then the positive ones
    const int lane = threadIdx.x % lanes, sub = threadIdx.x / lanes;
    const int turn = blockIdx.x % a.turns, pair = blockIdx.x / a.turns, hk = pair % a.Hkv, b = pair / a.Hkv;
    // page ids and queries are asked for before the length is there
    const int32_t *table = a.table + static_cast<size_t>(b) * a.max_pages;
    const auto ids = [&](int p0, int (&id)[U], int end) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = p0 + u * at_once + sub;
            id[u] = p < end ? table[p] : -1;
        }
    };
    int next[U];
    ids(a.n_first + turn * at_once * U, next, a.max_pages);
    const bool high = lane >= lanes / 2;
    const int d0 = lane % (lanes / 2) * 8;
    const T *q = static_cast<const T *>(a.q) + (static_cast<size_t>(b) * a.Hkv + hk) * a.G * D;
    constexpr int SUMS = 2 * D;
    T e[(SUMS + 255) / 256];
#pragma unroll
    for (int j = 0; j * 256 < SUMS; ++j) e[j] = q[(threadIdx.x + j * 256) % D];
    const int pages = pages_of(a, b), end = pages - a.n_last;
    if (pages <= a.n_select || a.n_first + turn * at_once * U >= end) return;
#pragma unroll
    for (int j = 0; j * 256 < SUMS; ++j) {
        const int x = threadIdx.x + j * 256;
        if (x >= SUMS) break;
        double sum = 0.0;
#pragma unroll 4
        for (int h = 0; h < a.G; ++h) {
            const float y = widen(h ? q[static_cast<size_t>(h) * D + x % D] : e[j]);
            // a NaN reaches both sums
            sum += static_cast<double>(x >= D ? (y < 0.0f ? 0.0f : y) : (y > 0.0f ? 0.0f : y));
        }
        sums[x] = sum;
    }
    __syncthreads();
    double w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = sums[high * D + d0 + i];
    uint32_t *keys = a.keys + (static_cast<size_t>(b) * a.Hkv + hk) * a.max_pages;
    for (int p0 = a.n_first + turn * at_once * U; p0 < end; p0 += a.turns * at_once * U) {
        uint4 v[U];
        bool there[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            there[u] = next[u] >= 0 && next[u] < a.n_pages && p0 + u * at_once + sub < end;
            v[u] = make_uint4(0, 0, 0, 0);
            if (there[u])
                v[u] = *reinterpret_cast<const uint4 *>(a.bounds + ((static_cast<size_t>(next[u]) * a.Hkv + hk) * 2 + high) * D + d0);
        }
        if (p0 + a.turns * at_once * U < end) ids(p0 + a.turns * at_once * U, next, end);
        double sum[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t y[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
            sum[u] = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum[u] = fma(w[i], static_cast<double>(__uint_as_float(i % 2 ? y[i / 2] & 0xffff0000u : y[i / 2] << 16)), sum[u]);
        }
        // each exchange halves the sums that a lane holds, so that lane u has score u (modulo 4), then adds their parts
        double mine;
        const bool odd = lane & 1, upper = lane & 2;
        {
            const double x = (odd ? sum[1] : sum[0]) + exchanged<0xB1>(odd ? sum[0] : sum[1]);     // quad_perm [1,0,3,2]
            const double y = (odd ? sum[3] : sum[2]) + exchanged<0xB1>(odd ? sum[2] : sum[3]);
            mine = (upper ? y : x) + exchanged<0x4E>(upper ? x : y);                               // quad_perm [2,3,0,1]
        }
#pragma unroll
        for (int m = 4; m < lanes; m <<= 1) mine += __shfl_xor(mine, m);
        const bool mine_there = upper ? (odd ? there[3] : there[2]) : (odd ? there[1] : there[0]);
        const int p = p0 + lane * at_once + sub;
        if (lane < U && p < end) keys[p] = mine_there ? key_of(static_cast<float>(mine)) : 0;
    }
}

// The n_first first and n_last last pages and the highest scores between them,
// ties to the lowest position.  The lowest score that is taken is found by
// counting scores in 2048 intervals of [low, high], which becomes the interval that
// holds it, until that is a single number (2 or 3 times as a rule: scores lie
// close together, so that intervals of their own range tell them apart where
// their first digits would not); then the pages are written in order.  A thread holds
// EACH pages of a stretch; more pages are read again, stretch by stretch.  Bound by its
// chain of steps: 64 of 217 pages, 512 times, in 6.6 us; 244 of 8180, 8 times, in 9 (17 with
// every thread adding up the waves' counts; 32 and 60 with 256 intervals of one digit).
// Counting for each of up to 512 scores how many are above it takes 12.8, not 6.6, and in one
// launch with the scores 31, not 26.
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void cache_select_kernel(SelectArgs a)
{
    constexpr int BINS = 2048, PER = BINS / THREADS, W = THREADS / 64, STRETCH = THREADS * EACH;
    __shared__ uint32_t count[BINS];
    __shared__ uint32_t found[2], ends[W][2], waves[W];
    __shared__ uint32_t mores[EACH][W], sames[EACH][W];
    const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pages = pages_of(a, b);
    int32_t *out = a.selected + (static_cast<size_t>(b) * a.Hkv + hk) * a.n_select;
    if (pages <= a.n_select) {
        for (int i = tid; i < a.n_select; i += THREADS) out[i] = i < pages ? i : -1;
        return;
    }
    const uint32_t *keys = a.keys + (static_cast<size_t>(b) * a.Hkv + hk) * a.max_pages;
    const int end = pages - a.n_last;
    uint32_t want = a.n_select - a.n_first - a.n_last;
    for (int i = tid; i < a.n_first; i += THREADS) out[i] = i;
    for (int i = tid; i < a.n_last; i += THREADS) out[a.n_select - a.n_last + i] = end + i;
    if (want == 0) return;
    const bool whole = end - a.n_first <= STRETCH;
    uint32_t k[EACH];
    const auto load = [&](int p0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int p = p0 + i * THREADS + tid;
            if (p < end) k[i] = keys[p];
        }
    };
    // f(i, p) for every page of the thread's, whose key is k[i]
    const auto each = [&](int p0, auto &&f) {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (p0 + i * THREADS + tid < end) f(i);
    };
    uint32_t low = 0xffffffffu, high = 0;
    for (int p0 = a.n_first; p0 < end; p0 += STRETCH) {
        load(p0);
        each(p0, [&](int i) { low = min(low, k[i]), high = max(high, k[i]); });
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        low = min(low, static_cast<uint32_t>(__shfl_xor(static_cast<int>(low), m)));
        high = max(high, static_cast<uint32_t>(__shfl_xor(static_cast<int>(high), m)));
    }
    if (lane == 0) ends[wave][0] = low, ends[wave][1] = high;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) low = min(low, ends[w][0]), high = max(high, ends[w][1]);
    while (low < high) {                              // the want-th highest of those in [low, high] is looked for
        const int shift = max(0, 21 - __clz(high - low));
#pragma unroll
        for (int i = 0; i < PER; ++i) count[i * THREADS + tid] = 0;
        __syncthreads();
        for (int p0 = a.n_first; p0 < end; p0 += STRETCH) {
            if (!whole) load(p0);
            each(p0, [&](int i) {
                if (k[i] >= low && k[i] <= high) atomicAdd(&count[(k[i] - low) >> shift], 1u);
            });
        }
        __syncthreads();
        // how many lie above each thread's intervals, PER neighbours of them
        uint32_t mine[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) mine[i] = count[tid * PER + i], sum += mine[i];
        uint32_t from = sum;                          // its own and those of the wave's higher lanes
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t y = __shfl_down(static_cast<int>(from), m);
            if (lane + m < 64) from += y;
        }
        if (lane == 0) waves[wave] = from;
        __syncthreads();
        uint32_t above = from - sum;
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w > wave) above += waves[w];
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) {
            if (above < want && above + mine[i] >= want) found[0] = tid * PER + i, found[1] = want - above;
            above += mine[i];
        }
        __syncthreads();
        low += found[0] << shift;
        high = low + min(high - low, (1u << shift) - 1);
        want = found[1];
    }
    // keys above `low`, and the first `want` of those equal to it
    uint32_t more0 = 0, same0 = 0;                    // of the stretches before
    for (int p0 = a.n_first; p0 < end; p0 += STRETCH) {
        if (!whole) load(p0);
        uint64_t bm[EACH], bs[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const bool in = p0 + i * THREADS + tid < end;
            bm[i] = __ballot(in && k[i] > low), bs[i] = __ballot(in && k[i] == low);
            if (lane == 0) mores[i][wave] = __popcll(bm[i]), sames[i][wave] = __popcll(bs[i]);
        }
        __syncthreads();
        if (wave == 0) {                              // how many before each (i, wave), and of all
            constexpr int N = EACH * W / 64 ? EACH * W / 64 : 1;
            uint32_t m[N], s[N], ms = 0, ss = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int e = lane * N + j;
                m[j] = e < EACH * W ? (&mores[0][0])[e] : 0, s[j] = e < EACH * W ? (&sames[0][0])[e] : 0;
                ms += m[j], ss += s[j];
            }
            uint32_t mx = ms, sx = ss;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t y = __shfl_up(static_cast<int>(mx), d), z = __shfl_up(static_cast<int>(sx), d);
                if (lane >= d) mx += y, sx += z;
            }
            if (lane == 63) waves[0] = mx, waves[1] = sx;
            mx -= ms, sx -= ss;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int e = lane * N + j;
                if (e < EACH * W) (&mores[0][0])[e] = mx, (&sames[0][0])[e] = sx;
                mx += m[j], sx += s[j];
            }
        }
        __syncthreads();
        const uint64_t below = (1ull << lane) - 1;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint32_t before = more0 + mores[i][wave] + __popcll(bm[i] & below);
            const uint32_t equal = same0 + sames[i][wave] + __popcll(bs[i] & below);
            const uint32_t at = a.n_first + before + min(equal, want);
            // within the row also where another call has written to the same workspace meanwhile
            if (((bm[i] >> lane & 1) || ((bs[i] >> lane & 1) && equal < want)) && at < static_cast<uint32_t>(a.n_select - a.n_last))
                out[at] = p0 + i * THREADS + tid;
        }
        more0 += waves[0], same0 += waves[1];
        __syncthreads();
    }
}

constexpr int kFewPages = 256 * 4;     // of a table: a quarter of the threads select among them

stepq_status check(const stepq_cache_desc *c, const stepq_cache_select_desc *d)
{
    if (const stepq_status st = check_cache(c)) return st;
    if (!d) return bad("desc is NULL");
    if (d->n_q_heads < 1 || d->n_q_heads % c->n_kv_heads) return bad("n_q_heads must be a multiple of the cache's n_kv_heads, >= 1");
    if (!known_dtype(d->act_dtype)) return bad("unknown activation dtype");
    if (d->batch < 0 || d->max_pages < 0) return bad("negative count");
    if (d->n_select < 1 || d->n_first < 0 || d->n_last < 0 || int64_t(d->n_first) + d->n_last > d->n_select)
        return bad("n_select must be >= 1 and hold the n_first first and n_last last pages");
    if (static_cast<int64_t>(std::max(d->max_pages, d->n_select)) * c->page_size >= (int64_t(1) << 30))
        return set_error(STEPQ_E_UNSUPPORTED, "2^30 tokens or more in a request's pages or in its selected ones");
    if (static_cast<int64_t>(d->batch) * d->n_q_heads > (int64_t(1) << 23))
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^23 (request, head) rows in one call: split the batch");
    if (d->max_pages > kFewPages && static_cast<int64_t>(d->batch) * c->n_kv_heads >= (int64_t(1) << 22))
        return set_error(STEPQ_E_UNSUPPORTED, "2^22 or more (request, key/value head) pairs of many pages: split the batch");
    return STEPQ_OK;
}

size_t workspace_of(const stepq_cache_desc *c, const stepq_cache_select_desc *d)
{
    if (d->max_pages <= d->n_select) return 0;               // all pages are taken
    return static_cast<size_t>(d->batch) * c->n_kv_heads * d->max_pages * sizeof(uint32_t);
}

template <typename T>
void score(const SelectArgs &a, int D, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.batch) * a.Hkv * a.turns));
    if (D == 64) cache_score_kernel<T, 64><<<grid, 256, 0, s>>>(a);
    else if (D == 128) cache_score_kernel<T, 128><<<grid, 256, 0, s>>>(a);
    else cache_score_kernel<T, 256><<<grid, 256, 0, s>>>(a);
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_cache_select_workspace(const stepq_cache_desc *c, const stepq_cache_select_desc *d, size_t *bytes)
{
    if (const stepq_status st = check(c, d)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = workspace_of(c, d);
    return STEPQ_OK;
}

extern "C" stepq_status stepq_cache_select(const stepq_cache_desc *c, const stepq_cache_select_desc *d, const void *bounds,
                                           const void *q, const int32_t *page_table, const int32_t *lengths,
                                           int32_t *selected, void *workspace, size_t workspace_bytes, void *stream)
{
    if (const stepq_status st = check(c, d)) return st;
    if (d->batch == 0) return STEPQ_OK;
    if (d->max_pages && !page_table) return bad("page_table is NULL");
    if (!q || !lengths || !selected) return bad("NULL q, lengths or selected");
    if (c->n_pages && !bounds) return bad("NULL bounds");
    if (!aligned(q, 16) || !aligned(bounds, 16)) return bad("q and bounds must be 16-byte aligned");
    const size_t need = workspace_of(c, d);
    if (need && (!workspace || workspace_bytes < need)) return bad("workspace is smaller than stepq_cache_select_workspace()");
    if (!aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
    const int64_t pairs = static_cast<int64_t>(d->batch) * c->n_kv_heads;
    SelectArgs a{q, static_cast<const bf16_t *>(bounds), page_table, lengths, static_cast<uint32_t *>(workspace), selected,
                 d->batch, c->n_kv_heads, d->n_q_heads / c->n_kv_heads, c->n_pages, c->page_size, d->max_pages, d->n_select,
                 d->n_first, d->n_last, 1, fast_div(static_cast<uint32_t>(c->page_size))};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (need) {
        const int64_t at_once = 4 * 1024 / c->head_dim;      // pages of a workgroup's turn
        a.turns = static_cast<int32_t>(std::clamp<int64_t>(2048 / pairs, 1, (d->max_pages + at_once - 1) / at_once));
        if (d->act_dtype == STEPQ_BF16) score<bf16_t>(a, c->head_dim, s);
        else score<float>(a, c->head_dim, s);
    }
    const dim3 grid(static_cast<unsigned>(pairs));
    if (d->max_pages <= kFewPages) cache_select_kernel<256, 4><<<grid, 256, 0, s>>>(a);
    else cache_select_kernel<1024, 8><<<grid, 1024, 0, s>>>(a);
    return launched("cache select launch");
}
