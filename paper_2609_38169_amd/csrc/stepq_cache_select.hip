// The pages of a quantized cache that a request's query may need most, by the bounds of their keys.
#include <algorithm>

#include "stepq_cache.h"

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
    return len ? page_of(len - 1, a.div_page) + 1 : 0;
}

// Scores as whole numbers that order as they do; NaN above all (and 0, below -inf, for a page that there is not).
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    return x != x ? 0xffffffffu : u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// score = sum_d hi_d sum_h max(q_hd, 0) + lo_d sum_h min(q_hd, 0): a lane keeps
// the sums over the heads for 8 dimensions of one bound and takes page after page;
// D/4 lanes make a page's score.  In 64 bits, so that no order of summation
// tells: the score is rounded once.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_score_kernel(SelectArgs a)
{
    constexpr int lanes = D / 4, at_once = 256 / lanes;
    const int lane = threadIdx.x % lanes, sub = threadIdx.x / lanes;
    int x = blockIdx.x;
    const int turn = x % a.turns;
    x /= a.turns;
    const int hk = x % a.Hkv, b = x / a.Hkv;
    const int pages = pages_of(a, b);
    if (pages <= a.n_select) return;             // all are taken
    const int end = pages - a.n_last;
    const bool high = lane >= lanes / 2;
    const int d0 = lane % (lanes / 2) * 8;
    double w[8] = {};
    const T *q = static_cast<const T *>(a.q) + (static_cast<size_t>(b) * a.Hkv + hk) * a.G * D + d0;
    for (int h = 0; h < a.G; ++h)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = widen(q[static_cast<size_t>(h) * D + i]);
            // a NaN reaches both sums
            w[i] += static_cast<double>(high ? (y < 0.0f ? 0.0f : y) : (y > 0.0f ? 0.0f : y));
        }
    const int32_t *table = a.table + static_cast<size_t>(b) * a.max_pages;
    uint32_t *keys = a.keys + (static_cast<size_t>(b) * a.Hkv + hk) * a.max_pages;
    for (int p0 = a.n_first + turn * at_once; p0 < end; p0 += a.turns * at_once) {
        const int p = p0 + sub;
        const int id = p < end ? table[p] : -1;
        const bool there = id >= 0 && id < a.n_pages;
        double sum = 0.0;
        if (there) {
            const uint4 v = *reinterpret_cast<const uint4 *>(a.bounds + ((static_cast<size_t>(id) * a.Hkv + hk) * 2 + high) * D + d0);
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                sum = fma(w[i], static_cast<double>(__uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16)), sum);
        }
#pragma unroll
        for (int m = 1; m < lanes; m <<= 1) sum += __shfl_xor(sum, m);
        if (lane == 0 && p < end) keys[p] = there ? key_of(static_cast<float>(sum)) : 0;
    }
}

// The n_first first and n_last last pages and the highest scores between them,
// ties to the lowest position: the lowest score that is taken found digit by digit
// of its key (8 bits each), then one pass over the pages in order.
__global__ __launch_bounds__(256) void cache_select_kernel(SelectArgs a)
{
    __shared__ uint32_t count[256];
    __shared__ uint32_t chosen[2], before[4][2];
    const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int pages = pages_of(a, b);
    int32_t *out = a.selected + (static_cast<size_t>(b) * a.Hkv + hk) * a.n_select;
    if (pages <= a.n_select) {
        for (int i = tid; i < a.n_select; i += 256) out[i] = i < pages ? i : -1;
        return;
    }
    const uint32_t *keys = a.keys + (static_cast<size_t>(b) * a.Hkv + hk) * a.max_pages;
    const int end = pages - a.n_last;
    uint32_t want = a.n_select - a.n_first - a.n_last, prefix = 0, mask = 0;
    for (int i = tid; i < a.n_first; i += 256) out[i] = i;
    for (int i = tid; i < a.n_last; i += 256) out[a.n_select - a.n_last + i] = end + i;
    if (want == 0) return;
    // of the keys that begin with `prefix`, the want-th highest is looked for
    for (int shift = 24; shift >= 0; shift -= 8) {
        count[tid] = 0;
        __syncthreads();
        for (int p = a.n_first + tid; p < end; p += 256) {
            const uint32_t k = keys[p];
            if ((k & mask) == prefix) atomicAdd(&count[k >> shift & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            uint32_t left = want;
            int d = 255;
            for (; d > 0 && count[d] < left; --d) left -= count[d];
            chosen[0] = static_cast<uint32_t>(d), chosen[1] = left;
        }
        __syncthreads();
        prefix |= chosen[0] << shift, mask |= 255u << shift, want = chosen[1];
        __syncthreads();
    }
    // keys above `prefix`, and the first `want` of those equal to it
    uint32_t taken = 0, equal = 0;
    for (int p0 = a.n_first; p0 < end; p0 += 256) {
        const int p = p0 + tid;
        const uint32_t k = p < end ? keys[p] : 0;
        const bool more = p < end && k > prefix, same = p < end && k == prefix;
        const uint64_t ms = __ballot(same);
        const uint32_t es = __popcll(ms & ((1ull << lane) - 1));
        if (lane == 0) before[wave][0] = __popcll(ms);
        __syncthreads();
        uint32_t e = equal + es, all_e = equal;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) e += before[w][0];
            all_e += before[w][0];
        }
        const bool take = more || (same && e < want);
        const uint64_t mt = __ballot(take);
        if (lane == 0) before[wave][1] = __popcll(mt);
        __syncthreads();
        uint32_t at = taken + __popcll(mt & ((1ull << lane) - 1)), all_t = taken;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) at += before[w][1];
            all_t += before[w][1];
        }
        if (take) out[a.n_first + at] = p;
        taken = all_t, equal = all_e;
        __syncthreads();
    }
}

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
    if (!aligned(q, d->act_dtype == STEPQ_F32 ? 4 : 2) || !aligned(bounds, 16)) return bad("bounds must be 16-byte aligned, q to its type");
    const size_t need = workspace_of(c, d);
    if (need && (!workspace || workspace_bytes < need)) return bad("workspace is smaller than stepq_cache_select_workspace()");
    if (!aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
    const int64_t pairs = static_cast<int64_t>(d->batch) * c->n_kv_heads;
    SelectArgs a{q, static_cast<const bf16_t *>(bounds), page_table, lengths, static_cast<uint32_t *>(workspace), selected,
                 d->batch, c->n_kv_heads, d->n_q_heads / c->n_kv_heads, c->n_pages, c->page_size, d->max_pages, d->n_select,
                 d->n_first, d->n_last, 1, fast_div(static_cast<uint32_t>(c->page_size))};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (need) {
        const int64_t at_once = 1024 / c->head_dim;          // pages of a workgroup's turn
        a.turns = static_cast<int32_t>(std::clamp<int64_t>(2048 / pairs, 1, (d->max_pages + at_once - 1) / at_once));
        if (d->act_dtype == STEPQ_BF16) score<bf16_t>(a, c->head_dim, s);
        else score<float>(a, c->head_dim, s);
    }
    cache_select_kernel<<<dim3(static_cast<unsigned>(pairs)), 256, 0, s>>>(a);
    return launched("cache select launch");
}
