// Attention of single tokens over a shared prefix and each request's own pages.
#include <cmath>

#include "stepq_plan.h"
#include "stepq_seq.h"

namespace stepq {
namespace {

struct AttnArgs {
    const void *q, *k, *v;
    const int32_t *prefix_pages, *table, *lengths;
    void *o;
    float *lse;
    int64_t prefix;
    int32_t batch, Hq, Hkv, n_pages, page, max_pages;
    FastDiv div_page;
    float scale;             // times log2 e: scores are kept in powers of two
};

__device__ __forceinline__ int fdiv(int n, FastDiv d)
{
    const uint32_t u = static_cast<uint32_t>(n);
    return static_cast<int>((__umulhi(u, d.mul) + u) >> d.shift);
}

constexpr float kLn2 = 0.6931471805599453f;

// One workgroup per (request, query head), a wave per key: the lanes hold the
// query, the key's product is summed over the wave, the running maximum and
// sum rescale the accumulator.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_rows_kernel(AttnArgs a)
{
    constexpr int E = D / 64;
    __shared__ float sm[4], sl[4], sacc[4][D];
    const int b = blockIdx.x / a.Hq, h = blockIdx.x - b * a.Hq, hk = h / (a.Hq / a.Hkv);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const size_t row = (static_cast<size_t>(b) * a.Hq + h) * D;
    float q[E], acc[E] = {}, m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = widen(static_cast<const T *>(a.q)[row + e * 64 + lane]) * a.scale;
    const int mine = static_cast<int>(min(static_cast<int64_t>(max(a.lengths[b], 0)), static_cast<int64_t>(a.max_pages) * a.page));
    for (int part = 0; part < 2; ++part) {
        const int n = part ? mine : static_cast<int>(a.prefix);
        const int32_t *pages = part ? a.table + static_cast<size_t>(b) * a.max_pages : a.prefix_pages;
        for (int t = wave; t < n; t += 4) {
            const int p = fdiv(t, a.div_page), id = pages[p];
            if (id < 0 || id >= a.n_pages) continue;
            const size_t at = ((static_cast<size_t>(id) * a.Hkv + hk) * a.page + (t - p * a.page)) * D;
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) s = fmaf(q[e], widen(static_cast<const T *>(a.k)[at + e * 64 + lane]), s);
#pragma unroll
            for (int x = 32; x > 0; x >>= 1) s += __shfl_xor(s, x);
            const float top = fmaxf(m, s), base = top == -INFINITY ? 0.0f : top;
            const float f = exp2f(m - base), w = exp2f(s - base);
            l = fmaf(l, f, w);
#pragma unroll
            for (int e = 0; e < E; ++e)
                acc[e] = fmaf(w, widen(static_cast<const T *>(a.v)[at + e * 64 + lane]), acc[e] * f);
            m = top;
        }
    }
    if (lane == 0) sm[wave] = m, sl[wave] = l;
#pragma unroll
    for (int e = 0; e < E; ++e) sacc[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    float top = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    const float base = top == -INFINITY ? 0.0f : top;
    float z = 0.0f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) f[w] = exp2f(sm[w] - base), z += sl[w] * f[w];
    for (int e = threadIdx.x; e < D; e += 256) {
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) y = fmaf(f[w], sacc[w][e], y);
        static_cast<T *>(a.o)[row + e] = narrow<T>(z == 0.0f ? 0.0f : y / z);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[row / D] = z == 0.0f ? -INFINITY : (base + log2f(z)) * kLn2;
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
    if (static_cast<int64_t>(d->batch) * d->n_q_heads > (int64_t(1) << 24))
        return set_error(STEPQ_E_UNSUPPORTED, "more than 2^24 (request, head) rows in one call: split the batch");
    return STEPQ_OK;
}

template <typename T>
void launch(const AttnArgs &a, int D, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(a.batch) * a.Hq);
    if (D == 64) attn_rows_kernel<T, 64><<<grid, 256, 0, s>>>(a);
    else if (D == 128) attn_rows_kernel<T, 128><<<grid, 256, 0, s>>>(a);
    else attn_rows_kernel<T, 256><<<grid, 256, 0, s>>>(a);
}

}  // namespace
}  // namespace stepq

using namespace stepq;

extern "C" stepq_status stepq_prefix_attention_workspace(const stepq_attn_desc *d, size_t *bytes)
{
    if (const stepq_status st = check(d)) return st;
    if (!bytes) return bad("bytes is NULL");
    *bytes = 0;
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
    AttnArgs a{q, k_cache, v_cache, prefix_pages, page_table, lengths, o, lse, d->prefix_len, d->batch, d->n_q_heads,
               d->n_kv_heads, d->n_pages, d->page_size, d->max_pages, fast_div(static_cast<uint32_t>(d->page_size)),
               d->scale * 1.4426950408889634f};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->act_dtype == STEPQ_BF16) launch<bf16_t>(a, d->head_dim, s);
    else launch<float>(a, d->head_dim, s);
    return launched("prefix attention launch");
}
