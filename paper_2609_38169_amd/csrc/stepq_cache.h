// Quantized key/value caches: the place of a token's rows in a page's record
// (the layout is defined in include/stepq.h), and the checks of their descriptor.
#pragma once

#include "stepq_div.h"
#include "stepq_plan.h"
#include "stepq_seq.h"

namespace stepq {

constexpr int kGroup4 = 64;              // elements under one scale of 4-bit codes; 8-bit codes: the whole row

struct CacheShape {
    int32_t row, scales;                 // bytes of a row's codes, scales of a row
    int64_t record;                      // bytes of a (page, head) record
};

inline CacheShape cache_shape(const stepq_cache_desc *d)
{
    CacheShape s{};
    s.row = d->head_dim * d->bits / 8;
    s.scales = d->bits == 8 ? 1 : d->head_dim / kGroup4;
    s.record = (int64_t(2) * d->page_size * (s.row + 2 * s.scales) + 127) / 128 * 128;
    return s;
}

// What the kernels see of a cache.
struct CacheView {
    uint8_t *mem;
    int64_t record;
    int32_t n_pages, Hkv, page;
    FastDiv div_page;
};

inline CacheView cache_view(const stepq_cache_desc *d, const void *mem)
{
    return {static_cast<uint8_t *>(const_cast<void *>(mem)), cache_shape(d).record, d->n_pages, d->n_kv_heads, d->page_size,
            fast_div(static_cast<uint32_t>(d->page_size))};
}

stepq_status check_cache(const stepq_cache_desc *d);
// A cache's memory and the tables of a call with n requests of max_pages pages each.
stepq_status check_paged(const stepq_cache_desc *d, const void *cache, int32_t n, int32_t max_pages, const int32_t *page_table);

// The record of head hk of page id; NULL: no such page.
__device__ __forceinline__ uint8_t *record_of(const CacheView &c, int id, int hk)
{
    return id >= 0 && id < c.n_pages ? c.mem + (static_cast<int64_t>(id) * c.Hkv + hk) * c.record : nullptr;
}

// Byte offsets in a record: row r's codes and scales; values lie behind keys.
template <int D, int BITS>
struct RowOf {
    static constexpr int bytes = D * BITS / 8, scales = BITS == 8 ? 1 : D / kGroup4;
    static __device__ __forceinline__ int codes(int page, bool value, int r) { return ((value ? page : 0) + r) * bytes; }
    static __device__ __forceinline__ int scale(int page, bool value, int r)
    {
        return 2 * page * bytes + ((value ? page : 0) + r) * 2 * scales;
    }
};

}  // namespace stepq
