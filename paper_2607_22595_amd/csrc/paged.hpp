// The paged cache on the device: where its pointers lie for the graph executor,
// and which page holds a position.
#pragma once

#include <stddef.h>

#include "common.hpp"
#include "kernels.hpp"
#include "launch.hpp"

namespace xmix {

template <>
struct ArgPointers<KvCacheIn> {
    static std::vector<uint16_t> offsets() {
        return {offsetof(KvCacheIn, k), offsetof(KvCacheIn, v), offsetof(KvCacheIn, pages),
                offsetof(KvCacheIn, k_scale), offsetof(KvCacheIn, v_scale)};
    }
};

// The page id at entry `nth` of request req's table; `nth` must lie in the table.
__device__ __forceinline__ int32_t page_at(const KvCacheIn& c, int32_t req, int32_t nth) {
    return c.pages[static_cast<int64_t>(req) * c.max_pages + nth];
}
__device__ __forceinline__ bool page_ok(const KvCacheIn& c, int32_t page) {
    return static_cast<uint32_t>(page) < static_cast<uint32_t>(c.n_pages);
}
// Row of the key (or value) of one head at slot `slot` of a page, counted in rows
// of head_dim values from the start of the cache.
__device__ __forceinline__ int64_t page_row(const KvCacheIn& c, int32_t page, int32_t head,
                                            int32_t slot) {
    return ((static_cast<int64_t>(page) * c.n_kv + head) << c.page_log2) + slot;
}

}  // namespace xmix
