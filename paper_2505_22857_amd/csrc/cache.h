// The paged cache of keys and values as the kernels see it.
#pragma once

#include "ngpu_lm.h"
#include "values.h"

namespace ngpu {

// A page table over a sequence's tokens.
struct PageTable {
    const int32_t *pages;
    int64_t count;       // tokens, no more than the table holds

    // The page of token j and its entry there; a page outside the cache: -1.
    __device__ __forceinline__ int64_t page(const ngpu_kv_cache_t &c, int64_t j, int64_t &entry) const {
        const int64_t at = j / c.page_size;
        entry = j - at * c.page_size;
        const int64_t p = pages[at];
        return p >= 0 && p < c.num_pages ? p : -1;
    }
};

}  // namespace ngpu
