// wq4_cache.h -- what the calls on a paged cache ask of its sizes.
#pragma once

#include "wq4_attn.h"

#include <cstdint>

namespace wq4 {

// Rows of a cache's keys: pages * heads * tokens of a page.  -1 where the kernels, which
// count them in int, could not; no product on the way passes 64 bits.
inline int64_t cache_rows(const wq4_kv_cache& c)
{
    constexpr int64_t kLimit = int64_t(1) << 31;
    const int64_t heads = static_cast<int64_t>(c.num_pages) * c.n_kv_heads;
    return heads < kLimit && heads * c.page_size < kLimit ? heads * c.page_size : -1;
}

}  // namespace wq4
