// Where a position of a sequence lies in the paged cache.
#pragma once

#include "lm_common.h"
#include "lm_internal.h"

namespace qnn_lm {

struct Slot {
    int32_t page, slot;  // page < 0: not in the cache
};

// Table entries are read from the device and bounded here, so that no length,
// position or page number leads outside of the cache.
__device__ __forceinline__ Slot find_slot(const CacheArgs &c, int32_t seq, int64_t pos)
{
    Slot s = {-1, 0};
    if (pos < 0 || pos >= (int64_t)c.width * c.page)
        return s;
    const int32_t p = qnn::fdiv((uint32_t)pos, c.page_div);  // width * page < 2^31
    const int32_t page = c.table[(int64_t)seq * c.width + p];
    if ((uint32_t)page < (uint32_t)c.pages) {
        s.page = page;
        s.slot = (int32_t)pos - p * c.page;
    }
    return s;
}

__device__ __forceinline__ int64_t scale_at(const CacheArgs &c, Slot s, int32_t head)
{
    return ((int64_t)s.page * c.heads + head) * c.page + s.slot;
}

}  // namespace qnn_lm
