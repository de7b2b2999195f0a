// A cache in 8 bits as kernels see it: codes as any cache's elements, and a scale byte for each slot and head, heads outside of slots, so that the
// scales of 16 slots lie next to each other.
#pragma once
#include "fgmp_cache.hpp"

namespace fgmp {

struct QuantCacheView {
    CacheView c;                          // codes: elements of one byte
    uint8_t *k_scales, *v_scales;
    int64_t scale_page, scale_head;       // bytes
    __device__ __forceinline__ int64_t scale_at(uint32_t page, uint32_t row, int h) const
    {
        return (int64_t)page * scale_page + (int64_t)h * scale_head + row;
    }
};

fgmp_status_t check_quant_cache(const fgmp_quant_cache_t *c, QuantCacheView *view);

}  // namespace fgmp
