// A cache of keys and values as kernels see it, and the host's check of the caller's description.
#pragma once
#include "fgmp_internal.hpp"

namespace fgmp {

// (16 slots of one page are the unit by which kernels address a cache: one page lookup for 16 rows)
constexpr int kSlotGroup = 16;

struct CacheView {
    char *k, *v;
    const int32_t *page_table;
    const int32_t *lengths;
    int64_t page_stride, token_stride, head_stride;   // bytes
    int64_t table_stride;
    uint32_t pages, pages_per_sequence;
    uint32_t page_groups;        // slot groups per page; 0: no page table, sequence b's slots are page b
    int32_t page_shift;          // log2 of page_groups, -1 where it is no power of two
    int32_t slots;               // of a sequence
    int32_t batch, heads, head_dim;

    __device__ __forceinline__ int32_t length(int b) const
    {
        const int32_t n = lengths[b];
        return n < 0 ? 0 : n > slots ? slots : n;
    }
    // Byte offset of row 0 of slot group `u` of sequence b and head h (b, u, h uniform over the wave).  `*there` is cleared
    // where the page table's entry is none of the cache's pages (page 0 is given instead).
    __device__ __forceinline__ int64_t group_offset(int b, uint32_t u, int h, bool *there = nullptr) const
    {
        uint32_t page = (uint32_t)b, row = u;
        if (page_groups != 0u) {
            const uint32_t at = page_shift >= 0 ? u >> page_shift : u / page_groups;
            row = u - at * page_groups;
            page = (uint32_t)page_table[b * table_stride + at];
            if (page >= pages) {
                page = 0u;
                if (there != nullptr) *there = false;
            }
        }
        return (int64_t)page * page_stride + (int64_t)(row * kSlotGroup) * token_stride + (int64_t)h * head_stride;
    }
};

inline int dtype_size(fgmp_dtype_t dt) { return dt == FGMP_F32 ? 4 : 2; }
inline bool known_dtype(fgmp_dtype_t dt) { return dt == FGMP_F32 || dt == FGMP_BF16; }
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0u; }

fgmp_status_t check_cache(const fgmp_cache_t *c, CacheView *view);
// batch x tokens x heads vectors of `dim` elements of `size` bytes; `written`: no two of them may share memory
fgmp_status_t check_heads(const fgmp_heads_t *x, int64_t batch, int64_t tokens, int64_t heads, int dim, int size, bool written);

}  // namespace fgmp
