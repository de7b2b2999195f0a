// A cache of keys and values as kernels see it, and the host's check of the caller's description.
#pragma once
#include "fgmp_internal.hpp"

namespace fgmp {

// (16 slots of one page are the unit by which kernels address a cache: one page lookup for 16 rows)
constexpr int kSlotGroup = 16;

struct CacheView {
    char *k, *v;
    const int32_t *page_table;   // null: sequence b's slots are page b
    const int32_t *lengths;
    int64_t page_stride, token_stride, head_stride;   // bytes
    int64_t table_stride;
    uint32_t pages, pages_per_sequence;
    uint32_t page_groups;        // slot groups per page
    uint32_t group_factor, group_shift;   // u / page_groups = u * factor >> shift for u < 2^27; factor 0 without a page table (one page, all slots)
    int32_t slots;               // of a sequence
    int32_t batch, heads, head_dim;

    __device__ __forceinline__ int32_t length(int b) const
    {
        const int32_t n = lengths[b];
        return n < 0 ? 0 : n > slots ? slots : n;
    }
    // Which entry of its row of the page table slot group `u` falls under; `*row`: its first slot in that page.
    __device__ __forceinline__ uint32_t entry_of(uint32_t u, uint32_t *row) const
    {
        const uint32_t at = (uint32_t)((uint64_t)u * group_factor >> group_shift);   // u / page_groups
        *row = (u - at * page_groups) * kSlotGroup;
        return at;
    }
    // The page table is not written while a kernel runs: read as constant memory, through the scalar cache where `at` is uniform.
    __device__ __forceinline__ uint32_t page_of(int b, uint32_t at) const
    {
        typedef const __attribute__((address_space(4))) int32_t *constant;
        return page_table != nullptr ? (uint32_t)((constant)(uintptr_t)page_table)[b * table_stride + at] : (uint32_t)b;
    }
    // Byte offset of row `row` of page `page` of a head; `*there`: whether there is such a page (if not, page 0 is given instead).
    __device__ __forceinline__ int64_t offset(uint32_t page, uint32_t row, int h, bool *there = nullptr) const
    {
        if (there != nullptr) *there = page < pages;
        page = page < pages ? page : 0u;
        return (int64_t)page * page_stride + (int64_t)row * token_stride + (int64_t)h * head_stride;
    }
    // ... of row 0 of slot group `u` of sequence b.
    __device__ __forceinline__ int64_t group_offset(int b, uint32_t u, int h, bool *there = nullptr) const
    {
        uint32_t row;
        const uint32_t at = entry_of(u, &row);
        return offset(page_of(b, at), row, h, there);
    }
};

// A launch counts its threads in 32 bits, not its workgroups: one of more does not take place.
inline bool launch_counts(int64_t workgroups, int64_t threads) { return workgroups < ((int64_t)1 << 32) / threads; }

inline int dtype_size(fgmp_dtype_t dt) { return dt == FGMP_F32 ? 4 : 2; }
inline bool known_dtype(fgmp_dtype_t dt) { return dt == FGMP_F32 || dt == FGMP_BF16; }
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0u; }

fgmp_status_t check_cache(const fgmp_cache_t *c, CacheView *view);
// batch x tokens x heads vectors of `dim` elements of `size` bytes; `written`: no two of them may share memory
fgmp_status_t check_heads(const fgmp_heads_t *x, int64_t batch, int64_t tokens, int64_t heads, int dim, int size, bool written);

}  // namespace fgmp
