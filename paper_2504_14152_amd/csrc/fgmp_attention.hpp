// What the attention kernels share: their arguments, how a sequence is split, and steps of the softmax.
#pragma once
#include <algorithm>

#include "fgmp_cache.hpp"

namespace fgmp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The maximum only keeps the exponentials in range: results are scaled to a new one when it is 2^kSlack times the old one's weight, not at
// every small step up, which some row of 32 makes in nearly every tile.
constexpr float kSlack = 8.0f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttendArgs {
    CacheView c;
    const char *q, *k, *v;
    char *out;
    float *lse;
    int64_t q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head, o_batch, o_token, o_head;   // bytes
    const uint64_t *tree;
    const int32_t *counts;
    int32_t tokens, q_heads, group, words;
    uint32_t row_blocks;             // workgroups that share the rows of a sequence and head
    uint32_t units;                  // ranges of keys: batch x heads x splits
    int32_t splits;                  // most ranges of a sequence
    int32_t tile_keys, min_tiles;    // ranges are whole tiles, and at least so many
    float c2;                        // scale * log2(e)
    float *part_o, *part_ml;         // partial results of each range: [row][split][dim], [row][split][2]

    __device__ __forceinline__ int32_t count(int b) const
    {
        const int32_t n = counts != nullptr ? counts[b] : tokens;
        return n < 0 ? 0 : n > tokens ? tokens : n;
    }
    // Tiles of a range, and ranges in use, of a sequence of n slots: it is dealt out in equal ranges.
    __device__ __forceinline__ int tiles(int32_t n) const { return (int)(((uint32_t)n + tile_keys - 1) / (uint32_t)tile_keys); }
    __device__ __forceinline__ int range(int32_t n) const { return std::max(min_tiles, (tiles(n) + splits - 1) / splits); }
    __device__ __forceinline__ int ranges(int32_t n) const { return std::max(1, (tiles(n) + range(n) - 1) / range(n)); }
};

// Which part of the work a workgroup has.  Workgroups go round the XCDs: those of the same rest of 8 follow each other on one XCD.  They
// are the row blocks of one head's range of keys, of which all but the first find its keys and values in that XCD's L2, then other ranges.
struct AttendPlace {
    int b, h, split, block;
    bool there;
    __device__ __forceinline__ explicit AttendPlace(const AttendArgs &a)
    {
        const uint32_t turn = blockIdx.x / 8u / a.row_blocks;
        block = (int)(blockIdx.x / 8u % a.row_blocks);
        uint32_t unit = turn * 8u + blockIdx.x % 8u;
        there = unit < a.units;
        split = (int)(unit % (uint32_t)a.splits);
        unit /= (uint32_t)a.splits;
        h = (int)(unit % (uint32_t)a.c.heads);
        b = (int)(unit / (uint32_t)a.c.heads);
    }
};

__device__ __forceinline__ float logsumexp(float most, float l, float c2)
{
    return l == 0.0f ? -INFINITY : (most * c2 + __builtin_amdgcn_logf(l)) * kLn2;
}
// 1 / l; 0 where nothing was seen; NaN stays
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l; }

// BF16: 32 rows in each of 4 or 8 waves, 4 with head_dim 256 (fgmp_attention_wide.hip)
constexpr int wide_keys(int head_dim) { return head_dim == 256 ? 32 : 64; }
void attend_wide(const AttendArgs &a, int waves, uint32_t workgroups, hipStream_t st);

}  // namespace fgmp
