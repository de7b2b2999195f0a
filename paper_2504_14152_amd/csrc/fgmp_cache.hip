// Upkeep of a cache of keys and values: accepted tokens appended, entries evicted by accumulated attention weight.
#include <algorithm>

#include "fgmp_cache.hpp"

namespace fgmp {

fgmp_status_t check_cache(const fgmp_cache_t *c, CacheView *view)
{
    if (c == nullptr || !known_dtype(c->dtype)) return FGMP_ERR_INVALID_ARG;
    return check_cache_of(c, dtype_size(c->dtype), view);
}

fgmp_status_t check_cache_of(const fgmp_cache_t *c, int size, CacheView *view)
{
    if (c->k == nullptr || c->v == nullptr || c->lengths == nullptr) return FGMP_ERR_INVALID_ARG;
    if (c->batch <= 0 || c->heads <= 0 || c->page_size <= 0 || c->pages_per_sequence <= 0 || c->pages <= 0) return FGMP_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return FGMP_ERR_UNSUPPORTED;
    const bool paged = c->page_table != nullptr;
    const int unit = 16 / size;
    if (paged ? c->page_size % kSlotGroup != 0 || c->table_stride < c->pages_per_sequence : c->pages_per_sequence != 1 || c->pages < c->batch)
        return FGMP_ERR_BAD_SHAPE;
    // (the stride of a single page or head is taken times zero)
    const int64_t page_stride = c->pages > 1 ? c->page_stride : c->head_dim, head_stride = c->heads > 1 ? c->head_stride : c->head_dim;
    if (c->token_stride < c->head_dim || head_stride < c->head_dim || page_stride < c->head_dim) return FGMP_ERR_BAD_SHAPE;
    if (!aligned16(c->k) || !aligned16(c->v) || page_stride % unit != 0 || c->token_stride % unit != 0 || head_stride % unit != 0)
        return FGMP_ERR_BAD_ALIGN;
    if (((uintptr_t)c->lengths & 3u) != 0u || ((uintptr_t)c->page_table & 3u) != 0u) return FGMP_ERR_BAD_ALIGN;
    // offsets within a group of slots are 32-bit, slots and pages are counted in 31 bits
    const int64_t slots = (int64_t)c->page_size * c->pages_per_sequence;
    if (c->token_stride > (int64_t)1 << 26 || page_stride > (int64_t)1 << 40 || head_stride > (int64_t)1 << 40 || slots > (int64_t)1 << 30 || c->pages > (int64_t)1 << 31 || c->batch > 65535 || c->heads > 65535)
        return FGMP_ERR_UNSUPPORTED;
    *view = CacheView{};
    view->k = static_cast<char *>(c->k);
    view->v = static_cast<char *>(c->v);
    view->page_table = c->page_table;
    view->lengths = c->lengths;
    view->page_stride = page_stride * size;
    view->token_stride = c->token_stride * size;
    view->head_stride = head_stride * size;
    view->table_stride = c->table_stride;
    view->pages = (uint32_t)c->pages;
    view->pages_per_sequence = (uint32_t)c->pages_per_sequence;
    view->page_groups = paged ? (uint32_t)(c->page_size / kSlotGroup) : 0u;
    if (paged) {
        // with 2^k >= d the factor 2^(27 + k) / d, rounded up, is off by less than 1 in 2^27 of a quotient's unit for u < 2^27
        uint32_t k = 0;
        while ((1u << k) < view->page_groups) ++k;
        view->group_shift = 27u + k;
        view->group_factor = (uint32_t)((((uint64_t)1 << view->group_shift) + view->page_groups - 1) / view->page_groups);
    }
    view->slots = (int32_t)slots;
    view->batch = c->batch;
    view->heads = c->heads;
    view->head_dim = c->head_dim;
    return FGMP_OK;
}

fgmp_status_t check_heads(const fgmp_heads_t *x, int64_t batch, int64_t tokens, int64_t heads, int dim, int size, bool written)
{
    if (x == nullptr || x->data == nullptr) return FGMP_ERR_INVALID_ARG;
    const int64_t strides[3] = {x->batch_stride, x->token_stride, x->head_stride}, counts[3] = {batch, tokens, heads};
    for (int i = 0; i < 3; ++i) {
        if (counts[i] == 1) continue;   // (always taken times zero)
        if (strides[i] < 0 || (written && strides[i] < dim)) return FGMP_ERR_BAD_SHAPE;
        if (strides[i] % (16 / size) != 0) return FGMP_ERR_BAD_ALIGN;
        if (strides[i] > (int64_t)1 << 40) return FGMP_ERR_UNSUPPORTED;
    }
    return aligned16(x->data) ? FGMP_OK : FGMP_ERR_BAD_ALIGN;
}

namespace {

struct HeadsView {
    const char *k, *v;
    int64_t k_batch, k_token, k_head, v_batch, v_token, v_head;   // bytes
};

// ---- append ----
//
// A copy: every thread moves 16 bytes of the cache's type at a time, first of a key, then of a value.

template <bool kFromF32, bool kToF32>
__device__ __forceinline__ uint4 converted(const char *src)   // 16 bytes of the cache's type
{
    if constexpr (kFromF32 == kToF32) {
        return *reinterpret_cast<const uint4 *>(src);
    } else if constexpr (kFromF32) {
        typedef float f32x8 __attribute__((ext_vector_type(8)));
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        const f32x8 x = *reinterpret_cast<const f32x8 *>(__builtin_assume_aligned(src, 16));
        return __builtin_bit_cast(uint4, __builtin_convertvector(x, bf16x8));   // (nearest even)
    } else {
        const uint2 x = *reinterpret_cast<const uint2 *>(src);
        return make_uint4(x.x << 16, x.x & 0xFFFF0000u, x.y << 16, x.y & 0xFFFF0000u);
    }
}

struct AppendArgs {
    CacheView c;
    HeadsView in;
    int64_t tokens, accepted;
    const int32_t *rows, *counts, *positions;
    int32_t *slot_positions, *lengths_out;
    float *slot_weights;
    int64_t slot_stride;
    int32_t pieces;       // 16-byte pieces of a token's keys
    int32_t per_token;    // workgroups that share a token
    int32_t piece_shift;  // log2 of the pieces of one head
};

template <bool kFromF32, bool kToF32>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a)
{
    const int64_t token = blockIdx.x / a.per_token;
    const int part = blockIdx.x % a.per_token;
    const int b = (int)(token / a.accepted), i = (int)(token % a.accepted);
    const int32_t n = a.c.length(b);
    int32_t count = a.counts != nullptr ? a.counts[b] : (int32_t)a.accepted;
    count = count < 0 ? 0 : count > a.accepted ? (int32_t)a.accepted : count;
    if (i == 0 && part == 0 && threadIdx.x == 0) {
        const int64_t left = (int64_t)n + count;
        a.lengths_out[b] = left > a.c.slots ? a.c.slots : (int32_t)left;
    }
    if (i >= count || n + i >= a.c.slots) return;
    const int32_t row = a.rows != nullptr ? a.rows[b * a.accepted + i] : i;
    if ((uint32_t)row >= (uint32_t)a.tokens) return;
    const int32_t slot = n + i;
    bool there = true;
    const int64_t to = a.c.group_offset(b, (uint32_t)slot / kSlotGroup, 0, &there) + (int64_t)(slot % kSlotGroup) * a.c.token_stride;
    const int64_t from_k = b * a.in.k_batch + row * a.in.k_token, from_v = b * a.in.v_batch + row * a.in.v_token;
    const int from_size = kFromF32 == kToF32 ? 16 : kFromF32 ? 32 : 8;
    if (there) {
        for (int p = part * 256 + (int)threadIdx.x; p < a.pieces; p += a.per_token * 256) {
            const int h = p >> a.piece_shift, at = p & ((1 << a.piece_shift) - 1);
            const uint4 x = converted<kFromF32, kToF32>(a.in.k + from_k + h * a.in.k_head + at * from_size);
            const uint4 y = converted<kFromF32, kToF32>(a.in.v + from_v + h * a.in.v_head + at * from_size);
            *reinterpret_cast<uint4 *>(a.c.k + to + h * a.c.head_stride + at * 16) = x;
            *reinterpret_cast<uint4 *>(a.c.v + to + h * a.c.head_stride + at * 16) = y;
        }
    }
    if (part == 0) {
        for (int h = threadIdx.x; h < a.c.heads; h += 256) {
            const int64_t e = ((int64_t)b * a.c.heads + h) * a.slot_stride + slot;
            if (a.slot_positions != nullptr) a.slot_positions[e] = a.positions[b * a.tokens + row];
            if (a.slot_weights != nullptr) a.slot_weights[e] = 0.0f;
        }
    }
}

// ---- evict ----

// Orders like the numbers (NaN below them, both zeros alike); the top value is kept for entries that stay whatever they weigh.
__device__ __forceinline__ uint32_t rank_of(float w)
{
    uint32_t bits = __builtin_bit_cast(uint32_t, w + 0.0f);
    if (w != w) return 0u;
    if (w == 0.0f) bits = 0u;
    return (bits & 0x80000000u) != 0u ? ~bits : bits | 0x80000000u;
}

struct EvictArgs {
    CacheView c;
    const float *weights;
    const int32_t *positions, *seen;
    float *weights_out;
    int32_t *positions_out, *lengths_out;
    int64_t slot_stride;
    int32_t budget, sinks, recent;
    uint32_t *moved;       // per sequence and head: entries that move
    int2 *moves;           // ... and their slots, (from, to), `room` each
    int64_t room;
};

constexpr int kRankBits = 11, kRankBins = 1 << kRankBits;   // 32 bits in digits of 11, 11 and 10

// Sum of `mine` over the threads before this one in the workgroup, and over all of them.  One barrier: two calls that follow each other
// need parts of their own.
template <int kWaves>
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t mine, uint32_t *part, uint32_t *all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // within rows of 16 lanes, then the rows' sums on to the rows behind
    uint32_t incl = mine;
    incl += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, 0x111, 0xF, 0xF, false);
    incl += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, 0x112, 0xF, 0xF, false);
    incl += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, 0x114, 0xF, 0xF, false);
    incl += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, 0x118, 0xF, 0xF, false);
    incl += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, 0x142, 0xA, 0xF, false);
    incl += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)incl, 0x143, 0xC, 0xF, false);
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    uint32_t before = 0u, sum = 0u;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t v = part[w];
        before += w < wave ? v : 0u;
        sum += v;
    }
    *all = sum;
    return before + incl - mine;
}

// One workgroup per sequence and head: the rank of the budget-th entry by radix selection, then who stays, and the i-th entry that stays
// behind the budget is paired with the i-th place that becomes free below it.  A thread holds the ranks of 4 kQuads slots next to each other
// in registers (of that many times kThreads slots at a time where a sequence has more: then they are read again in every pass), so weights
// and positions are read once, and the order over the workgroup takes one sum over threads instead of one for every kThreads slots.
// Weights share a few exponents: digits of 11 bits take mantissa bits in from the first pass on, and copies of the bins keep the lanes of a
// wave apart.  64 heads of 16381 slots: 62 us with digits of 8 bits and two sums for every 1024 slots, 19 so (64 of 1031: 11 and 6.5); what
// is left is latency, of the first loads, of bins and barriers.
template <int kThreads, int kQuads>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(EvictArgs a)
{
    constexpr int kWaves = kThreads / 64, kCopies = kThreads / 256, kSpan = 4 * kQuads, kBinsPer = kRankBins / kThreads;
    __shared__ uint32_t hist[kCopies][kRankBins];
    __shared__ uint32_t part[2][kWaves];
    __shared__ uint32_t found[2];
    const int b = blockIdx.x / a.c.heads, h = blockIdx.x % a.c.heads, tid = threadIdx.x;
    const int64_t at = (int64_t)blockIdx.x * a.slot_stride;
    const int64_t newest = (int64_t)a.seen[b] - a.recent;
    const int32_t n = a.c.length(b), keep = n < a.budget ? n : a.budget;
    if (h == 0 && tid == 0) a.lengths_out[b] = keep;
    const float *w = a.weights + at;
    const int32_t *pos = a.positions + at;
    float *w_out = a.weights_out + at;
    int32_t *pos_out = a.positions_out + at;
    const bool quads = (((uintptr_t)w | (uintptr_t)pos | (uintptr_t)w_out | (uintptr_t)pos_out) & 15u) == 0u;   // (16 bytes at a time)
    uint32_t rank[kSpan];
    // `copy`: and what lies below the new length goes to the outputs, places that become free included (they are filled by the moves)
    auto load = [&](int start, bool copy) {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            const int i = start + tid * kSpan + 4 * q;
            float x[4] = {};
            int32_t p[4] = {};
            if (quads && i + 4 <= n) {
                const float4 f = *reinterpret_cast<const float4 *>(w + i);
                const int4 e = *reinterpret_cast<const int4 *>(pos + i);
                x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
                p[0] = e.x, p[1] = e.y, p[2] = e.z, p[3] = e.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i + j < n) x[j] = w[i + j], p[j] = pos[i + j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) rank[4 * q + j] = p[j] < a.sinks || p[j] >= newest ? 0xFFFFFFFFu : rank_of(x[j]);
            if (copy) {
                if (quads && i + 4 <= keep) {
                    *reinterpret_cast<float4 *>(w_out + i) = make_float4(x[0], x[1], x[2], x[3]);
                    *reinterpret_cast<int4 *>(pos_out + i) = make_int4(p[0], p[1], p[2], p[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (i + j < keep) w_out[i + j] = x[j], pos_out[i + j] = p[j];
                }
            }
        }
    };
    const bool once = n <= kSpan * kThreads, copies = w != w_out || pos != pos_out;
    if (n <= a.budget) {
        if (copies)
            for (int start = 0; start < n; start += kSpan * kThreads) load(start, true);
        if (tid == 0) a.moved[blockIdx.x] = 0u;
        return;
    }
    if (once) load(0, copies);
    uint32_t prefix = 0u, wanted = (uint32_t)a.budget;   // the wanted-th largest among those that match the prefix
    for (int i = tid; i < kCopies * kRankBins; i += kThreads) (&hist[0][0])[i] = 0u;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : kRankBits;
        for (int start = 0; start < n; start += kSpan * kThreads) {
            if (!once) load(start, copies && pass == 0);
#pragma unroll
            for (int j = 0; j < kSpan; ++j)
                if (start + tid * kSpan + j < n && (pass == 0 || rank[j] >> (shift + bits) == prefix))
                    atomicAdd(&hist[tid % kCopies][(rank[j] >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // thread t holds kBinsPer bins, from the top: the bins above them are those of the threads before
        const int top = kRankBins - 1 - kBinsPer * tid;
        uint32_t bin[kBinsPer], mine = 0u, all;
#pragma unroll
        for (int i = 0; i < kBinsPer; ++i) {
            bin[i] = 0u;
#pragma unroll
            for (int c = 0; c < kCopies; ++c) bin[i] += hist[c][top - i];
            mine += bin[i];
        }
        uint32_t above = exclusive_sum<kWaves>(mine, part[pass & 1], &all);
#pragma unroll
        for (int i = 0; i < kBinsPer; ++i) {
            if (above < wanted && wanted <= above + bin[i]) {
                found[0] = (prefix << bits) | (uint32_t)(top - i);
                found[1] = wanted - above;
            }
            above += bin[i];
        }
        if (pass < 2)
            for (int i = tid; i < kCopies * kRankBins; i += kThreads) (&hist[0][0])[i] = 0u;
        __syncthreads();
        prefix = found[0];
        wanted = found[1];
    }
    // entries above `prefix` stay, and the first `wanted` of those that equal it
    int2 *moves = a.moves + blockIdx.x * a.room;
    uint32_t equal = 0u, holes = 0u, movers = 0u;
    for (int start = 0; start < n; start += kSpan * kThreads) {
        if (!once) load(start, false);
        const int first = start + tid * kSpan;
        uint32_t same = 0u, sum;
#pragma unroll
        for (int j = 0; j < kSpan; ++j) same += first + j < n && rank[j] == prefix ? 1u : 0u;
        uint32_t left = equal + exclusive_sum<kWaves>(same, part[1], &sum);   // of those equal, how many come before
        equal += sum;
        uint32_t stays = 0u, mine = 0u;   // (holes in the lower half, movers in the upper one: no more than 16384 of either)
#pragma unroll
        for (int j = 0; j < kSpan; ++j) {
            const int i = first + j;
            bool stay = i < n && rank[j] > prefix;
            if (i < n && rank[j] == prefix) stay = left++ < wanted;
            stays |= stay ? 1u << j : 0u;
            mine += (i < a.budget && !stay ? 1u : 0u) + (i >= a.budget && stay ? 0x10000u : 0u);   // (the budget is below n)
        }
        const uint32_t order = exclusive_sum<kWaves>(mine, part[0], &sum);
        uint32_t hole = holes + (order & 0xFFFFu), mover = movers + (order >> 16);
        holes += sum & 0xFFFFu;
        movers += sum >> 16;
#pragma unroll
        for (int j = 0; j < kSpan; ++j) {
            const int i = first + j;
            if ((stays >> j & 1u) != 0u) {
                if (i >= a.budget) moves[mover++].x = i;
            } else if (i < a.budget) {
                moves[hole++].y = i;
            }
        }
    }
    if (tid == 0) a.moved[blockIdx.x] = holes;
}

// Moves keys and values: 16 bytes a thread, a workgroup 256 / pieces entries at a time.  What is read lies behind the budget and
// what is written before it.
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a, int per_head, int piece_shift)
{
    const int bh = blockIdx.x / per_head, part = blockIdx.x % per_head;
    const int b = bh / a.c.heads, h = bh % a.c.heads;
    const uint32_t moved = a.moved[bh];
    const int2 *moves = a.moves + bh * a.room;
    const int64_t at = (int64_t)bh * a.slot_stride;
    const int piece = threadIdx.x & ((1 << piece_shift) - 1), per_step = 256 >> piece_shift;
    for (uint32_t m = part * per_step + (threadIdx.x >> piece_shift); m < moved; m += per_head * per_step) {
        const int2 move = moves[m];
        bool there = true;
        const int64_t from = a.c.group_offset(b, (uint32_t)move.x / kSlotGroup, h) + (int64_t)(move.x % kSlotGroup) * a.c.token_stride + piece * 16;
        const int64_t to = a.c.group_offset(b, (uint32_t)move.y / kSlotGroup, h, &there) + (int64_t)(move.y % kSlotGroup) * a.c.token_stride + piece * 16;
        if (there) {
            const uint4 x = *reinterpret_cast<const uint4 *>(a.c.k + from);
            const uint4 y = *reinterpret_cast<const uint4 *>(a.c.v + from);
            *reinterpret_cast<uint4 *>(a.c.k + to) = x;
            *reinterpret_cast<uint4 *>(a.c.v + to) = y;
        }
        if (piece == 0) {
            const float w = a.weights[at + move.x];
            const int32_t p = a.positions[at + move.x];
            a.weights_out[at + move.y] = w;
            a.positions_out[at + move.y] = p;
        }
    }
}

int log2_of(int x)
{
    int s = 0;
    while (1 << s < x) ++s;
    return s;
}

fgmp_status_t launched() { return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP; }

int64_t evict_room(int64_t slots, int64_t budget) { return std::max<int64_t>(0, std::min(budget, slots - budget)); }

// the counts, on lines of their own, then the moves
size_t evict_bytes(int64_t pairs, int64_t room) { return (size_t)(align_up((uint64_t)pairs * 4, 256) + (uint64_t)pairs * room * 8); }

}  // namespace

}  // namespace fgmp

using namespace fgmp;

extern "C" {

fgmp_status_t fgmp_cache_append(const fgmp_heads_t *k, const fgmp_heads_t *v, fgmp_dtype_t dt, int64_t tokens, const fgmp_cache_t *cache,
                                const int32_t *rows, int64_t accepted, const int32_t *counts, const int32_t *positions,
                                int32_t *slot_positions, float *slot_weights, int64_t slot_stride, int32_t *lengths_out, void *stream)
{
    AppendArgs a = {};
    fgmp_status_t rc = check_cache(cache, &a.c);
    if (rc != FGMP_OK) return rc;
    if (tokens <= 0 || accepted <= 0 || !known_dtype(dt) || lengths_out == nullptr || lengths_out == cache->lengths) return FGMP_ERR_INVALID_ARG;
    if (slot_positions != nullptr && positions == nullptr) return FGMP_ERR_INVALID_ARG;
    if (rows == nullptr && accepted > tokens) return FGMP_ERR_BAD_SHAPE;
    if ((slot_positions != nullptr || slot_weights != nullptr) && slot_stride < a.c.slots) return FGMP_ERR_BAD_SHAPE;
    const int size = dtype_size(dt);
    if ((rc = check_heads(k, a.c.batch, tokens, a.c.heads, a.c.head_dim, size, false)) != FGMP_OK) return rc;
    if ((rc = check_heads(v, a.c.batch, tokens, a.c.heads, a.c.head_dim, size, false)) != FGMP_OK) return rc;
    const int per_head = a.c.head_dim * dtype_size(cache->dtype) / 16;
    const int64_t pieces = (int64_t)a.c.heads * per_head;
    const int64_t per_token = std::max<int64_t>(1, std::min<int64_t>((pieces + 255) / 256, 64));
    if (tokens > (int64_t)1 << 30 || accepted > (int64_t)1 << 30 || !launch_counts(a.c.batch * accepted * per_token, 256)) return FGMP_ERR_UNSUPPORTED;
    a.in = {static_cast<const char *>(k->data), static_cast<const char *>(v->data), k->batch_stride * size, k->token_stride * size,
            k->head_stride * size, v->batch_stride * size, v->token_stride * size, v->head_stride * size};
    a.tokens = tokens;
    a.accepted = accepted;
    a.rows = rows;
    a.counts = counts;
    a.positions = positions;
    a.slot_positions = slot_positions;
    a.slot_weights = slot_weights;
    a.slot_stride = slot_stride;
    a.lengths_out = lengths_out;
    a.pieces = (int32_t)pieces;
    a.per_token = (int32_t)per_token;
    a.piece_shift = log2_of(per_head);
    const dim3 grid((unsigned)(a.c.batch * accepted * per_token));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool from = dt == FGMP_F32, to = cache->dtype == FGMP_F32;
    if (from && to) append_kernel<true, true><<<grid, 256, 0, st>>>(a);
    else if (from) append_kernel<true, false><<<grid, 256, 0, st>>>(a);
    else if (to) append_kernel<false, true><<<grid, 256, 0, st>>>(a);
    else append_kernel<false, false><<<grid, 256, 0, st>>>(a);
    return launched();
}

size_t fgmp_cache_evict_workspace_bytes(int64_t batch, int64_t heads, int64_t slots, int64_t budget)
{
    if (batch <= 0 || heads <= 0 || slots <= 0 || budget <= 0 || batch > 65535 || heads > 65535 || slots > (int64_t)1 << 30) return 0;
    return evict_bytes(batch * heads, evict_room(slots, budget));
}

fgmp_status_t fgmp_cache_evict(const fgmp_cache_t *cache, const float *weights, const int32_t *positions, int64_t slot_stride,
                               const int32_t *seen, int64_t budget, int64_t sinks, int64_t recent, float *weights_out,
                               int32_t *positions_out, int32_t *lengths_out, void *workspace, size_t workspace_bytes, void *stream)
{
    EvictArgs a = {};
    const fgmp_status_t rc = check_cache(cache, &a.c);
    if (rc != FGMP_OK) return rc;
    if (weights == nullptr || positions == nullptr || seen == nullptr || weights_out == nullptr || positions_out == nullptr ||
        lengths_out == nullptr || lengths_out == cache->lengths || workspace == nullptr || budget < 1 || sinks < 0 || recent < 0)
        return FGMP_ERR_INVALID_ARG;
    if (slot_stride < a.c.slots) return FGMP_ERR_BAD_SHAPE;
    if (!aligned16(workspace)) return FGMP_ERR_BAD_ALIGN;
    const int64_t pairs = (int64_t)a.c.batch * a.c.heads;
    a.room = evict_room(a.c.slots, budget);
    if (workspace_bytes < evict_bytes(pairs, a.room)) return FGMP_ERR_BUFFER_TOO_SMALL;
    a.weights = weights;
    a.positions = positions;
    a.seen = seen;
    a.weights_out = weights_out;
    a.positions_out = positions_out;
    a.lengths_out = lengths_out;
    a.slot_stride = slot_stride;
    a.budget = (int32_t)std::min<int64_t>(budget, a.c.slots);   // (no sequence holds more)
    a.sinks = (int32_t)std::min<int64_t>(sinks, INT32_MAX);
    a.recent = (int32_t)std::min<int64_t>(recent, INT32_MAX);
    a.moved = static_cast<uint32_t *>(workspace);
    a.moves = reinterpret_cast<int2 *>(static_cast<char *>(workspace) + align_up((uint64_t)pairs * 4, 256));
    const int piece_shift = log2_of(a.c.head_dim * dtype_size(cache->dtype) / 16);
    const int64_t steps = (a.room + (256 >> piece_shift) - 1) / (256 >> piece_shift);
    const int64_t per_head = std::max<int64_t>(1, std::min<int64_t>(steps, std::max<int64_t>(1, 4096 / pairs)));
    if (!launch_counts(pairs, a.c.slots <= 2048 ? 512 : 1024) || !launch_counts(pairs * per_head, 256)) return FGMP_ERR_UNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.c.slots <= 2048) evict_select_kernel<512, 1><<<dim3((unsigned)pairs), 512, 0, st>>>(a);
    else if (a.c.slots <= 8192) evict_select_kernel<1024, 2><<<dim3((unsigned)pairs), 1024, 0, st>>>(a);
    else evict_select_kernel<1024, 4><<<dim3((unsigned)pairs), 1024, 0, st>>>(a);
    // (the moves are read from the workspace: not without the launch that writes them)
    if (launched() != FGMP_OK) return FGMP_ERR_HIP;
    if (a.room > 0) evict_move_kernel<<<dim3((unsigned)(pairs * per_head)), 256, 0, st>>>(a, (int)per_head, piece_shift);
    return launched();
}

}  // extern "C"
