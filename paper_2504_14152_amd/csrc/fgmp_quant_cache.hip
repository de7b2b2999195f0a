// A cache of keys and values in 8 bits: written as it is quantized, and read back.
//
// A vector of a slot and head is E4M3 codes and one power of two 2^e, the smallest (e >= -100) that brings all of its elements within 448.  A
// power of two loses nothing against a scale of its own making: the format's steps are relative to an element, not to the vector, and x 2^-e
// and code 2^e are exact, the latter in BF16 too.  Both calls are bounded by memory, as long as a vector, eight elements to each of kLanes lanes, takes few
// instructions (the card's own conversions, with their scales) and enough vectors are under way: 16387 tokens of 32 heads of 128, FP32, are appended in 114 us,
// 5.9 TB/s; 32768 of 8 heads, BF16, in 44 us, 4.5 TB/s (65536 in 83, 4.9 TB/s); 4 sequences of up to 16381 slots of 32 heads are read back as BF16 in 254 us, 5.1 TB/s, two thirds of it written.
#include <algorithm>
#include <type_traits>

#include "fgmp_quant_cache.hpp"

namespace fgmp {

fgmp_status_t check_quant_cache(const fgmp_quant_cache_t *c, QuantCacheView *view)
{
    if (c == nullptr || c->k_scales == nullptr || c->v_scales == nullptr || c->codes.dtype != FGMP_E4M3) return FGMP_ERR_INVALID_ARG;
    const fgmp_status_t rc = check_cache_of(&c->codes, 1, &view->c);
    if (rc != FGMP_OK) return rc;
    const int64_t page_stride = c->codes.pages > 1 ? c->scale_page_stride : c->codes.page_size, head_stride = c->codes.heads > 1 ? c->scale_head_stride : c->codes.page_size;
    if (c->codes.page_size % kSlotGroup != 0 || page_stride < c->codes.page_size || head_stride < c->codes.page_size) return FGMP_ERR_BAD_SHAPE;
    if (!aligned16(c->k_scales) || !aligned16(c->v_scales) || page_stride % 16 != 0 || head_stride % 16 != 0) return FGMP_ERR_BAD_ALIGN;
    if (page_stride > (int64_t)1 << 40 || head_stride > (int64_t)1 << 40) return FGMP_ERR_UNSUPPORTED;
    view->k_scales = c->k_scales;
    view->v_scales = c->v_scales;
    view->scale_page = page_stride;
    view->scale_head = head_stride;
    return FGMP_OK;
}

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
constexpr int kThreads = 256;
// Appended tokens go several to a workgroup where that leaves as many workgroups, but for FP32 whose tokens fill one by themselves: 32768 tokens of 8 heads of 128, BF16,
// 54 -> 44 us, FP32 63 -> 67; 262144 of one head, BF16, 213 -> 45 (FP32 67).  Below, a call is mostly its launch either way.
constexpr int64_t kManyWorkgroups = 256;

struct HeadsAt {
    char *data;
    int64_t batch, token, head;   // bytes
};

struct QuantAppendArgs {
    QuantCacheView q;
    HeadsAt in[2];
    int64_t tokens, accepted;
    const int32_t *rows, *counts;
    int32_t *lengths_out;
    uint32_t per_token;    // workgroups that share a token
    uint32_t take, chunks; // else: tokens of a workgroup, and workgroups of a sequence
    uint32_t by_vectors;   // 2^16 / (2 heads), rounded up
};

// The largest over a vector's lanes, the same in all of them: neighbours, pairs, quads, eights change places within rows of 16 lanes, then rows.
template <int kLanes>
__device__ __forceinline__ uint32_t most_of_lanes(uint32_t most)
{
    auto step = [&](auto control) { most = std::max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, decltype(control)::value, 0xF, 0xF, true)); };
    step(std::integral_constant<int, 0xB1>());                                // lane ^ 1
    step(std::integral_constant<int, 0x4E>());                                // lane ^ 2
    step(std::integral_constant<int, 0x141>());                               // 7 - lane of eight
    if constexpr (kLanes >= 16) step(std::integral_constant<int, 0x140>());   // 15 - lane of a row
    if constexpr (kLanes >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(most, most, false, false);
        most = std::max((uint32_t)r[0], (uint32_t)r[1]);
    }
    return most;
}

// Eight elements of a vector, and what they become.
template <bool kF32>
struct Eight {
    u32x4 w[kF32 ? 2 : 1];
    __device__ __forceinline__ void load(const char *vector, int lane)
    {
#pragma unroll
        for (int i = 0; i < (kF32 ? 2 : 1); ++i) w[i] = *reinterpret_cast<const u32x4 *>(vector + (kF32 ? 32 : 16) * lane + 16 * i);
    }
    __device__ __forceinline__ float value(int i) const
    {
        if constexpr (kF32) return u2f(w[i / 4][i % 4]);
        else return u2f(i % 2 != 0 ? w[0][i / 2] & 0xFFFF0000u : w[0][i / 2] << 16);
    }
    // The bits of the largest magnitude; those of a NaN or infinity where there is one.
    __device__ __forceinline__ uint32_t most() const
    {
        if constexpr (kF32) {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = __builtin_elementwise_maximum(m, fabsf(value(i)));
            return f2u(m) & 0x7FFFFFFFu;
        } else {
            u16x2 m = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[0][i] & 0x7FFF7FFFu));
            return (uint32_t)std::max(m[0], m[1]) << 16;
        }
    }
    __device__ __forceinline__ uint2 codes(float scale) const
    {
        uint32_t c[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 x = {0, 0};
            if constexpr (kF32) {
                x = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x, value(4 * i), value(4 * i + 1), scale, false);
                x = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(x, value(4 * i + 2), value(4 * i + 3), scale, true);
            } else {
                const uint32_t low = w[0][2 * i], high = w[0][2 * i + 1];   // (cast in place, all would be the vector's first element)
                x = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(x, __builtin_bit_cast(bf16x2, low), scale, false);
                x = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(x, __builtin_bit_cast(bf16x2, high), scale, true);
            }
            c[i] = __builtin_bit_cast(uint32_t, x);
        }
        return make_uint2(c[0], c[1]);
    }
};

// e + 127.  448 = 1.75 * 2^8: a magnitude of up to 1.75 * 2^p takes e = p - 8, a larger one e = p - 7; -100 at least
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) { return std::max(35u, (most + 0x1FFFFFu) >> 23) - 8u; }

// A vector's codes and scale byte, for all of its lanes.
template <bool kF32, int kLanes>
__device__ __forceinline__ uint2 quantized(const Eight<kF32> &x, uint32_t *byte)
{
    uint32_t most = most_of_lanes<kLanes>(x.most());
    if (most < 0x7F800000u) {
        *byte = scale_byte(most);
        return x.codes(u2f(*byte << 23));
    }
    // (something is not finite: the largest of the others, and NaN in its places)
    most = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = f2u(x.value(i)) & 0x7FFFFFFFu;
        most = std::max(most, bits < 0x7F800000u ? bits : 0u);
    }
    *byte = scale_byte(most_of_lanes<kLanes>(most));
    const uint2 codes = x.codes(u2f(*byte << 23));
    uint32_t w[2] = {codes.x, codes.y};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(fabsf(x.value(i)) < INFINITY)) w[i / 4] |= 0x7Fu << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}

// How many tokens of a sequence are stored.
__device__ __forceinline__ int32_t stored(const QuantAppendArgs &a, int b)
{
    const int32_t count = a.counts != nullptr ? a.counts[b] : (int32_t)a.accepted;
    return count < 0 ? 0 : count > a.accepted ? (int32_t)a.accepted : count;
}
__device__ __forceinline__ void store_length(const QuantAppendArgs &a, int b, int32_t n, int32_t count)
{
    const int64_t left = (int64_t)n + count;
    a.lengths_out[b] = left > a.q.c.slots ? a.q.c.slots : (int32_t)left;
}

// A token to a workgroup, or to several.
template <bool kF32, int kLanes>
__global__ void __launch_bounds__(kThreads) quant_append_kernel(QuantAppendArgs a)
{
    constexpr int kVectors = kThreads / kLanes;
    const CacheView &c = a.q.c;
    const int64_t token = blockIdx.x / a.per_token;
    const int part = (int)(blockIdx.x % a.per_token);
    const int b = (int)(token / a.accepted), i = (int)(token % a.accepted);
    const int32_t n = c.length(b), count = stored(a, b);
    if (i == 0 && part == 0 && threadIdx.x == 0) store_length(a, b, n, count);
    if (i >= count || n + i >= c.slots) return;
    const int32_t row = a.rows != nullptr ? a.rows[b * a.accepted + i] : i;
    if ((uint32_t)row >= (uint32_t)a.tokens) return;
    const int32_t slot = n + i;
    uint32_t in_page;
    const uint32_t page = c.page_of(b, c.entry_of((uint32_t)slot / kSlotGroup, &in_page));
    if (page >= c.pages) return;
    in_page += (uint32_t)slot % kSlotGroup;
    const int lane = threadIdx.x % kLanes;
    // (a wave has keys or values of its vectors, not both)
    for (int at = part * kVectors + (int)threadIdx.x / kLanes; at < 2 * c.heads; at += (int)a.per_token * kVectors) {
        const int which = at >= c.heads ? 1 : 0, h = at - which * c.heads;
        const HeadsAt &in = a.in[which];
        Eight<kF32> x;
        x.load(in.data + b * in.batch + row * in.token + h * in.head, lane);
        uint32_t byte;
        const uint2 codes = quantized<kF32, kLanes>(x, &byte);
        char *to = (which == 0 ? c.k : c.v) + c.offset(page, in_page, h);
        *reinterpret_cast<uint2 *>(to + 8 * lane) = codes;
        if (lane == 0) (which == 0 ? a.q.k_scales : a.q.v_scales)[a.q.scale_at(page, in_page, h)] = (uint8_t)byte;
    }
}

// Several tokens to a workgroup, whose places are found by a thread each: all that lies in front of a vector's load is waited for once, and kAtATime vectors
// of a lane are asked for together.
constexpr int kMostTaken = 64, kAtATime = 4;
template <bool kF32, int kLanes>
__global__ void __launch_bounds__(kThreads) quant_append_many_kernel(QuantAppendArgs a)
{
    constexpr int kVectors = kThreads / kLanes;
    struct Place {
        int64_t from[2], to, scale;
    };
    __shared__ Place places[kMostTaken];
    __shared__ bool there[kMostTaken];
    const CacheView &c = a.q.c;
    const int b = (int)(blockIdx.x / a.chunks);
    const int64_t first = (int64_t)(blockIdx.x % a.chunks) * a.take;
    const int32_t n = c.length(b), count = stored(a, b);
    if (first == 0 && threadIdx.x == 0) store_length(a, b, n, count);
    const int tokens = (int)std::min<int64_t>(a.take, std::min<int64_t>(count, c.slots - n) - first);
    if (tokens <= 0) return;
    if ((int)threadIdx.x < tokens) {
        const int32_t i = (int32_t)first + (int)threadIdx.x, slot = n + i, row = a.rows != nullptr ? a.rows[b * a.accepted + i] : i;
        uint32_t in_page;
        const uint32_t page = c.page_of(b, c.entry_of((uint32_t)slot / kSlotGroup, &in_page));
        in_page += (uint32_t)slot % kSlotGroup;
        const bool fine = (uint32_t)row < (uint32_t)a.tokens && page < c.pages;
        there[threadIdx.x] = fine;
        const int64_t from = fine ? row : 0;   // (one that is none is read all the same)
        places[threadIdx.x] = {{from * a.in[0].token, from * a.in[1].token}, c.offset(page, in_page, 0), a.q.scale_at(fine ? page : 0u, in_page, 0)};
    }
    __syncthreads();
    const int lane = threadIdx.x % kLanes, vectors = tokens * 2 * c.heads;
    for (int base = (int)threadIdx.x / kLanes; base < vectors; base += kAtATime * kVectors) {
        Eight<kF32> x[kAtATime];
        int token[kAtATime], at[kAtATime];
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) {
            const int f = std::min(base + j * kVectors, vectors - 1);
            token[j] = (int)((uint32_t)f * a.by_vectors >> 16);
            at[j] = f - token[j] * 2 * c.heads;
            const int which = at[j] >= c.heads ? 1 : 0, h = at[j] - which * c.heads;
            const char *const from = which == 0 ? a.in[0].data + b * a.in[0].batch + h * a.in[0].head : a.in[1].data + b * a.in[1].batch + h * a.in[1].head;
            x[j].load(from + places[token[j]].from[which], lane);
        }
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) {
            uint32_t byte;
            const uint2 codes = quantized<kF32, kLanes>(x[j], &byte);
            if (base + j * kVectors >= vectors || !there[token[j]]) continue;
            const int which = at[j] >= c.heads ? 1 : 0, h = at[j] - which * c.heads;
            char *const to = (which == 0 ? c.k : c.v) + places[token[j]].to + (int64_t)h * c.head_stride;
            *reinterpret_cast<uint2 *>(to + 8 * lane) = codes;
            if (lane == 0) (which == 0 ? a.q.k_scales : a.q.v_scales)[places[token[j]].scale + h * a.q.scale_head] = (uint8_t)byte;
        }
    }
}

template <bool kF32, int kLanes>
void append_launch(const QuantAppendArgs &a, dim3 grid, hipStream_t st)
{
    if (a.take > 1u) quant_append_many_kernel<kF32, kLanes><<<grid, kThreads, 0, st>>>(a);
    else quant_append_kernel<kF32, kLanes><<<grid, kThreads, 0, st>>>(a);
}

struct QuantReadArgs {
    QuantCacheView q;
    HeadsAt out[2];
    int32_t first, tokens;
    uint32_t groups;       // slot groups from that of `first` on
    uint32_t head_parts;   // workgroups that share a group's heads
    int32_t step_slots, step_heads;   // from a lane's vector to its next one: slots, and of keys' and values' heads
};

// The values of eight codes: consecutive ones of lane `lane`, or, of 32 bits each, two runs of four, so that the lanes' stores lie next to each other (64 MB of codes: 97 -> 71 us).
template <bool kF32, int kLanes>
__device__ __forceinline__ uint2 load_codes(const char *vector, int lane)
{
    if constexpr (!kF32) return *reinterpret_cast<const uint2 *>(vector + 8 * lane);
    else return make_uint2(*reinterpret_cast<const uint32_t *>(vector + 4 * lane), *reinterpret_cast<const uint32_t *>(vector + 4 * kLanes + 4 * lane));
}
template <bool kF32, int kLanes>
__device__ __forceinline__ void store_values(char *to, int lane, uint2 codes, float scale)
{
    const uint32_t w[2] = {codes.x, codes.y};
    if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto low = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, false), high = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], scale, true);
            *reinterpret_cast<f32x4 *>(to + 16 * kLanes * i + 16 * lane) = f32x4{low[0], low[1], high[0], high[1]};
        }
    } else {
        u32x4 x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // (exact)
            x[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false));
            x[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true));
        }
        *reinterpret_cast<u32x4 *>(to + 16 * lane) = x;
    }
}

// kTogether: vectors of a lane that are asked for together.
template <bool kF32, int kLanes, int kTogether>
__global__ void __launch_bounds__(kThreads) quant_read_kernel(QuantReadArgs a)
{
    constexpr int kVectors = kThreads / kLanes;
    const CacheView &c = a.q.c;
    uint32_t id = blockIdx.x;
    const int part = (int)(id % a.head_parts);
    id /= a.head_parts;
    const uint32_t u = (uint32_t)a.first / kSlotGroup + id % a.groups;
    const int b = (int)(id / a.groups);
    const int32_t end = std::min((int64_t)c.length(b), (int64_t)a.first + a.tokens);
    const int32_t slot = (int32_t)(u * kSlotGroup);
    if (slot >= end) return;
    uint32_t in_page;
    uint32_t page = c.page_of(b, c.entry_of(u, &in_page));
    page = page < c.pages ? page : 0u;
    const int64_t codes_at = c.offset(page, in_page, 0), scales_at = a.q.scale_at(page, in_page, 0);
    const int lane = threadIdx.x % kLanes, both = 2 * c.heads;
    // The vectors of a group: 16 slots, of each its heads, keys and values.  Of slots that are not asked for or not in use they are loaded all the same (the
    // group is there): with loads left out, each would be waited for by itself.
    int h2 = part * kVectors + (int)threadIdx.x / kLanes, r = h2 / both;
    h2 -= r * both;
    while (r < kSlotGroup) {
        uint2 codes[kTogether];
        uint32_t scale[kTogether];
        char *to[kTogether];
#pragma unroll
        for (int j = 0; j < kTogether; ++j) {
            const int here = std::min(r, kSlotGroup - 1), which = h2 >= c.heads ? 1 : 0, h = h2 - which * c.heads;
            codes[j] = load_codes<kF32, kLanes>((which == 0 ? c.k : c.v) + codes_at + here * c.token_stride + h * c.head_stride, lane);
            scale[j] = (which == 0 ? a.q.k_scales : a.q.v_scales)[scales_at + h * a.q.scale_head + here];
            const HeadsAt &out = a.out[which];
            to[j] = r < kSlotGroup && slot + r >= a.first && slot + r < end ? out.data + b * out.batch + (int64_t)(slot + r - a.first) * out.token + h * out.head : nullptr;
            r += a.step_slots, h2 += a.step_heads;
            if (h2 >= both) h2 -= both, ++r;
        }
#pragma unroll
        for (int j = 0; j < kTogether; ++j)
            if (to[j] != nullptr) store_values<kF32, kLanes>(to[j], lane, codes[j], u2f(scale[j] << 23));
    }
}

template <bool kF32, int kLanes>
void read_launch(const QuantReadArgs &a, bool many, dim3 grid, hipStream_t st)
{
    if (many) quant_read_kernel<kF32, kLanes, kAtATime><<<grid, kThreads, 0, st>>>(a);
    else quant_read_kernel<kF32, kLanes, 1><<<grid, kThreads, 0, st>>>(a);
}

HeadsAt at_of(const fgmp_heads_t *x, int size)
{
    return {static_cast<char *>(x->data), x->batch_stride * size, x->token_stride * size, x->head_stride * size};
}

fgmp_status_t launched() { return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP; }

}  // namespace

}  // namespace fgmp

using namespace fgmp;

extern "C" {

fgmp_status_t fgmp_quant_cache_append(const fgmp_heads_t *k, const fgmp_heads_t *v, fgmp_dtype_t dt, int64_t tokens, const fgmp_quant_cache_t *cache,
                                      const int32_t *rows, int64_t accepted, const int32_t *counts, int32_t *lengths_out, void *stream)
{
    QuantAppendArgs a = {};
    fgmp_status_t rc = check_quant_cache(cache, &a.q);
    if (rc != FGMP_OK) return rc;
    const CacheView &c = a.q.c;
    if (!known_dtype(dt) || tokens <= 0 || accepted <= 0 || lengths_out == nullptr || lengths_out == c.lengths) return FGMP_ERR_INVALID_ARG;
    if (rows == nullptr && accepted > tokens) return FGMP_ERR_BAD_SHAPE;
    if (tokens > INT32_MAX || accepted > INT32_MAX) return FGMP_ERR_UNSUPPORTED;
    const int size = dtype_size(dt);
    if ((rc = check_heads(k, c.batch, tokens, c.heads, c.head_dim, size, false)) != FGMP_OK) return rc;
    if ((rc = check_heads(v, c.batch, tokens, c.heads, c.head_dim, size, false)) != FGMP_OK) return rc;
    a.in[0] = at_of(k, size), a.in[1] = at_of(v, size);
    a.tokens = tokens;
    a.accepted = accepted;
    a.rows = rows;
    a.counts = counts;
    a.lengths_out = lengths_out;
    const int vectors = kThreads * 8 / c.head_dim, of_token = 2 * c.heads;
    a.per_token = (uint32_t)((of_token + vectors - 1) / vectors);
    a.take = (uint32_t)std::min((kAtATime * vectors + of_token - 1) / of_token, kMostTaken);
    a.chunks = (uint32_t)((accepted + a.take - 1) / a.take);
    if (c.batch * (int64_t)a.chunks < kManyWorkgroups || (dt == FGMP_F32 && of_token >= vectors)) a.take = 1u;
    a.by_vectors = (65536u + of_token - 1) / of_token;
    const int64_t workgroups = a.take > 1u ? c.batch * (int64_t)a.chunks : (int64_t)c.batch * accepted * a.per_token;
    if (!launch_counts(workgroups, kThreads)) return FGMP_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)workgroups);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32) {
        if (c.head_dim == 64) append_launch<true, 8>(a, grid, st);
        else if (c.head_dim == 128) append_launch<true, 16>(a, grid, st);
        else append_launch<true, 32>(a, grid, st);
    } else {
        if (c.head_dim == 64) append_launch<false, 8>(a, grid, st);
        else if (c.head_dim == 128) append_launch<false, 16>(a, grid, st);
        else append_launch<false, 32>(a, grid, st);
    }
    return launched();
}

fgmp_status_t fgmp_quant_cache_read(const fgmp_quant_cache_t *cache, int64_t first, int64_t tokens, const fgmp_heads_t *k_out, const fgmp_heads_t *v_out,
                                    fgmp_dtype_t dt, void *stream)
{
    QuantReadArgs a = {};
    fgmp_status_t rc = check_quant_cache(cache, &a.q);
    if (rc != FGMP_OK) return rc;
    const CacheView &c = a.q.c;
    if (!known_dtype(dt) || first < 0 || tokens <= 0) return FGMP_ERR_INVALID_ARG;
    if (tokens > c.slots || first > c.slots - tokens) return FGMP_ERR_BAD_SHAPE;
    const int size = dtype_size(dt);
    if ((rc = check_heads(k_out, c.batch, tokens, c.heads, c.head_dim, size, true)) != FGMP_OK) return rc;
    if ((rc = check_heads(v_out, c.batch, tokens, c.heads, c.head_dim, size, true)) != FGMP_OK) return rc;
    a.out[0] = at_of(k_out, size), a.out[1] = at_of(v_out, size);
    a.first = (int32_t)first;
    a.tokens = (int32_t)tokens;
    a.groups = (uint32_t)((first + tokens - 1) / kSlotGroup - first / kSlotGroup + 1);
    const int64_t vectors = kThreads * 8 / c.head_dim, turns = (kSlotGroup * 2 * (int64_t)c.heads + vectors - 1) / vectors;
    const int64_t all = (int64_t)c.batch * a.groups;
    a.head_parts = (uint32_t)std::min<int64_t>(turns, std::max<int64_t>((turns + 7) / 8, 2048 / all));
    if (!launch_counts(all * a.head_parts, kThreads)) return FGMP_ERR_UNSUPPORTED;
    a.step_slots = (int32_t)(vectors * a.head_parts / (2 * c.heads));
    a.step_heads = (int32_t)(vectors * a.head_parts % (2 * c.heads));
    const dim3 grid((unsigned)(all * a.head_parts));
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool many = a.head_parts < turns;
    if (dt == FGMP_F32) {
        if (c.head_dim == 64) read_launch<true, 8>(a, many, grid, st);
        else if (c.head_dim == 128) read_launch<true, 16>(a, many, grid, st);
        else read_launch<true, 32>(a, many, grid, st);
    } else {
        if (c.head_dim == 64) read_launch<false, 8>(a, many, grid, st);
        else if (c.head_dim == 128) read_launch<false, 16>(a, many, grid, st);
        else read_launch<false, 32>(a, many, grid, st);
    }
    return launched();
}

}  // extern "C"
