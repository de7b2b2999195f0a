// A cache of keys and values in 8 bits: written as it is quantized, and read back.
//
// A vector of a slot and head is E4M3 codes and one power of two 2^e, the smallest (e >= -100) that brings all of its elements within 448.  A
// power of two loses nothing against a scale of its own making: the format's steps are relative to an element, not to the vector, and x 2^-e
// and code 2^e are exact, the latter in BF16 too.  Both calls are bounded by memory; kLanes lanes have a vector, eight elements each (16387 tokens of 32 heads of 128,
// FP32, appended in 114 us, 5.9 TB/s; 4 sequences of up to 16381 slots of 32 heads read back as BF16 in 257 us, 5.1 TB/s, two thirds of it written).
#include <algorithm>

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

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
constexpr int kThreads = 256;

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
};

// The largest magnitude of those that are finite, over a vector's lanes.
template <int kLanes>
__device__ __forceinline__ uint32_t most_bits(f32x8 x)
{
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = f2u(x[i]) & 0x7FFFFFFFu;
        most = std::max(most, bits < 0x7F800000u ? bits : 0u);
    }
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) most = std::max(most, (uint32_t)__shfl_xor((int)most, d));
    return most;
}

// Eight codes; NaN for what is not finite.
__device__ __forceinline__ uint2 codes_of(f32x8 x, float inverse)
{
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; i += 2) w[i / 4] |= e4m3_encode_pair_hw(x[i] * inverse, x[i + 1] * inverse) << (8 * (i & 2));
    bool fine = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) fine = fine && fabsf(x[i]) < INFINITY;
    if (!fine) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(x[i]) < INFINITY)) w[i / 4] |= 0x7Fu << (8 * (i & 3));
    }
    return make_uint2(w[0], w[1]);
}

template <bool kF32, int kLanes>
__global__ void __launch_bounds__(kThreads) quant_append_kernel(QuantAppendArgs a)
{
    constexpr int kVectors = kThreads / kLanes;
    const CacheView &c = a.q.c;
    const int64_t token = blockIdx.x / a.per_token;
    const int part = (int)(blockIdx.x % a.per_token);
    const int b = (int)(token / a.accepted), i = (int)(token % a.accepted);
    const int32_t n = c.length(b);
    int32_t count = a.counts != nullptr ? a.counts[b] : (int32_t)a.accepted;
    count = count < 0 ? 0 : count > a.accepted ? (int32_t)a.accepted : count;
    if (i == 0 && part == 0 && threadIdx.x == 0) {
        const int64_t left = (int64_t)n + count;
        a.lengths_out[b] = left > c.slots ? c.slots : (int32_t)left;
    }
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
        const char *from = in.data + b * in.batch + row * in.token + h * in.head;
        f32x8 x;
        if constexpr (kF32) x = *reinterpret_cast<const f32x8 *>(__builtin_assume_aligned(from + 32 * lane, 16));
        else x = __builtin_convertvector(*reinterpret_cast<const bf16x8 *>(from + 16 * lane), f32x8);
        // 448 = 1.75 * 2^8: a magnitude of up to 1.75 * 2^p takes e = p - 8, a larger one e = p - 7
        const int e = std::max(-100, (int)((most_bits<kLanes>(x) + 0x1FFFFFu) >> 23) - 135);
        const uint2 codes = codes_of(x, u2f((uint32_t)(127 - e) << 23));
        char *to = (which == 0 ? c.k : c.v) + c.offset(page, in_page, h);
        *reinterpret_cast<uint2 *>(to + 8 * lane) = codes;
        if (lane == 0) (which == 0 ? a.q.k_scales : a.q.v_scales)[a.q.scale_at(page, in_page, h)] = (uint8_t)(e + 127);
    }
}

struct QuantReadArgs {
    QuantCacheView q;
    HeadsAt out[2];
    int32_t first, tokens;
    uint32_t groups;       // slot groups from that of `first` on
    uint32_t head_parts;   // workgroups that share a group's heads
};

template <bool kF32, int kLanes>
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
    if ((int32_t)(u * kSlotGroup) >= end) return;
    uint32_t in_page;
    uint32_t page = c.page_of(b, c.entry_of(u, &in_page));
    page = page < c.pages ? page : 0u;
    const int lane = threadIdx.x % kLanes;
    // the vectors of a group: 16 slots, of each its heads, keys and values
    for (int at = part * kVectors + (int)threadIdx.x / kLanes; at < kSlotGroup * 2 * c.heads; at += (int)a.head_parts * kVectors) {
        const int h2 = at % (2 * c.heads), which = h2 >= c.heads ? 1 : 0, h = h2 - which * c.heads;
        const int r = at / (2 * c.heads), slot = (int)(u * kSlotGroup) + r;
        if (slot < a.first || slot >= end) continue;
        const uint2 codes = *reinterpret_cast<const uint2 *>((which == 0 ? c.k : c.v) + c.offset(page, in_page + r, h) + 8 * lane);
        const float scale = u2f((uint32_t)(which == 0 ? a.q.k_scales : a.q.v_scales)[a.q.scale_at(page, in_page + r, h)] << 23);
        f32x8 x;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float2_t p = e4m3_decode_pair_hw((i < 4 ? codes.x : codes.y) >> (8 * (i & 2)) & 0xFFFFu);
            x[i] = p[0] * scale, x[i + 1] = p[1] * scale;
        }
        const HeadsAt &out = a.out[which];
        char *to = out.data + b * out.batch + (int64_t)(slot - a.first) * out.token + h * out.head;
        if constexpr (kF32) {
            *reinterpret_cast<f32x4 *>(to + 32 * lane) = f32x4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f32x4 *>(to + 32 * lane + 16) = f32x4{x[4], x[5], x[6], x[7]};
        } else {
            *reinterpret_cast<bf16x8 *>(to + 16 * lane) = __builtin_convertvector(x, bf16x8);   // (exact)
        }
    }
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
    const int vectors = kThreads * 8 / c.head_dim;
    a.per_token = (uint32_t)((2 * c.heads + vectors - 1) / vectors);
    if (!launch_counts((int64_t)c.batch * accepted * a.per_token, kThreads)) return FGMP_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(c.batch * accepted * a.per_token));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32) {
        if (c.head_dim == 64) quant_append_kernel<true, 8><<<grid, kThreads, 0, st>>>(a);
        else if (c.head_dim == 128) quant_append_kernel<true, 16><<<grid, kThreads, 0, st>>>(a);
        else quant_append_kernel<true, 32><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (c.head_dim == 64) quant_append_kernel<false, 8><<<grid, kThreads, 0, st>>>(a);
        else if (c.head_dim == 128) quant_append_kernel<false, 16><<<grid, kThreads, 0, st>>>(a);
        else quant_append_kernel<false, 32><<<grid, kThreads, 0, st>>>(a);
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
    const dim3 grid((unsigned)(all * a.head_parts));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32) {
        if (c.head_dim == 64) quant_read_kernel<true, 8><<<grid, kThreads, 0, st>>>(a);
        else if (c.head_dim == 128) quant_read_kernel<true, 16><<<grid, kThreads, 0, st>>>(a);
        else quant_read_kernel<true, 32><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (c.head_dim == 64) quant_read_kernel<false, 8><<<grid, kThreads, 0, st>>>(a);
        else if (c.head_dim == 128) quant_read_kernel<false, 16><<<grid, kThreads, 0, st>>>(a);
        else quant_read_kernel<false, 32><<<grid, kThreads, 0, st>>>(a);
    }
    return launched();
}

}  // extern "C"
