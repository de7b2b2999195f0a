// Queries, keys and values as a product leaves them, made ready for attention in one pass: queries and keys normed for each head and rotated by
// their positions, values converted.
//   u = w (x - mean) / sqrt(mean((x - mean)^2) + eps);   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * inv_freq
// Memory bounds it: every element is read and written once (16384 tokens of 80 heads of 128, FP32 to BF16: 192 us, 5.2 TB/s).  kLanes lanes have a vector of a
// head, each two runs of four elements, which are the two halves of four pairs: a rotation stays in a lane, and a norm's sums take log2(kLanes) steps
// between lanes.  A workgroup has kTokens tokens and goes over the heads; the tokens' sines and cosines are found once, by one thread for each pair, and go
// through LDS.  With one token the loop is bound by its own instructions, the places, weights and sines of eight elements a lane: two share the first two
// (the 16384 tokens with 1 / 2 / 4 / 8: 214 / 192 / 197 / 200 us).
#include <algorithm>
#include <type_traits>

#include "fgmp_cache.hpp"

namespace fgmp {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kMaxDim = 512;
// Tokens of a workgroup where there are enough of them to fill the chip; fewer have a workgroup each, or several that share their heads.
constexpr int kTokensOfMany = 2;
constexpr int64_t kMany = 1024;

struct RotatePart {
    const char *from;
    char *to;
    int64_t from_batch, from_token, from_head, to_batch, to_token, to_head;   // bytes
    const float *weight;
};

struct RotateArgs {
    RotatePart part[3];        // queries, keys, values
    int32_t ends[3];           // heads up to the end of each
    int32_t tokens, dim, pairs, axes, interleaved, layer;
    uint32_t per_chunk;        // workgroups that share the heads of some tokens
    float eps, inverse_dim;
    const int32_t *positions, *axis_of;
    const float *inv_freq;
};

// The angle is exact to 2^-53 of itself; it is brought to a quarter of a turn around a multiple of one in 64 bits (pi/2 in two parts), where the sums of
// the power series, to x^9 and x^10, leave out less than 2^-29 and 2^-33.
__device__ __forceinline__ float2 turn(int32_t position, float inv_freq)
{
    const double angle = (double)position * (double)inv_freq;
    const double quarters = __builtin_rint(angle * 0.63661977236758134308);
    const double left = __builtin_fma(-quarters, 6.123233995736766036e-17, __builtin_fma(-quarters, 1.5707963267948965580, angle));
    const int quadrant = (int)(quarters - 4.0 * __builtin_rint(quarters * 0.25)) & 3;
    const float x = (float)left, x2 = x * x;
    float s = 1.0f / 362880.0f;
    s = __builtin_fmaf(s, x2, -1.0f / 5040.0f);
    s = __builtin_fmaf(s, x2, 1.0f / 120.0f);
    s = __builtin_fmaf(s, x2, -1.0f / 6.0f);
    s = __builtin_fmaf(s * x2, x, x);
    float c = -1.0f / 3628800.0f;
    c = __builtin_fmaf(c, x2, 1.0f / 40320.0f);
    c = __builtin_fmaf(c, x2, -1.0f / 720.0f);
    c = __builtin_fmaf(c, x2, 1.0f / 24.0f);
    c = __builtin_fmaf(c, x2, -0.5f);
    c = __builtin_fmaf(c, x2, 1.0f);
    const float cs = (quadrant & 1) != 0 ? s : c, sn = (quadrant & 1) != 0 ? c : s;
    return make_float2(quadrant == 1 || quadrant == 2 ? -cs : cs, quadrant >= 2 ? -sn : sn);
}

template <bool kF32>
__device__ __forceinline__ f32x4 load4(const char *at, int e)
{
    if constexpr (kF32) return *reinterpret_cast<const f32x4 *>(at + 4 * e);
    else return __builtin_convertvector(*reinterpret_cast<const bf16x4 *>(at + 2 * e), f32x4);
}

template <bool kF32>
__device__ __forceinline__ void store4(char *at, int e, f32x4 x)
{
    if constexpr (kF32) *reinterpret_cast<f32x4 *>(at + 4 * e) = x;
    else *reinterpret_cast<bf16x4 *>(at + 2 * e) = __builtin_convertvector(x, bf16x4);   // (nearest even)
}

// Sum over a vector's lanes, the same in all of them: neighbours, pairs, quads, eights change places within rows of 16 lanes, then rows and halves.
template <int kLanes>
__device__ __forceinline__ float head_sum(f32x4 x, f32x4 y)
{
    float v = ((x[0] + x[1]) + (x[2] + x[3])) + ((y[0] + y[1]) + (y[2] + y[3]));
    auto add = [&](auto control) {
        v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xF, 0xF, true));
    };
    add(std::integral_constant<int, 0xB1>());                           // lane ^ 1
    add(std::integral_constant<int, 0x4E>());                           // lane ^ 2
    add(std::integral_constant<int, 0x141>());                          // 7 - lane of eight
    if constexpr (kLanes >= 16) add(std::integral_constant<int, 0x140>());   // 15 - lane of a row
    if constexpr (kLanes >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        v = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    if constexpr (kLanes == 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        v = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    return v;
}

// 1 / sqrt(x), off by 2^-23 of itself at most; of numbers below the normal ones, too
__device__ __forceinline__ float inverse_root(float x)
{
    return x < 0x1p-100f ? __builtin_amdgcn_rsqf(x * 0x1p100f) * 0x1p50f : __builtin_amdgcn_rsqf(x);
}

template <bool kFromF32, bool kToF32, int kLanes, int kTokens>
__global__ void __launch_bounds__(kThreads) rotate_kernel(RotateArgs a)
{
    constexpr int kHeads = kThreads / kLanes;
    __shared__ float2 turns[kTokens][kMaxDim / 2];
    const uint32_t chunk = blockIdx.x / a.per_chunk, chunks = ((uint32_t)a.tokens + kTokens - 1) / kTokens;
    const int b = (int)(chunk / chunks), t = (int)(chunk % chunks) * kTokens, here = std::min(kTokens, a.tokens - t);
    const int lane = threadIdx.x % kLanes;
    int head = (int)(blockIdx.x % a.per_chunk) * kHeads + (int)threadIdx.x / kLanes;
    const int step = kHeads * (int)a.per_chunk, end = a.ends[2];
    // a lane's two runs: of the rotated part, elements p .. p + 3 of its pairs' two halves, or both behind each other
    const bool there = 8 * lane < a.dim, rotated = 4 * lane < a.pairs;
    const int e0 = rotated && a.interleaved == 0 ? 4 * lane : 8 * lane, e1 = rotated && a.interleaved == 0 ? a.pairs + 4 * lane : 8 * lane + 4;
    const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 x[kTokens], y[kTokens], w0 = none, w1 = none;
    int which = 0;
    char *to = nullptr;
    int64_t to_token = 0;
    auto load = [&] {
        which = head < a.ends[0] ? 0 : head < a.ends[1] ? 1 : 2;
        const char *from = nullptr;
        int64_t from_token = 0;
        const float *weight = nullptr;
        // (a part of the arguments for each: chosen by number they would be read through memory, and every load would wait for that)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (which != i) continue;
            const RotatePart &p = a.part[i];
            const int h = head - (i == 0 ? 0 : a.ends[i - 1]);
            from = p.from + b * p.from_batch + t * p.from_token + h * p.from_head;
            to = p.to + b * p.to_batch + t * p.to_token + h * p.to_head;
            from_token = p.from_token, to_token = p.to_token;
            weight = p.weight;
        }
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            x[j] = load4<kFromF32>(from, e0);
            y[j] = load4<kFromF32>(from, e1);
            if (j + 1 < here) from += from_token;    // (the last one again, where there are fewer)
        }
        if (weight != nullptr) {
            w0 = *reinterpret_cast<const f32x4 *>(weight + e0);
            w1 = *reinterpret_cast<const f32x4 *>(weight + e1);
        }
    };
#pragma unroll
    for (int j = 0; j < kTokens; ++j) x[j] = y[j] = none;
    if (there && head < end) load();
    for (int i = threadIdx.x; i < kTokens * a.pairs; i += kThreads) {
        const int j = kTokens == 1 ? 0 : i / a.pairs, pair = i - j * a.pairs;
        const int axis = a.axis_of != nullptr ? a.axis_of[pair] : 0;
        const int64_t token = (int64_t)b * a.tokens + t + std::min(j, here - 1);
        const int32_t position = (uint32_t)axis < (uint32_t)a.axes ? a.positions[token * a.axes + axis] : 0;
        turns[j][pair] = turn(position, a.inv_freq[pair]);
    }
    __syncthreads();
    const bool normed[2] = {a.part[0].weight != nullptr, a.part[1].weight != nullptr};
    while (head < end) {
        // (lanes behind a vector's end have zeros, and the part of the others)
        const bool is_v = head >= a.ends[1], norm = !is_v && (head < a.ends[0] ? normed[0] : normed[1]);
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            if (norm) {
                if (a.layer != 0) {
                    const float mean = head_sum<kLanes>(x[j], y[j]) * a.inverse_dim;
                    if (there) x[j] -= mean, y[j] -= mean;
                }
                const float scale = inverse_root(head_sum<kLanes>(x[j] * x[j], y[j] * y[j]) * a.inverse_dim + a.eps);
                x[j] *= scale * w0;
                y[j] *= scale * w1;
            }
            if (rotated && !is_v) {
                const f32x4 t0 = *reinterpret_cast<const f32x4 *>(&turns[j][4 * lane]), t1 = *reinterpret_cast<const f32x4 *>(&turns[j][4 * lane + 2]);
                const float c[4] = {t0[0], t0[2], t1[0], t1[2]}, s[4] = {t0[1], t0[3], t1[1], t1[3]};
                f32x4 u, v;
                if (a.interleaved == 0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        u[i] = __builtin_fmaf(x[j][i], c[i], -(y[j][i] * s[i]));
                        v[i] = __builtin_fmaf(x[j][i], s[i], y[j][i] * c[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        u[2 * i] = __builtin_fmaf(x[j][2 * i], c[i], -(x[j][2 * i + 1] * s[i]));
                        u[2 * i + 1] = __builtin_fmaf(x[j][2 * i], s[i], x[j][2 * i + 1] * c[i]);
                        v[2 * i] = __builtin_fmaf(y[j][2 * i], c[i + 2], -(y[j][2 * i + 1] * s[i + 2]));
                        v[2 * i + 1] = __builtin_fmaf(y[j][2 * i], s[i + 2], y[j][2 * i + 1] * c[i + 2]);
                    }
                }
                x[j] = u, y[j] = v;
            }
            if (there && j < here) {
                store4<kToF32>(to, e0, x[j]);
                store4<kToF32>(to, e1, y[j]);
                to += to_token;
            }
        }
        head += step;
        if (there && head < end) load();
    }
}

template <bool kFromF32, bool kToF32, int kTokens>
void launch(const RotateArgs &a, int lanes, dim3 grid, hipStream_t st)
{
    if (lanes == 8) rotate_kernel<kFromF32, kToF32, 8, kTokens><<<grid, kThreads, 0, st>>>(a);
    else if (lanes == 16) rotate_kernel<kFromF32, kToF32, 16, kTokens><<<grid, kThreads, 0, st>>>(a);
    else if (lanes == 32) rotate_kernel<kFromF32, kToF32, 32, kTokens><<<grid, kThreads, 0, st>>>(a);
    else rotate_kernel<kFromF32, kToF32, 64, kTokens><<<grid, kThreads, 0, st>>>(a);
}

template <bool kFromF32, bool kToF32>
void launch(const RotateArgs &a, int lanes, int at_a_time, dim3 grid, hipStream_t st)
{
    if (at_a_time == 1) launch<kFromF32, kToF32, 1>(a, lanes, grid, st);
    else launch<kFromF32, kToF32, kTokensOfMany>(a, lanes, grid, st);
}

}  // namespace

}  // namespace fgmp

using namespace fgmp;

extern "C" {

fgmp_status_t fgmp_rotate_heads(const fgmp_heads_t *q, const fgmp_heads_t *k, const fgmp_heads_t *v, fgmp_dtype_t dt, int64_t batch, int64_t tokens,
                                int64_t q_heads, int64_t heads, int64_t head_dim, const float *q_weight, const float *k_weight, fgmp_norm_t kind,
                                float eps, const int32_t *positions, int64_t axes, const int32_t *axis_of, const float *inv_freq, int64_t rotary_dim,
                                int interleaved, const fgmp_heads_t *q_out, const fgmp_heads_t *k_out, const fgmp_heads_t *v_out,
                                fgmp_dtype_t out_dt, void *stream)
{
    if (q == nullptr || (k == nullptr && v != nullptr) || (k == nullptr) != (k_out == nullptr) || (v == nullptr) != (v_out == nullptr) || !known_dtype(dt) ||
        !known_dtype(out_dt) || batch <= 0 || tokens <= 0 || q_heads <= 0 || (k != nullptr && heads <= 0) || head_dim <= 0 || rotary_dim < 0 ||
        (k == nullptr && k_weight != nullptr) || (kind != FGMP_NORM_RMS && kind != FGMP_NORM_LAYER) || !(eps >= 0.0f) || !(eps < INFINITY))
        return FGMP_ERR_INVALID_ARG;
    if (rotary_dim > 0 && (positions == nullptr || inv_freq == nullptr || axes <= 0 || (axes > 1 && axis_of == nullptr))) return FGMP_ERR_INVALID_ARG;
    if (head_dim % 8 != 0 || rotary_dim % 8 != 0 || rotary_dim > head_dim) return FGMP_ERR_BAD_SHAPE;
    if (head_dim > kMaxDim || batch > 65535 || q_heads > 65535 || heads > 65535 || tokens > (int64_t)1 << 30 || axes > 65535) return FGMP_ERR_UNSUPPORTED;
    if (!aligned16(q_weight) || !aligned16(k_weight) || ((uintptr_t)positions & 3u) != 0u || ((uintptr_t)axis_of & 3u) != 0u || ((uintptr_t)inv_freq & 3u) != 0u)
        return FGMP_ERR_BAD_ALIGN;
    RotateArgs a = {};
    const fgmp_heads_t *const from[3] = {q, k, v}, *const to[3] = {q_out, k_out, v_out};
    const int size = dtype_size(dt), out_size = dtype_size(out_dt);
    int32_t end = 0;
    for (int i = 0; i < 3; ++i) {
        if (from[i] != nullptr) {
            const int64_t n = i == 0 ? q_heads : heads;
            fgmp_status_t rc = check_heads(from[i], batch, tokens, n, (int)head_dim, size, false);
            if (rc == FGMP_OK) rc = check_heads(to[i], batch, tokens, n, (int)head_dim, out_size, true);
            if (rc != FGMP_OK) return rc;
            a.part[i] = {static_cast<const char *>(from[i]->data), static_cast<char *>(to[i]->data), from[i]->batch_stride * size, from[i]->token_stride * size,
                         from[i]->head_stride * size, to[i]->batch_stride * out_size, to[i]->token_stride * out_size, to[i]->head_stride * out_size,
                         i == 0 ? q_weight : i == 1 ? k_weight : nullptr};
            end += (int32_t)n;
        }
        a.ends[i] = end;
    }
    int lanes = 8;
    while (8 * lanes < head_dim) lanes *= 2;
    const int at_a_time = tokens >= kTokensOfMany && batch * tokens >= kMany ? kTokensOfMany : 1;
    const int64_t all = batch * ((tokens + at_a_time - 1) / at_a_time), turns = (end + kThreads / lanes - 1) / (kThreads / lanes);
    a.per_chunk = (uint32_t)std::min<int64_t>(turns, std::max<int64_t>(1, 1024 / all));
    if (!launch_counts(all * a.per_chunk, kThreads)) return FGMP_ERR_UNSUPPORTED;
    a.tokens = (int32_t)tokens;
    a.dim = (int32_t)head_dim;
    a.pairs = (int32_t)(rotary_dim / 2);
    a.axes = (int32_t)axes;
    a.interleaved = interleaved != 0;
    a.layer = kind == FGMP_NORM_LAYER;
    a.eps = eps;
    a.inverse_dim = 1.0f / (float)head_dim;
    a.positions = positions;
    a.axis_of = axis_of;
    a.inv_freq = inv_freq;
    const dim3 grid((unsigned)(all * a.per_chunk));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32 && out_dt == FGMP_F32) launch<true, true>(a, lanes, at_a_time, grid, st);
    else if (dt == FGMP_F32) launch<true, false>(a, lanes, at_a_time, grid, st);
    else if (out_dt == FGMP_F32) launch<false, true>(a, lanes, at_a_time, grid, st);
    else launch<false, false>(a, lanes, at_a_time, grid, st);
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

}  // extern "C"
