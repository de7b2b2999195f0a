// Queries, keys and values as a product leaves them, made ready for attention in one pass: queries and keys normed for each head and rotated by
// their positions, values converted.
//   u = w (x - mean) / sqrt(mean((x - mean)^2) + eps);   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * inv_freq
// Memory bounds it: every element is read and written once.  kLanes lanes have a vector of a head, each two runs of four elements, which are
// the two halves of four pairs: a rotation stays in a lane, and a norm's sums take log2(kLanes) steps between lanes.  A workgroup has
// one token and the heads behind each other; the token's sines and cosines are found once, by one thread for each pair, and go through LDS.
#include <algorithm>

#include "fgmp_cache.hpp"

namespace fgmp {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kMaxDim = 512;

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
    uint32_t per_token;        // workgroups that share a token's heads
    float eps;
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

template <int kLanes>
__device__ __forceinline__ float head_sum(f32x4 x, f32x4 y)
{
    float v = ((x[0] + x[1]) + (x[2] + x[3])) + ((y[0] + y[1]) + (y[2] + y[3]));
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

template <bool kFromF32, bool kToF32, int kLanes>
__global__ void __launch_bounds__(kThreads) rotate_kernel(RotateArgs a)
{
    constexpr int kHeads = kThreads / kLanes;
    __shared__ float2 turns[kMaxDim / 2];
    const uint32_t token = blockIdx.x / a.per_token;
    const int b = (int)(token / (uint32_t)a.tokens), t = (int)(token % (uint32_t)a.tokens);
    const int lane = threadIdx.x % kLanes, first = (int)(blockIdx.x % a.per_token) * kHeads + (int)threadIdx.x / kLanes;
    // a lane's two runs: of the rotated part, elements p .. p + 3 of its pairs' two halves, or both behind each other
    const bool there = 8 * lane < a.dim, rotated = 4 * lane < a.pairs;
    const int e0 = rotated && a.interleaved == 0 ? 4 * lane : 8 * lane, e1 = rotated && a.interleaved == 0 ? a.pairs + 4 * lane : 8 * lane + 4;
    auto load = [&](int head, f32x4 &x, f32x4 &y) {
        const RotatePart &p = a.part[head < a.ends[0] ? 0 : head < a.ends[1] ? 1 : 2];
        const int h = head < a.ends[0] ? head : head < a.ends[1] ? head - a.ends[0] : head - a.ends[1];
        const char *from = p.from + b * p.from_batch + t * p.from_token + h * p.from_head;
        x = load4<kFromF32>(from, e0);
        y = load4<kFromF32>(from, e1);
    };
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
    if (there && first < a.ends[2]) load(first, x, y);
    for (int i = threadIdx.x; i < a.pairs; i += kThreads) {
        const int axis = a.axis_of != nullptr ? a.axis_of[i] : 0;
        const int32_t position = (uint32_t)axis < (uint32_t)a.axes ? a.positions[(int64_t)token * a.axes + axis] : 0;
        turns[i] = turn(position, a.inv_freq[i]);
    }
    __syncthreads();
    for (int head = first; head < a.ends[2]; head += kHeads * (int)a.per_token) {
        if (head != first && there) load(head, x, y);
        const int which = head < a.ends[0] ? 0 : head < a.ends[1] ? 1 : 2;
        const RotatePart &p = a.part[which];
        if (which < 2) {
            if (p.weight != nullptr) {
                if (a.layer != 0) {
                    const float mean = head_sum<kLanes>(x, y) / (float)a.dim;
                    if (there) x -= mean, y -= mean;
                }
                const float scale = 1.0f / __builtin_sqrtf(head_sum<kLanes>(x * x, y * y) / (float)a.dim + a.eps);
                if (there) {
                    x *= scale * *reinterpret_cast<const f32x4 *>(p.weight + e0);
                    y *= scale * *reinterpret_cast<const f32x4 *>(p.weight + e1);
                }
            }
            if (rotated) {
                const float2 *c = turns + 4 * lane;
                f32x4 u, v;
                if (a.interleaved == 0) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        u[j] = __builtin_fmaf(x[j], c[j].x, -(y[j] * c[j].y));
                        v[j] = __builtin_fmaf(x[j], c[j].y, y[j] * c[j].x);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        u[2 * j] = __builtin_fmaf(x[2 * j], c[j].x, -(x[2 * j + 1] * c[j].y));
                        u[2 * j + 1] = __builtin_fmaf(x[2 * j], c[j].y, x[2 * j + 1] * c[j].x);
                        v[2 * j] = __builtin_fmaf(y[2 * j], c[j + 2].x, -(y[2 * j + 1] * c[j + 2].y));
                        v[2 * j + 1] = __builtin_fmaf(y[2 * j], c[j + 2].y, y[2 * j + 1] * c[j + 2].x);
                    }
                }
                x = u, y = v;
            }
        }
        if (there) {
            const int h = which == 0 ? head : head - a.ends[which - 1];
            char *to = p.to + b * p.to_batch + t * p.to_token + h * p.to_head;
            store4<kToF32>(to, e0, x);
            store4<kToF32>(to, e1, y);
        }
    }
}

template <bool kFromF32, bool kToF32>
void launch(const RotateArgs &a, int lanes, dim3 grid, hipStream_t st)
{
    if (lanes == 8) rotate_kernel<kFromF32, kToF32, 8><<<grid, kThreads, 0, st>>>(a);
    else if (lanes == 16) rotate_kernel<kFromF32, kToF32, 16><<<grid, kThreads, 0, st>>>(a);
    else if (lanes == 32) rotate_kernel<kFromF32, kToF32, 32><<<grid, kThreads, 0, st>>>(a);
    else rotate_kernel<kFromF32, kToF32, 64><<<grid, kThreads, 0, st>>>(a);
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
    const int64_t all = batch * tokens, turns = (end + kThreads / lanes - 1) / (kThreads / lanes);
    a.per_token = (uint32_t)std::min<int64_t>(turns, std::max<int64_t>(1, 1024 / all));
    if (!launch_counts(all * a.per_token, kThreads)) return FGMP_ERR_UNSUPPORTED;
    a.tokens = (int32_t)tokens;
    a.dim = (int32_t)head_dim;
    a.pairs = (int32_t)(rotary_dim / 2);
    a.axes = (int32_t)axes;
    a.interleaved = interleaved != 0;
    a.layer = kind == FGMP_NORM_LAYER;
    a.eps = eps;
    a.positions = positions;
    a.axis_of = axis_of;
    a.inv_freq = inv_freq;
    const dim3 grid((unsigned)(all * a.per_token));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32 && out_dt == FGMP_F32) launch<true, true>(a, lanes, grid, st);
    else if (dt == FGMP_F32) launch<true, false>(a, lanes, grid, st);
    else if (out_dt == FGMP_F32) launch<false, true>(a, lanes, grid, st);
    else launch<false, false>(a, lanes, grid, st);
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

}  // extern "C"
