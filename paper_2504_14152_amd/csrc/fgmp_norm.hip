// The norms around a block, with its gate and residual scale, in one pass over the residual stream and the block's result:
//   y = residual_scale * x + branch_scale * act(gate) * N(o; post),   h = N(y; pre)
// Nothing but memory bounds it: a row's elements stay in registers from their load to the store of h, each row read and written once.
// A workgroup has one row; every thread holds 8 kChunks of its elements, and the sums over the row (mean, then squares of
// what is left: no difference of large numbers) go through LDS.
#include <algorithm>

#include "fgmp_cache.hpp"

namespace fgmp {

namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int64_t kMaxWidth = 32768;

struct NormArgs {
    const char *x, *o, *gate;
    char *y, *h;
    int64_t ldx, ldo, ld_gate, ldy, ldh;   // bytes
    int64_t gate_rows;
    const float *post_w, *post_b, *pre_w, *pre_b;
    int32_t K, gate_act, layer;
    float eps, residual_scale, branch_scale;
};

template <bool kF32>
__device__ __forceinline__ f32x8 load8(const char *row, int e)
{
    if constexpr (kF32) return *reinterpret_cast<const f32x8 *>(__builtin_assume_aligned(row + 4 * (int64_t)e, 16));
    else return __builtin_convertvector(*reinterpret_cast<const bf16x8 *>(row + 2 * (int64_t)e), f32x8);
}

template <bool kF32>
__device__ __forceinline__ void store8(char *row, int e, f32x8 v)
{
    if constexpr (kF32) {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<f32x4 *>(row + 4 * (int64_t)e) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4 *>(row + 4 * (int64_t)e + 16) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        *reinterpret_cast<bf16x8 *>(row + 2 * (int64_t)e) = __builtin_convertvector(v, bf16x8);   // (nearest even)
    }
}

// Sum over the workgroup, the same in every thread.
template <int kThreads>
__device__ __forceinline__ float row_sum(float v, float *part)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    if constexpr (kThreads > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) v += part[w];
    }
    return v;
}

// N(z; w, b), element e of the row at z[c][e % 8]; elements behind K are not looked at
template <int kThreads, int kChunks>
__device__ __forceinline__ void normalize(f32x8 *z, const NormArgs &a, const float *w, const float *b, float *part)
{
    const int tid = threadIdx.x;
    if (a.layer) {
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (8 * (tid + c * kThreads) < a.K)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += z[c][e];
        const float mean = row_sum<kThreads>(sum, part) / (float)a.K;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) z[c] -= mean;
    }
    float squares = 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (8 * (tid + c * kThreads) < a.K)
#pragma unroll
            for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(z[c][e], z[c][e], squares);
    const float scale = 1.0f / __builtin_sqrtf(row_sum<kThreads>(squares, part) / (float)a.K + a.eps);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int e = 8 * (tid + c * kThreads);
        if (e < a.K) {
            z[c] *= scale * load8<true>(reinterpret_cast<const char *>(w), e);
            if (b != nullptr) z[c] += load8<true>(reinterpret_cast<const char *>(b), e);
        }
    }
}

template <bool kXF32, bool kOF32, bool kHF32, int kThreads, int kChunks>
__global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs a)
{
    __shared__ float part[kThreads / 64];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const char *x = a.x + row * a.ldx;
    f32x8 y[kChunks], u[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int e = 8 * (tid + c * kThreads);
        if (e < a.K) {
            y[c] = load8<kXF32>(x, e);
            if (a.o != nullptr) u[c] = load8<kOF32>(a.o + row * a.ldo, e);
        }
    }
    if (a.o != nullptr) {
        if (a.post_w != nullptr) normalize<kThreads, kChunks>(u, a, a.post_w, a.post_b, part);
        const char *gate = a.gate + row / a.gate_rows * a.ld_gate;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int e = 8 * (tid + c * kThreads);
            if (e < a.K) {
                if (a.gate != nullptr) {
                    f32x8 f = load8<kOF32>(gate, e);
                    if (a.gate_act != FGMP_GATE_NONE) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float s = 1.0f / (1.0f + __expf(-f[i]));
                            f[i] = a.gate_act == FGMP_GATE_SILU ? f[i] * s : s;
                        }
                    }
                    u[c] *= f;
                }
                y[c] = a.residual_scale * y[c] + a.branch_scale * u[c];
                store8<kXF32>(a.y + row * a.ldy, e, y[c]);
            }
        }
    }
    if (a.pre_w != nullptr) {
        normalize<kThreads, kChunks>(y, a, a.pre_w, a.pre_b, part);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int e = 8 * (tid + c * kThreads);
            if (e < a.K) store8<kHF32>(a.h + row * a.ldh, e, y[c]);
        }
    }
}

template <bool kXF32, bool kOF32, bool kHF32>
void norm_launch(const NormArgs &a, int64_t M, hipStream_t st)
{
    const dim3 grid((unsigned)M);
    if (a.K <= 2048) norm_kernel<kXF32, kOF32, kHF32, 256, 1><<<grid, 256, 0, st>>>(a);
    else if (a.K <= 8192) norm_kernel<kXF32, kOF32, kHF32, 512, 2><<<grid, 512, 0, st>>>(a);
    else if (a.K <= 16384) norm_kernel<kXF32, kOF32, kHF32, 512, 4><<<grid, 512, 0, st>>>(a);
    else norm_kernel<kXF32, kOF32, kHF32, 1024, 4><<<grid, 1024, 0, st>>>(a);
}

// a row of K elements of type `dt` for each of M rows
fgmp_status_t check_rows(const void *p, fgmp_dtype_t dt, int64_t ld, int64_t M, int64_t K)
{
    if (!known_dtype(dt)) return FGMP_ERR_INVALID_ARG;
    if (M > 1 && ld < K) return FGMP_ERR_BAD_SHAPE;
    return aligned16(p) && (M == 1 || ld % (16 / dtype_size(dt)) == 0) ? FGMP_OK : FGMP_ERR_BAD_ALIGN;
}

}  // namespace

}  // namespace fgmp

using namespace fgmp;

extern "C" fgmp_status_t fgmp_block_norm(const void *x, fgmp_dtype_t x_dt, int64_t ldx, const void *o, fgmp_dtype_t o_dt, int64_t ldo, const void *gate,
                                         int64_t ld_gate, int64_t gate_rows, fgmp_gate_t gate_act, int64_t M, int64_t K,
                                         const float *post_weight, const float *post_bias, const float *pre_weight, const float *pre_bias,
                                         fgmp_norm_t kind, float eps, float residual_scale, float branch_scale, void *y, int64_t ldy,
                                         void *h, fgmp_dtype_t h_dt, int64_t ldh, void *stream)
{
    if (x == nullptr || M <= 0 || K <= 0 || (kind != FGMP_NORM_RMS && kind != FGMP_NORM_LAYER) || gate_act < FGMP_GATE_NONE ||
        gate_act > FGMP_GATE_SILU || !(eps >= 0.0f) || !(eps < INFINITY))
        return FGMP_ERR_INVALID_ARG;
    if ((o == nullptr) != (y == nullptr) || (pre_weight == nullptr) != (h == nullptr) || (o == nullptr && h == nullptr)) return FGMP_ERR_INVALID_ARG;
    if (o == nullptr && (gate != nullptr || post_weight != nullptr)) return FGMP_ERR_INVALID_ARG;
    if ((post_weight == nullptr && post_bias != nullptr) || (pre_weight == nullptr && pre_bias != nullptr) || (gate != nullptr && gate_rows <= 0))
        return FGMP_ERR_INVALID_ARG;
    if (K % kBlock != 0) return FGMP_ERR_BAD_SHAPE;
    if (K > kMaxWidth || M >= (int64_t)1 << 31) return FGMP_ERR_UNSUPPORTED;
    if (!aligned16(post_weight) || !aligned16(post_bias) || !aligned16(pre_weight) || !aligned16(pre_bias)) return FGMP_ERR_BAD_ALIGN;
    fgmp_status_t rc = check_rows(x, x_dt, ldx, M, K);
    if (rc != FGMP_OK) return rc;
    NormArgs a = {};
    a.x = static_cast<const char *>(x);
    a.ldx = ldx * dtype_size(x_dt);
    a.gate_rows = 1;
    if (o != nullptr) {
        if ((rc = check_rows(o, o_dt, ldo, M, K)) != FGMP_OK || (rc = check_rows(y, x_dt, ldy, M, K)) != FGMP_OK) return rc;
        a.o = static_cast<const char *>(o);
        a.ldo = ldo * dtype_size(o_dt);
        a.y = static_cast<char *>(y);
        a.ldy = ldy * dtype_size(x_dt);
        if (gate != nullptr) {
            if ((rc = check_rows(gate, o_dt, ld_gate, gate_rows < M ? 2 : 1, K)) != FGMP_OK) return rc;
            a.gate = static_cast<const char *>(gate);
            a.ld_gate = ld_gate * dtype_size(o_dt);
            a.gate_rows = gate_rows;
        }
    }
    if (h != nullptr) {
        if ((rc = check_rows(h, h_dt, ldh, M, K)) != FGMP_OK) return rc;
        a.h = static_cast<char *>(h);
        a.ldh = ldh * dtype_size(h_dt);
    }
    a.post_w = post_weight;
    a.post_b = post_bias;
    a.pre_w = pre_weight;
    a.pre_b = pre_bias;
    a.K = (int32_t)K;
    a.gate_act = gate_act;
    a.layer = kind == FGMP_NORM_LAYER;
    a.eps = eps;
    a.residual_scale = residual_scale;
    a.branch_scale = branch_scale;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int types = (x_dt == FGMP_F32 ? 4 : 0) + (o != nullptr && o_dt == FGMP_F32 ? 2 : 0) + (h != nullptr && h_dt == FGMP_F32 ? 1 : 0);
    switch (types) {
    case 0: norm_launch<false, false, false>(a, M, st); break;
    case 1: norm_launch<false, false, true>(a, M, st); break;
    case 2: norm_launch<false, true, false>(a, M, st); break;
    case 3: norm_launch<false, true, true>(a, M, st); break;
    case 4: norm_launch<true, false, false>(a, M, st); break;
    case 5: norm_launch<true, false, true>(a, M, st); break;
    case 6: norm_launch<true, true, false>(a, M, st); break;
    default: norm_launch<true, true, true>(a, M, st); break;
    }
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}
