// The norms around a block, with its gate and residual scale, in one pass over the residual stream and the block's result:
//   y = residual_scale * x + branch_scale * act(gate) * N(o; post),   h = N(y; pre)
// Nothing but memory bounds it: a row's elements stay in registers from their load to the store of h, each row read and written once.
// kThreads threads have a row, each 8 kChunks of its elements, and a workgroup as many rows as make 256 threads.  Sums over the row (the mean,
// then the squares of what is left: no difference of large numbers) stay in a wave where the row does, and go through LDS otherwise.
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
    int64_t gate_rows, M;
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

// Sum over a row's threads, the same in every one of them.
template <int kThreads>
__device__ __forceinline__ float row_sum(float v, float *part)
{
#pragma unroll
    for (int d = 1; d < 64 && d < kThreads; d <<= 1) v += __shfl_xor(v, d);
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
    const int tid = threadIdx.x % kThreads;
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
__global__ void __launch_bounds__(kThreads < 256 ? 256 : kThreads) norm_kernel(NormArgs a)
{
    constexpr int kRows = kThreads < 256 ? 256 / kThreads : 1;
    static_assert(kRows == 1 || kThreads <= 64, "rows of several waves have a workgroup of their own: its barriers are for all");
    __shared__ float part[kThreads < 256 ? 1 : kThreads / 64];
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kThreads;
    const int tid = threadIdx.x % kThreads;
    if (row >= a.M) return;
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

template <bool kXF32, bool kOF32, bool kHF32, int kThreads, int kChunks>
fgmp_status_t norm_launch(const NormArgs &a, hipStream_t st)
{
    constexpr int kRows = kThreads < 256 ? 256 / kThreads : 1;
    const int64_t workgroups = (a.M + kRows - 1) / kRows;
    if (!launch_counts(workgroups, kThreads * kRows)) return FGMP_ERR_UNSUPPORTED;
    norm_kernel<kXF32, kOF32, kHF32, kThreads, kChunks><<<dim3((unsigned)workgroups), kThreads * kRows, 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

// Threads of a row by its width: 64 M elements, residual stream and h in BF16, o in FP32, at 5.3 to 5.8 TB/s from 128 columns to 16384 (4.1 at
// 64, 4.3 above).  With a workgroup to every row 64 columns ran at 0.5 TB/s and 512 at 3.3; with 512 threads holding 32 elements each
// 11008 and 16384 columns at 3.7 and 4.0.
template <bool kXF32, bool kOF32, bool kHF32>
fgmp_status_t norm_launch_width(const NormArgs &a, hipStream_t st)
{
    if (a.K <= 128) return norm_launch<kXF32, kOF32, kHF32, 16, 1>(a, st);
    if (a.K <= 256) return norm_launch<kXF32, kOF32, kHF32, 32, 1>(a, st);
    if (a.K <= 512) return norm_launch<kXF32, kOF32, kHF32, 64, 1>(a, st);
    if (a.K <= 1024) return norm_launch<kXF32, kOF32, kHF32, 64, 2>(a, st);
    if (a.K <= 2048) return norm_launch<kXF32, kOF32, kHF32, 256, 1>(a, st);
    if (a.K <= 4096) return norm_launch<kXF32, kOF32, kHF32, 256, 2>(a, st);
    if (a.K <= 8192) return norm_launch<kXF32, kOF32, kHF32, 512, 2>(a, st);
    if (a.K <= 16384) return norm_launch<kXF32, kOF32, kHF32, 1024, 2>(a, st);
    return norm_launch<kXF32, kOF32, kHF32, 1024, 4>(a, st);
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
    a.M = M;
    a.K = (int32_t)K;
    a.gate_act = gate_act;
    a.layer = kind == FGMP_NORM_LAYER;
    a.eps = eps;
    a.residual_scale = residual_scale;
    a.branch_scale = branch_scale;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int types = (x_dt == FGMP_F32 ? 4 : 0) + (o != nullptr && o_dt == FGMP_F32 ? 2 : 0) + (h != nullptr && h_dt == FGMP_F32 ? 1 : 0);
    switch (types) {
    case 0: return norm_launch_width<false, false, false>(a, st);
    case 1: return norm_launch_width<false, false, true>(a, st);
    case 2: return norm_launch_width<false, true, false>(a, st);
    case 3: return norm_launch_width<false, true, true>(a, st);
    case 4: return norm_launch_width<true, false, false>(a, st);
    case 5: return norm_launch_width<true, false, true>(a, st);
    case 6: return norm_launch_width<true, true, false>(a, st);
    default: return norm_launch_width<true, true, true>(a, st);
    }
}
