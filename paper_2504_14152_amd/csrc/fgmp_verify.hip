// Which drafted tokens of a step are kept, by the target's probabilities and given random numbers, and the token behind them.
//
// The walk over a sequence's drafted tokens needs a few numbers of its rows only: a child t of the last kept token, whose row is r, is kept if
// u_t q_t(x_t) < p_r(x_t), or, for tokens that were not drawn from a distribution, u_t c < p_r(x_t), c being 1 less the probabilities of the children refused before.
// Every workgroup of a sequence does that for itself.  Of one row, where it ends, all of the vocabulary counts: w = max(p_r - q_r, 0), or p_r without the
// refused tokens, and the token behind is the first one up to which the sum of w exceeds u_0 times the whole sum.
// Memory and a few round trips bound it: waves add up segments of kSegment elements each, and the workgroup that is the last of its sequence finds the segment,
// of which one wave finds the element.  Sums are of 64 bits: in 32, those over a vocabulary are off by more than many a token's probability.
#include <algorithm>

#include "fgmp_cache.hpp"

namespace fgmp {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kRows = 16, kSegment = 64 * kRows;
constexpr int kMaxTokens = 1024;
constexpr int64_t kMaxVocab = (int64_t)1 << 24, kMaxBatch = 16384;

struct VerifyArgs {
    const char *target, *draft;
    int64_t target_batch, target_row, draft_batch, draft_row;   // bytes
    const int32_t *tokens, *parents, *counts;
    const float *uniforms;
    int32_t *rows, *accepted, *next;
    int32_t n, vocab, segments;
    uint32_t workgroups;       // of a sequence
    uint32_t counter_shift;
    uint32_t *counters;        // arrivals, zero between calls
    double *sums;              // of each sequence's segments
};

template <bool kF32>
__device__ __forceinline__ float element(const char *row, int64_t i)
{
    if constexpr (kF32) return reinterpret_cast<const float *>(row)[i];
    else return (float)reinterpret_cast<const __bf16 *>(row)[i];
}

// (partial sums cross XCDs: accesses of agent scope, which every XCD sees once they are complete)
__device__ __forceinline__ void store_sum(double *to, double x)
{
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(to), __builtin_bit_cast(unsigned long long, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ double load_sum(double *from)
{
    return __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<unsigned long long *>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
// Sum over this lane and those before it.
__device__ __forceinline__ double wave_scan(double x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double before = __shfl_up(x, d);
        if (lane >= d) x += before;
    }
    return x;
}

// Where a sequence's walk ends.
struct Walk {
    int32_t count;             // tokens of the sequence, its first one included
    int32_t last, kept;        // the last kept token, and how many are
    int32_t refused;           // of a tree: children of it that were refused, in refused_token[]; of drawn tokens: 1 if one was
};

struct Shared {
    float p[kMaxTokens], u[kMaxTokens];
    int32_t parent[kMaxTokens], token[kMaxTokens], row[kMaxTokens], refused_token[kMaxTokens];
    Walk walk;
    double part[kWaves];
    int32_t first_refused, segment;
    double rest;
    bool last_workgroup;
};

template <bool kF32>
__device__ __forceinline__ void walk_of(const VerifyArgs &a, int b, Shared &s)
{
    const int32_t given = a.counts != nullptr ? a.counts[b] : a.n, count = given < 0 ? 0 : given > a.n ? a.n : given;
    const char *target = a.target + b * a.target_batch;
    const int64_t at = (int64_t)b * a.n;
    if (threadIdx.x == 0) s.first_refused = count;
    __syncthreads();
    for (int t = threadIdx.x; t < count; t += kThreads) {
        const int32_t token = a.tokens[at + t], parent = a.parents != nullptr ? a.parents[at + t] : t - 1;
        const bool there = t > 0 && (uint32_t)token < (uint32_t)a.vocab && (uint32_t)parent < (uint32_t)t;
        const float u = a.uniforms[at + t];
        const float p = there ? element<kF32>(target + parent * a.target_row, token) : 0.0f;
        if (a.parents == nullptr) {
            // a chain: up to the first one that is refused
            const float q = a.draft != nullptr && there ? element<kF32>(a.draft + b * a.draft_batch + parent * a.draft_row, token) : 1.0f;
            s.row[t] = t;
            s.token[t] = token;
            if (t > 0 && !((double)u * (double)q < (double)p)) atomicMin(&s.first_refused, t);
        } else {
            s.p[t] = p, s.u[t] = u, s.token[t] = token;
            s.parent[t] = there ? parent : -1;
        }
    }
    __syncthreads();
    if (a.parents == nullptr) {
        if (threadIdx.x == 0) {
            s.walk = {count, s.first_refused - 1, s.first_refused, s.first_refused < count ? 1 : 0};
            if (s.first_refused < count) s.refused_token[0] = s.token[s.first_refused];
        }
    } else if (threadIdx.x == 0) {
        Walk w = {count, 0, count > 0 ? 1 : 0, 0};
        double left = 1.0;
        if (count > 0) s.row[0] = 0;
        for (int t = 1; t < count; ++t) {
            if (s.parent[t] != w.last) continue;
            bool fresh = true;      // (a token that was refused already has nothing left)
            for (int i = 0; i < w.refused; ++i) fresh = fresh && s.refused_token[i] != s.token[t];
            if (!fresh) continue;
            const double p = s.p[t];
            if ((double)s.u[t] * left < p) {
                s.row[w.kept++] = t;
                w.last = t, w.refused = 0, left = 1.0;
            } else {
                s.refused_token[w.refused++] = s.token[t];
                left -= p > 0.0 ? p : 0.0;
            }
        }
        s.walk = w;
    }
    __syncthreads();
}

// Weights of a segment's elements: w[r] that of element kSegment * segment + 64 r + lane.  `whole`: the row as it is, nothing taken from it.
template <bool kF32>
__device__ __forceinline__ void weights_of(const VerifyArgs &a, int b, int segment, const Shared &s, bool whole, double *w)
{
    const int lane = threadIdx.x & 63, first = segment * kSegment + lane;
    const char *target = a.target + b * a.target_batch + s.walk.last * a.target_row;
    const bool less = !whole && a.draft != nullptr && s.walk.refused != 0;
    float p[kRows], q[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) p[r] = first + 64 * r < a.vocab ? element<kF32>(target, first + 64 * r) : 0.0f;
    if (less) {
        const char *draft = a.draft + b * a.draft_batch + s.walk.last * a.draft_row;
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[r] = first + 64 * r < a.vocab ? element<kF32>(draft, first + 64 * r) : 0.0f;
    } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[r] = 0.0f;
        if (a.draft == nullptr && !whole) {
            for (int i = 0; i < s.walk.refused; ++i) {
                const int at = s.refused_token[i] - first;
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    if (at == 64 * r) p[r] = 0.0f;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const double x = (double)p[r] - (double)q[r];
        w[r] = x > 0.0 ? x : 0.0;   // (NaN counts as nothing)
    }
}

template <bool kF32>
__device__ __forceinline__ double segment_sum(const VerifyArgs &a, int b, int segment, const Shared &s, bool whole)
{
    double w[kRows], sum = 0.0;
    weights_of<kF32>(a, b, segment, s, whole, w);
#pragma unroll
    for (int r = 0; r < kRows; ++r) sum += w[r];
    return wave_sum(sum);
}

// The token behind, by the sums of the segments; -1 where they are all nothing.  For all threads of a workgroup.
template <bool kF32>
__device__ __forceinline__ int32_t pick(const VerifyArgs &a, int b, Shared &s, bool whole)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double *const sums = a.sums + (int64_t)b * a.segments;
    const int each = (a.segments + kThreads - 1) / kThreads, first = std::min(tid * each, a.segments), end = std::min(first + each, a.segments);
    double mine = 0.0;
    for (int i = first; i < end; ++i) mine += load_sum(&sums[i]);
    const double incl = wave_scan(mine);
    __syncthreads();
    if (lane == 63) s.part[wave] = incl;
    if (tid == 0) s.segment = -1;
    __syncthreads();
    double before = 0.0, total = 0.0;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
        before += x < wave ? s.part[x] : 0.0;
        total += s.part[x];
    }
    if (!(total > 0.0)) return -1;
    double u = (double)a.uniforms[(int64_t)b * a.n];
    u = u > 0.0 ? u < 1.0 ? u : 1.0 : 0.0;   // (outside of 0 .. 1: nearest to it)
    const double wanted = u * total;
    // The first segment behind whose end more than that is summed up; where rounding leaves none, the last one that has anything.
    const double ahead = __shfl_up(incl, 1);
    double sum = before + (lane > 0 ? ahead : 0.0);
    int32_t found = -1, any = -1;
    double rest = 0.0;
    for (int i = first; i < end; ++i) {
        const double x = load_sum(&sums[i]);
        if (x > 0.0) any = i;
        if (found < 0 && x > 0.0 && sum + x > wanted) found = i, rest = wanted - sum;
        sum += x;
    }
    if (found >= 0) atomicMin((unsigned int *)&s.segment, (unsigned int)found);
    __syncthreads();
    const int32_t segment = s.segment;
    __syncthreads();
    if (segment == found && found >= 0) s.rest = rest;
    if (segment < 0 && any >= 0) atomicMax(&s.segment, any);
    __syncthreads();
    const bool none = segment < 0;
    const int32_t here = s.segment;
    if (wave != 0) return 0;
    // one wave: the row of 64 elements, then the element
    double w[kRows];
    weights_of<kF32>(a, b, here, s, whole, w);
    const double left = none ? INFINITY : s.rest;
    double up_to = 0.0;
    int32_t token = -1, last = 0;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const double in_row = wave_scan(w[r]), all = __shfl(in_row, 63);
        const uint64_t over = __ballot(w[r] > 0.0 && up_to + in_row > left), some = __ballot(w[r] > 0.0);
        if (token < 0 && over != 0ull) token = 64 * r + __builtin_ctzll(over);
        if (some != 0ull) last = 64 * r + 63 - __builtin_clzll(some);
        up_to += all;
    }
    return kSegment * here + (token >= 0 ? token : last);
}

template <bool kF32>
__global__ void __launch_bounds__(kThreads) verify_kernel(VerifyArgs a)
{
    __shared__ Shared s;
    const int b = (int)(blockIdx.x / a.workgroups), part = (int)(blockIdx.x % a.workgroups), wave = threadIdx.x >> 6;
    walk_of<kF32>(a, b, s);
    if (part == 0) {
        for (int t = threadIdx.x; t < a.n; t += kThreads) a.rows[(int64_t)b * a.n + t] = t < s.walk.kept ? s.row[t] : -1;
        if (threadIdx.x == 0) a.accepted[b] = s.walk.kept;
        if (threadIdx.x == 0 && s.walk.count == 0) a.next[b] = -1;
    }
    if (s.walk.count == 0) return;
    for (int segment = part * kWaves + wave; segment < a.segments; segment += (int)a.workgroups * kWaves) {
        const double sum = segment_sum<kF32>(a, b, segment, s, false);
        if ((threadIdx.x & 63) == 0) store_sum(&a.sums[(int64_t)b * a.segments + segment], sum);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    uint32_t *const counter = &a.counters[(uint32_t)b << a.counter_shift];
    if (threadIdx.x == 0) {
        s.last_workgroup = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.workgroups - 1u;
        if (s.last_workgroup) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s.last_workgroup) return;
    int32_t token = pick<kF32>(a, b, s, false);
    if (token < 0) {
        // nothing is left of the row by rounding alone (or the row is all zeros): the row as it is
        __syncthreads();
        for (int segment = wave; segment < a.segments; segment += kWaves) {
            const double sum = segment_sum<kF32>(a, b, segment, s, true);
            if ((threadIdx.x & 63) == 0) store_sum(&a.sums[(int64_t)b * a.segments + segment], sum);
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        token = pick<kF32>(a, b, s, true);
    }
    if (threadIdx.x == 0) a.next[b] = token;
}

}  // namespace

}  // namespace fgmp

using namespace fgmp;

extern "C" {

size_t fgmp_verify_drafts_workspace_bytes(int64_t batch, int64_t tokens, int64_t vocab)
{
    if (batch <= 0 || batch > kMaxBatch || tokens <= 0 || tokens > kMaxTokens || vocab <= 0 || vocab > kMaxVocab) return 0;
    return kWsCtrlRegion + (size_t)(batch * ((vocab + kSegment - 1) / kSegment)) * sizeof(double);
}

fgmp_status_t fgmp_verify_drafts(const void *target, fgmp_dtype_t dt, int64_t target_batch_stride, int64_t target_row_stride, const void *draft,
                                 int64_t draft_batch_stride, int64_t draft_row_stride, int64_t batch, int64_t tokens, int64_t vocab,
                                 const int32_t *token_ids, const int32_t *parents, const int32_t *counts, const float *uniforms, int32_t *rows,
                                 int32_t *accepted, int32_t *next, void *workspace, size_t workspace_bytes, void *stream)
{
    if (target == nullptr || token_ids == nullptr || uniforms == nullptr || rows == nullptr || accepted == nullptr || next == nullptr ||
        workspace == nullptr || !known_dtype(dt) || batch <= 0 || tokens <= 0 || vocab <= 0 || (draft != nullptr && parents != nullptr))
        return FGMP_ERR_INVALID_ARG;
    if (batch > kMaxBatch || tokens > kMaxTokens || vocab > kMaxVocab) return FGMP_ERR_UNSUPPORTED;
    const int64_t strides[4] = {target_batch_stride, target_row_stride, draft_batch_stride, draft_row_stride};
    const int64_t counted[4] = {batch, tokens, batch, tokens - 1};
    for (int i = 0; i < (draft != nullptr ? 4 : 2); ++i) {
        if (counted[i] > 1 && strides[i] < 0) return FGMP_ERR_BAD_SHAPE;
        if (counted[i] > 1 && strides[i] > (int64_t)1 << 40) return FGMP_ERR_UNSUPPORTED;
    }
    const int size = dtype_size(dt);
    if ((uintptr_t)target % size != 0u || (uintptr_t)draft % size != 0u || ((uintptr_t)token_ids & 3u) != 0u || ((uintptr_t)parents & 3u) != 0u ||
        ((uintptr_t)counts & 3u) != 0u || ((uintptr_t)uniforms & 3u) != 0u || ((uintptr_t)rows & 3u) != 0u || ((uintptr_t)accepted & 3u) != 0u ||
        ((uintptr_t)next & 3u) != 0u || !aligned16(workspace))
        return FGMP_ERR_BAD_ALIGN;
    if (workspace_bytes < fgmp_verify_drafts_workspace_bytes(batch, tokens, vocab)) return FGMP_ERR_BUFFER_TOO_SMALL;
    VerifyArgs a = {};
    a.target = static_cast<const char *>(target);
    a.draft = static_cast<const char *>(draft);
    // (a single one's stride is taken times zero, and might be anything)
    a.target_batch = batch > 1 ? target_batch_stride * size : 0;
    a.target_row = tokens > 1 ? target_row_stride * size : 0;
    a.draft_batch = batch > 1 ? draft_batch_stride * size : 0;
    a.draft_row = tokens > 2 ? draft_row_stride * size : 0;
    a.tokens = token_ids;
    a.parents = parents;
    a.counts = counts;
    a.uniforms = uniforms;
    a.rows = rows;
    a.accepted = accepted;
    a.next = next;
    a.n = (int32_t)tokens;
    a.vocab = (int32_t)vocab;
    a.segments = (int32_t)((vocab + kSegment - 1) / kSegment);
    a.counter_shift = batch <= 1024 ? 4u : 0u;   // (lines of their own, where the control region has room)
    a.counters = static_cast<uint32_t *>(workspace);
    a.sums = reinterpret_cast<double *>(static_cast<char *>(workspace) + kWsCtrlRegion);
    const int64_t most = (a.segments + kWaves - 1) / kWaves;
    a.workgroups = (uint32_t)std::min<int64_t>(most, std::max<int64_t>(1, 8192 / batch));
    const dim3 grid((unsigned)(batch * a.workgroups));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32) verify_kernel<true><<<grid, kThreads, 0, st>>>(a);
    else verify_kernel<false><<<grid, kThreads, 0, st>>>(a);
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

}  // extern "C"
