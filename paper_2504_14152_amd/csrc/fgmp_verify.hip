// Which drafted tokens of a step are kept, by the target's probabilities and given random numbers, and the token behind them.
//
// The walk over a sequence's drafted tokens needs a few numbers of its rows only: a child t of the last kept token, whose row is r, is kept if
// u_t q_t(x_t) < p_r(x_t), or, for tokens that were not drawn from a distribution, u_t c < p_r(x_t), c being 1 less the probabilities of the children refused before.
// Every workgroup of a sequence does that for itself.  Of one row, where it ends, all of the vocabulary counts: w = max(p_r - q_r, 0), or p_r without the
// refused tokens, and the token behind is the first one up to which the sum of w exceeds u_0 times the whole sum.
// A few dependent round trips to memory bound it (tokens, their probabilities, the row), then the row's bytes: waves add up segments of 64 kRows elements
// each, a wave of the workgroup that is its sequence's last finds the segment, and in it the element.  Up to 64 tokens each wave does the
// walk in its own lanes.  Sums are of 64 bits: in 32, those over a vocabulary are off by more than many a token's probability.
// Of more than 64 tokens one thread of each workgroup walks, in LDS: a tree of 65 / 256 / 1024 over 32000: 12 / 21 / 64 us.  Tokens refused where the walk ends are gone through
// again for each segment, and past 64 tokens for each child behind them too: 24 / 63 / 255 / 1023 refused children of one token: 26 / 58 / 1700 / 24000 us.
// A tree of 25 tokens over 32000: 7.1 us; 32 chains of 8 over 151937, two rows each: 13 us, of which 5 pass before the 39 MB are asked for.
#include <algorithm>
#include <type_traits>

#include "fgmp_cache.hpp"

namespace fgmp {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxTokens = 1024, kFewTokens = 64;
// Rows of 64 elements in a segment.  Short ones where the chip holds all their waves at a time, long ones else: one sequence of 32000, 4 / 8 / 16 rows: 7.5 / 7.5 / 10.4
// us; 64 of 50000, 8 / 16: 11.9 / 14.8; 32 of 2 x 151937, 4 / 8 / 16 / 32: 19.9 / 13.7 / 13.1 / 15.
constexpr int kShortRows = 8, kLongRows = 16, kWavesAtATime = 8192;
// Workgroups at most: about as many as the chip holds, whose waves then have several segments but walk once (64 sequences of 262144 at 768 / 1280 / 2048 / 8192: 21.7 /
// 21.2 / 25.0 / 28.3 us).
constexpr int64_t kMostWorkgroups = 1280;
constexpr int kHeld = 8;           // sums of segments that a lane keeps in registers
constexpr int64_t kMaxVocab = (int64_t)1 << 24, kMaxBatch = 16384;

struct VerifyArgs {
    const char *target, *draft;
    int64_t target_batch, target_row, draft_batch, draft_row;   // bytes
    const int32_t *tokens, *parents, *counts;
    const float *uniforms;
    int32_t *rows, *accepted, *next;
    int32_t n, vocab, segments;
    uint32_t workgroups;       // of a sequence; the sums of a single one stay in its LDS
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

// (NaN: the smaller one of the others.  One instruction, where fmaxf takes another to quiet a NaN)
__device__ __forceinline__ float at_least_zero(float x) { return __builtin_amdgcn_fmed3f(x, 0.0f, INFINITY); }

// A probability: NaN and what is negative count as nothing.
template <bool kF32>
__device__ __forceinline__ float probability(const char *row, int64_t i)
{
    return at_least_zero(element<kF32>(row, i));
}

// A random number; outside of 0 .. 1 the nearest to it.
__device__ __forceinline__ float within_one(float u) { return __builtin_amdgcn_fmed3f(u, 0.0f, 1.0f); }

// (partial sums cross XCDs: system-coherent accesses that bypass the per-XCD L2)
__device__ __forceinline__ void store_sum(double *to, double x)
{
    __hip_atomic_store(reinterpret_cast<unsigned long long *>(to), __builtin_bit_cast(unsigned long long, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
__device__ __forceinline__ double load_sum(double *from)
{
    return __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<unsigned long long *>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM));
}

template <int kControl, int kRowMask>
__device__ __forceinline__ double moved(double x)   // zeros where nothing comes from
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, kControl, kRowMask, 0xF, false);
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), kControl, kRowMask, 0xF, false);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
__device__ __forceinline__ double of_lane(double x, int lane)   // (a lane that is the same for all)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)bits, lane), high = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
// Sum over this lane and those before it: within rows of 16 lanes, then the rows' sums on to the rows behind.
__device__ __forceinline__ double wave_scan(double x)
{
    x += moved<0x111, 0xF>(x);
    x += moved<0x112, 0xF>(x);
    x += moved<0x114, 0xF>(x);
    x += moved<0x118, 0xF>(x);
    x += moved<0x142, 0xA>(x);
    x += moved<0x143, 0xC>(x);
    return x;
}

// What a walk goes over and leaves, of more tokens than a wave has lanes.
struct ManyTokens {
    float p[kMaxTokens], u[kMaxTokens];
    int32_t parent[kMaxTokens], token[kMaxTokens], row[kMaxTokens], refused_token[kMaxTokens];
    int32_t count, last, kept, refused, first_refused;
};
struct NoTokens {};

// Where a sequence's walk ended: the last kept token and how many are, and the tokens refused there.
struct Walk {
    int32_t count, last, kept;
    int32_t refused;            // kFew false: how many, in LDS
    uint64_t kept_lanes, refused_lanes;
    int32_t token;              // kFew: of the lane's
};

// A token's probability in its parent's row, and in what it was drawn from (1 where it was not); `there`: it has a parent and is a token.
template <bool kF32>
__device__ __forceinline__ bool look_up(const VerifyArgs &a, int b, int t, int32_t token, int32_t parent, float *p, float *q)
{
    const bool there = t > 0 && (uint32_t)token < (uint32_t)a.vocab && (uint32_t)parent < (uint32_t)t;
    *p = there ? probability<kF32>(a.target + b * a.target_batch + parent * a.target_row, token) : 0.0f;
    *q = there && a.draft != nullptr ? probability<kF32>(a.draft + b * a.draft_batch + parent * a.draft_row, token) : 1.0f;
    return there;
}

template <bool kF32>
__device__ __forceinline__ Walk walk_of_few(const VerifyArgs &a, int b)
{
    const int t = threadIdx.x & 63;
    const int64_t at = (int64_t)b * a.n + t;
    int32_t count = a.counts != nullptr ? a.counts[b] : a.n;
    Walk w = {};
    w.token = t < a.n ? a.tokens[at] : -1;
    const int32_t up = a.parents != nullptr ? t < a.n ? a.parents[at] : -1 : t - 1;
    const float u_read = t < a.n ? a.uniforms[at] : 0.0f;
    w.count = count = count < 0 ? 0 : count > a.n ? a.n : count;
    if (count == 0) return w;
    float p, q;
    const bool there = look_up<kF32>(a, b, t < count ? t : 0, w.token, up, &p, &q);
    const float u = within_one(u_read);
    if (a.parents == nullptr) {
        // up to the first one that is refused
        const uint64_t fails = __ballot(t > 0 && t < count && !((double)u * (double)q < (double)p));
        w.kept = fails != 0ull ? __builtin_ctzll(fails) : count;
        w.last = w.kept - 1;
        w.kept_lanes = w.kept == 64 ? ~0ull : (1ull << w.kept) - 1ull;
        w.refused_lanes = fails != 0ull ? 1ull << w.kept : 0ull;
        return w;
    }
    w.kept_lanes = 1ull;
    for (;;) {
        uint64_t children = __ballot(there && up == w.last);
        double left = 1.0;
        w.refused_lanes = 0ull;
        bool kept = false;
        while (children != 0ull && !kept) {
            const int child = __builtin_ctzll(children);
            children &= children - 1ull;
            const int32_t token = __builtin_amdgcn_readlane(w.token, child);
            if ((__ballot(w.token == token) & w.refused_lanes) != 0ull) continue;   // (nothing is left for a token that was refused)
            const float p_child = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, p), child));
            const float u_child = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u), child));
            kept = (double)u_child * left < (double)p_child;
            if (kept) {
                w.last = child;
                w.kept_lanes |= 1ull << child;
            } else {
                w.refused_lanes |= 1ull << child;
                left -= (double)p_child;
            }
        }
        if (!kept) break;
    }
    w.kept = __builtin_popcountll(w.kept_lanes);
    return w;
}

template <bool kF32>
__device__ __forceinline__ Walk walk_of_many(const VerifyArgs &a, int b, ManyTokens &s)
{
    const int32_t given = a.counts != nullptr ? a.counts[b] : a.n, count = given < 0 ? 0 : given > a.n ? a.n : given;
    const int64_t at = (int64_t)b * a.n;
    if (threadIdx.x == 0) s.first_refused = count;
    __syncthreads();
    for (int t = threadIdx.x; t < count; t += kThreads) {
        const int32_t token = a.tokens[at + t], parent = a.parents != nullptr ? a.parents[at + t] : t - 1;
        const float u = within_one(a.uniforms[at + t]);
        float p, q;
        const bool there = look_up<kF32>(a, b, t, token, parent, &p, &q);
        if (a.parents == nullptr && t > 0 && !((double)u * (double)q < (double)p)) atomicMin(&s.first_refused, t);
        s.p[t] = p, s.u[t] = u, s.token[t] = token;
        s.parent[t] = there ? parent : -1;
        s.row[t] = t;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s.count = count, s.last = 0, s.kept = count > 0 ? 1 : 0, s.refused = 0;
        if (a.parents == nullptr) {
            s.last = s.first_refused - 1, s.kept = s.first_refused;
            if (s.first_refused < count) s.refused = 1, s.refused_token[0] = s.token[s.first_refused];
        } else {
            double left = 1.0;
            for (int t = 1; t < count; ++t) {
                if (s.parent[t] != s.last) continue;
                bool fresh = true;      // (nothing is left for a token that was refused)
                for (int i = 0; i < s.refused; ++i) fresh = fresh && s.refused_token[i] != s.token[t];
                if (!fresh) continue;
                const double p = s.p[t];
                if ((double)s.u[t] * left < p) {
                    s.row[s.kept++] = t;
                    s.last = t, s.refused = 0, left = 1.0;
                } else {
                    s.refused_token[s.refused++] = s.token[t];
                    left -= p;
                }
            }
        }
    }
    __syncthreads();
    Walk w = {};
    w.count = s.count, w.last = s.last, w.kept = s.kept, w.refused = s.refused;
    return w;
}

// Weights of a segment's elements: w[r] that of element kSegment * segment + 64 r + lane.  `whole`: the row as it is, nothing taken from it.
template <bool kF32, bool kFew, int kRows, typename Tokens>
__device__ __forceinline__ void weights_of(const VerifyArgs &a, int b, int segment, const Walk &walk, const Tokens &s, bool whole, double *w)
{
    constexpr int kSegment = 64 * kRows;
    const int lane = threadIdx.x & 63, first = segment * kSegment + lane;
    const char *target = a.target + b * a.target_batch + walk.last * a.target_row;
    const bool refused = !whole && (kFew ? walk.refused_lanes != 0ull : walk.refused != 0);
    float p[kRows], q[kRows];
    const bool full = (segment + 1) * kSegment <= a.vocab;
    // (a lane behind the vocabulary reads its last element: no load is left out, and none waits for another)
#pragma unroll
    for (int r = 0; r < kRows; ++r) p[r] = element<kF32>(target, full ? first + 64 * r : std::min(first + 64 * r, a.vocab - 1));
    if (refused && a.draft != nullptr) {
        const char *draft = a.draft + b * a.draft_batch + walk.last * a.draft_row;
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[r] = element<kF32>(draft, full ? first + 64 * r : std::min(first + 64 * r, a.vocab - 1));
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[r] = at_least_zero(q[r]);
    } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r) q[r] = 0.0f;
        auto leave_out = [&](int32_t token) {
            const int at = token - first;
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (at == 64 * r) p[r] = 0.0f;
        };
        if (refused) {
            if constexpr (kFew) {
                for (uint64_t left = walk.refused_lanes; left != 0ull; left &= left - 1ull) leave_out(__builtin_amdgcn_readlane(walk.token, __builtin_ctzll(left)));
            } else {
                for (int i = 0; i < walk.refused; ++i) leave_out(s.refused_token[i]);
            }
        }
    }
    // (what is not above 0, or NaN, is nothing)
#pragma unroll
    for (int r = 0; r < kRows; ++r) w[r] = fmax((double)p[r] - (double)q[r], 0.0);
    if (full) return;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if (first + 64 * r >= a.vocab) w[r] = 0.0;
}

template <bool kF32, bool kFew, int kRows, typename Tokens>
__device__ __forceinline__ double segment_sum(const VerifyArgs &a, int b, int segment, const Walk &walk, const Tokens &s, bool whole)
{
    double w[kRows];
    weights_of<kF32, kFew, kRows>(a, b, segment, walk, s, whole, w);
    double sum[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
    for (int r = 4; r < kRows; ++r) sum[r % 4] += w[r];
    return of_lane(wave_scan((sum[0] + sum[1]) + (sum[2] + sum[3])), 63);
}

// The token behind, by the sums of the segments; -1 where they are all nothing.  For one wave.
template <bool kF32, bool kFew, int kRows, typename Tokens, typename Sum>
__device__ __forceinline__ int32_t pick(const VerifyArgs &a, int b, const Walk &walk, const Tokens &s, bool whole, float u0, Sum sum_at)
{
    const int lane = threadIdx.x & 63;
    const int each = (a.segments + 63) / 64, first = std::min(lane * each, a.segments), end = std::min(first + each, a.segments);
    double held[kHeld], mine = 0.0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = first + i < end ? sum_at(first + i) : 0.0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) mine += held[i];
    for (int i = first + kHeld; i < end; ++i) mine += sum_at(i);
    const double incl = wave_scan(mine), total = of_lane(incl, 63);
    if (!(total > 0.0)) return -1;
    const double wanted = (double)within_one(u0) * total;
    // The first lane up to which more than that is summed up, and of its segments the first one; where rounding leaves none, the last that has anything.
    const uint64_t over = __ballot(mine > 0.0 && incl > wanted), some = __ballot(mine > 0.0);
    const int owner = over != 0ull ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
    const double in_lane = wanted - (owner > 0 ? of_lane(incl, owner - 1) : 0.0);
    int32_t found = -1, last_any = first;
    double sum = 0.0, before = 0.0, before_last = 0.0;
    auto look = [&](int i, double x) {
        if (!(x > 0.0)) return;
        last_any = i, before_last = sum;
        if (found < 0 && sum + x > in_lane) found = i, before = sum;
        sum += x;
    };
#pragma unroll
    for (int i = 0; i < kHeld; ++i) look(first + i, held[i]);
    for (int i = first + kHeld; i < end; ++i) look(i, sum_at(i));
    const int32_t segment = __builtin_amdgcn_readlane(found >= 0 ? found : last_any, owner);
    const double rest = in_lane - of_lane(found >= 0 ? before : before_last, owner);
    // the row of 64 elements, then the element
    double w[kRows];
    weights_of<kF32, kFew, kRows>(a, b, segment, walk, s, whole, w);
    double up_to = 0.0, before_row = 0.0, x = w[0];
    int row = -1, last_row = 0;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const double all = of_lane(wave_scan(w[r]), 63);
        if (all > 0.0) last_row = r;
        if (row < 0 && all > 0.0 && up_to + all > rest) row = r, before_row = up_to;
        up_to += all;
    }
    const bool in_row = over != 0ull && row >= 0;
    row = row >= 0 ? row : last_row;
#pragma unroll
    for (int r = 1; r < kRows; ++r) x = row == r ? w[r] : x;
    const double scan = wave_scan(x);
    const uint64_t here = __ballot(x > 0.0 && before_row + scan > rest), any = __ballot(x > 0.0);
    return 64 * kRows * segment + 64 * row + (in_row && here != 0ull ? __builtin_ctzll(here) : 63 - __builtin_clzll(any));
}

template <bool kF32, bool kFew, int kRows>
__global__ void __launch_bounds__(kThreads) verify_kernel(VerifyArgs a)
{
    __shared__ std::conditional_t<kFew, NoTokens, ManyTokens> s;
    __shared__ double own_sums[kWaves];
    __shared__ bool last_workgroup, nothing;
    const int b = (int)(blockIdx.x / a.workgroups), part = (int)(blockIdx.x % a.workgroups);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float u0 = a.uniforms[(int64_t)b * a.n];
    Walk walk;
    if constexpr (kFew) walk = walk_of_few<kF32>(a, b);
    else walk = walk_of_many<kF32>(a, b, s);
    const bool one = a.workgroups == 1u;
    double *const sums = a.sums + (int64_t)b * a.segments;
    if (walk.count > 0) {
        for (int segment = part * kWaves + wave; segment < a.segments; segment += (int)a.workgroups * kWaves) {
            const double sum = segment_sum<kF32, kFew, kRows>(a, b, segment, walk, s, false);
            if (lane == 0) {
                if (one) own_sums[segment] = sum;
                else store_sum(&sums[segment], sum);
            }
        }
    }
    if (part == 0) {
        int32_t *const rows = a.rows + (int64_t)b * a.n;
        if constexpr (kFew) {
            if (wave == kWaves - 1 && lane < a.n) {
                if (lane >= walk.kept) rows[lane] = -1;
                if ((walk.kept_lanes >> lane & 1ull) != 0ull) rows[__builtin_popcountll(walk.kept_lanes & ((1ull << lane) - 1ull))] = lane;
            }
        } else {
            for (int t = tid; t < a.n; t += kThreads) rows[t] = t < walk.kept ? s.row[t] : -1;
        }
        if (tid == kThreads - 1) {
            a.accepted[b] = walk.kept;
            if (walk.count == 0) a.next[b] = -1;
        }
    }
    if (walk.count == 0) return;
    if (!one) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) {
            uint32_t *const counter = &a.counters[(uint32_t)b << a.counter_shift];
            last_workgroup = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.workgroups - 1u;
            if (last_workgroup) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!last_workgroup) return;
    } else {
        __syncthreads();
    }
    auto sum_at = [&](int i) { return one ? own_sums[i] : load_sum(&sums[i]); };
    if (wave == 0) {
        const int32_t token = pick<kF32, kFew, kRows>(a, b, walk, s, false, u0, sum_at);
        if (lane == 0) {
            nothing = token < 0;
            if (token >= 0) a.next[b] = token;
        }
    }
    __syncthreads();
    if (!nothing) return;
    // nothing is left of the row by rounding alone (or the row is all zeros): the row as it is
    for (int segment = wave; segment < a.segments; segment += kWaves) {
        const double sum = segment_sum<kF32, kFew, kRows>(a, b, segment, walk, s, true);
        if (lane == 0) {
            if (one) own_sums[segment] = sum;
            else store_sum(&sums[segment], sum);
        }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (wave == 0) {
        const int32_t token = pick<kF32, kFew, kRows>(a, b, walk, s, true, u0, sum_at);
        if (lane == 0) a.next[b] = token;
    }
}

template <bool kF32, int kRows>
void launch(const VerifyArgs &a, dim3 grid, hipStream_t st)
{
    if (a.n <= kFewTokens) verify_kernel<kF32, true, kRows><<<grid, kThreads, 0, st>>>(a);
    else verify_kernel<kF32, false, kRows><<<grid, kThreads, 0, st>>>(a);
}

template <bool kF32>
void launch(const VerifyArgs &a, int rows, dim3 grid, hipStream_t st)
{
    if (rows == kShortRows) launch<kF32, kShortRows>(a, grid, st);
    else launch<kF32, kLongRows>(a, grid, st);
}

}  // namespace

}  // namespace fgmp

using namespace fgmp;

extern "C" {

size_t fgmp_verify_drafts_workspace_bytes(int64_t batch, int64_t tokens, int64_t vocab)
{
    if (batch <= 0 || batch > kMaxBatch || tokens <= 0 || tokens > kMaxTokens || vocab <= 0 || vocab > kMaxVocab) return 0;
    return kWsCtrlRegion + (size_t)(batch * ((vocab + 64 * kShortRows - 1) / (64 * kShortRows))) * sizeof(double);
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
    const int64_t short_segments = (vocab + 64 * kShortRows - 1) / (64 * kShortRows);
    const int row_count = batch * short_segments <= kWavesAtATime ? kShortRows : kLongRows;
    a.segments = (int32_t)((vocab + 64 * row_count - 1) / (64 * row_count));
    a.counter_shift = batch <= 1024 ? 4u : 0u;   // (lines of their own, where the control region has room)
    a.counters = static_cast<uint32_t *>(workspace);
    a.sums = reinterpret_cast<double *>(static_cast<char *>(workspace) + kWsCtrlRegion);
    const int64_t most = (a.segments + kWaves - 1) / kWaves;
    a.workgroups = (uint32_t)std::min<int64_t>(most, std::max<int64_t>(2, kMostWorkgroups / batch));
    const dim3 grid((unsigned)(batch * a.workgroups));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dt == FGMP_F32) launch<true>(a, row_count, grid, st);
    else launch<false>(a, row_count, grid, st);
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

}  // extern "C"
