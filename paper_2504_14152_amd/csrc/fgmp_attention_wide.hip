// Attention of many rows (query heads of a group, for all new tokens): from 33 rows on, 17 where head_dim is 256, the waves of a workgroup have
// rows of their own, 32 each, and share the keys and values, which go through LDS in tiles of 64 (32 where head_dim is 256) and are read once
// for up to 256 rows (128).
//
// The two products of fgmp_attention.hip in 32 x 32 tiles, S^T = K Q^T and O^T += V^T P^T: of a tile of scores lane 32 g + i has row i
// and keys 8 a + 4 g + j (a, j = 0 .. 3), so the softmax has one step between lanes, and the weights go into the second product from the
// registers they were computed in.  V is transposed on its way into LDS, its keys in the order in which a lane holds the weights.  Two
// buffers: while one tile is worked on, the next one is in registers on its way; one barrier per tile.  Pieces of 16 bytes
// change places within an LDS row (by XOR), so that neither the rows written nor the columns read meet in a bank.
#include <type_traits>

#include "fgmp_attention.hpp"

namespace fgmp {

namespace {

template <int kDim>
struct Tile {
    static constexpr int kKeys = wide_keys(kDim);
    static constexpr int kPieces = kDim / 8;                       // 16-byte pieces of a key
    u32x4 k[kKeys * kPieces];                                      // [key][piece ^ key]
    u32x4 v[kDim * kKeys / 8];                                     // [element][piece ^ element]
    // LDS gives 16 lanes 16 bytes each in a cycle: a piece of 16 keys in a row, or of 16 elements, lies in 16 different places of 256 bytes
    static __device__ __forceinline__ int key_piece(int key, int piece) { return key * kPieces + (piece ^ (kPieces >= 16 ? key & 15 : key >> 1 & 7)); }
    // 16 keys are the k index of a matrix instruction: piece 2 s + g is what lane half g takes of the s-th 16, the groups
    // of four keys 4 s + g and 4 s + g + 2
    static __device__ __forceinline__ int value_piece(int d, int piece)
    {
        return d * (kKeys / 8) + (piece ^ (kKeys == 64 ? ((d >> 1) ^ (d >> 4)) & 7 : ((d >> 2) ^ (d >> 5)) & 3));
    }
    __device__ __forceinline__ u32x2 *value_quad(int d, int quad)
    {
        return reinterpret_cast<u32x2 *>(&v[value_piece(d, quad / 4 * 2 + (quad & 1))]) + (quad >> 1 & 1);
    }
};

__device__ __forceinline__ bool finite_pair(uint32_t w) { return (w & 0x7F800000u) != 0x7F800000u && (w & 0x7F80u) != 0x7F80u; }
__device__ __forceinline__ uint32_t finite_part(uint32_t w)
{
    return ((w & 0x7F80u) != 0x7F80u ? w & 0xFFFFu : 0u) | ((w & 0x7F800000u) != 0x7F800000u ? w & 0xFFFF0000u : 0u);
}

__device__ __forceinline__ float halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// In the order of the instructions before it: kN reads from LDS, each for one matrix instruction, run kAhead in front of them.
template <int kN>
__device__ __forceinline__ void read_ahead()
{
    constexpr int kAhead = 4, kRead = 0x100, kMatrix = 0x008;
    __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
    for (int x = 0; x < kN - kAhead; ++x) {
        __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMatrix, kAhead, 0);
}

template <int kDim, int kWaves>
__global__ void __launch_bounds__(64 * kWaves, kDim == 256 ? 1 : 2) attend_wide_kernel(AttendArgs a)
{
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    constexpr int kKeys = wide_keys(kDim), kHalves = kKeys / 32, kGroups = kKeys / 16;   // (of 16 keys: slots of one page)
    constexpr int kThreads = 64 * kWaves, kPieces = kDim / 8, kBlocks = kDim / 32, kSteps = kDim / 16;
    // loads of a thread: kKeyLoads pieces of keys, kKeyRows rows apart; and of values, kRounds times four keys x 2 kWords elements, of which
    // kQuadThreads threads have a row
    constexpr int kKeyLoads = kKeys * kPieces / kThreads, kKeyRows = kThreads / kPieces;
    constexpr int kWords = kWaves == 8 ? kDim / 64 : kDim == 256 ? 4 : kDim / 32, kQuadThreads = kDim / (2 * kWords), kQuads = kThreads / kQuadThreads;
    constexpr int kRounds = kKeys / 4 / kQuads;
    __shared__ Tile<kDim> buffer[2];
    __shared__ int32_t not_finite;    // the last tile of new tokens some of whose values are not finite

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 5, i = lane & 31;
    const AttendPlace place(a);
    if (!place.there) return;
    const int split = place.split, h = place.h, b = place.b;
    const int32_t n = a.c.length(b), count = a.count(b);
    const int rows = a.tokens * a.group, first = place.block * (32 * kWaves), row = first + 32 * wave + i, t = row / a.group;
    const int head = h * a.group + row - t * a.group;
    const bool empty = first >= count * a.group;
    if (empty && a.splits > 1) return;                       // (written by the launch that joins the ranges)
    const int per = a.range(n), used = a.ranges(n);
    if (split >= used) return;
    const int begin = split * per, tiles = empty ? 0 : std::min(a.tiles(n), begin + per) - begin;
    const int drafted = a.k != nullptr && !empty && split == used - 1 ? count : 0;
    const bool active = first + 32 * wave < count * a.group;   // (a wave without rows loads, and keeps the barriers)

    // ---- a tile on its way: global memory -> registers -> LDS ----
    const uint32_t step = (uint32_t)a.c.token_stride;
    const int key_row = tid / kPieces, key_at = tid % kPieces * 16, quad = tid / kQuadThreads, value_at = tid % kQuadThreads * (4 * kWords);
    // (the even tiles in one set of registers, the odd ones in the other: room for two tiles on their way)
    u32x4 key[2][kKeyLoads];
    uint32_t value[2][kRounds][4][kWords];
    // A wave's loads of one kind and round are of one group of 16 slots, whose page is looked up a tile ahead of the load.
    uint32_t key_page[kKeyLoads], value_page[kRounds], key_first[kKeyLoads], value_first[kRounds];
    const int key_group = wave * (64 / kPieces), value_group = wave * (64 / kQuadThreads);   // (in rows, and in quads)
    const uint32_t last_group = (uint32_t)(n - 1) / 16u;     // (used where there are slots)
    auto look_up = [&](int tile) {
        const uint32_t u = (uint32_t)(begin + tile) * kGroups;
#pragma unroll
        for (int c = 0; c < kKeyLoads; ++c)
            key_page[c] = a.c.page_of(b, a.c.entry_of(std::min(u + (key_group + c * kKeyRows) / 16, last_group), &key_first[c]));
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            value_page[r] = a.c.page_of(b, a.c.entry_of(std::min(u + (value_group + r * kQuads) / 4, last_group), &value_first[r]));
    };
    constexpr std::integral_constant<int, 0> even = {};
    constexpr std::integral_constant<int, 1> odd = {};
    auto load_value = [&](auto set, int r, int j, const char *at) {
        if constexpr (kWords == 1) {
            value[set][r][j][0] = *reinterpret_cast<const uint32_t *>(at);
        } else if constexpr (kWords == 2) {
            const u32x2 x = *reinterpret_cast<const u32x2 *>(at);
            value[set][r][j][0] = x[0], value[set][r][j][1] = x[1];
        } else {
            const u32x4 x = *reinterpret_cast<const u32x4 *>(at);
#pragma unroll
            for (int w = 0; w < 4; ++w) value[set][r][j][w] = x[w];
        }
    };
    // rows behind the last slot in use are read as that one
    auto load_keys = [&](auto set, int tile) {
        const int left = n - (begin + tile) * kKeys;
#pragma unroll
        for (int c = 0; c < kKeyLoads; ++c) {
            const char *base = a.c.k + a.c.offset(key_page[c], key_first[c], h);
            int r = (key_row + c * kKeyRows) % 16;
            if (left < kKeys && (key_group + c * kKeyRows) / 16 >= (left - 1) / 16) r = std::min(r, (n - 1) & 15);
            key[set][c] = *reinterpret_cast<const u32x4 *>(base + ((uint32_t)r * step + (uint32_t)key_at));
        }
    };
    auto load_values = [&](auto set, int tile) {
        const int left = n - (begin + tile) * kKeys;
#pragma unroll
        for (int round = 0; round < kRounds; ++round) {
            const char *base = a.c.v + a.c.offset(value_page[round], value_first[round], h);
            const bool last = left < kKeys && (value_group + round * kQuads) / 4 >= (left - 1) / 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                int r = (quad + round * kQuads) % 4 * 4 + j;
                if (last) r = std::min(r, (n - 1) & 15);
                load_value(set, round, j, base + ((uint32_t)r * step + (uint32_t)value_at));
            }
        }
    };
    auto load_new = [&](int start) {
#pragma unroll
        for (int c = 0; c < kKeyLoads; ++c)
            key[0][c] = *reinterpret_cast<const u32x4 *>(a.k + b * a.k_batch + std::min(start + key_row + c * kKeyRows, drafted - 1) * a.k_token + h * a.k_head + key_at);
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                load_value(even, r, j, a.v + b * a.v_batch + std::min(start + 4 * (quad + r * kQuads) + j, drafted - 1) * a.v_token + h * a.v_head + value_at);
    };
    // `left`: keys of the tile that there are; what lies behind them must not meet a weight of zero: it might not be finite
    auto store = [&](auto set, int left) {
        Tile<kDim> &to = buffer[set];
#pragma unroll
        for (int c = 0; c < kKeyLoads; ++c) to.k[Tile<kDim>::key_piece(key_row + c * kKeyRows, tid % kPieces)] = key[set][c];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int at = quad + r * kQuads;
            if (left < kKeys) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int w = 0; w < kWords; ++w) value[set][r][j][w] = 4 * at + j < left ? value[set][r][j][w] : 0u;
            }
#pragma unroll
            for (int m = 0; m < 2 * kWords; ++m) {
                const uint32_t select = (m & 1) != 0 ? 0x07060302u : 0x05040100u;
                *to.value_quad(tid % kQuadThreads * (2 * kWords) + m, at) = u32x2{__builtin_amdgcn_perm(value[set][r][1][m / 2], value[set][r][0][m / 2], select),
                                                                                  __builtin_amdgcn_perm(value[set][r][3][m / 2], value[set][r][2][m / 2], select)};
            }
        }
    };

    u32x4 q[kSteps];      // lane 32 g + i: row i, of every 32 bytes the g-th 16
    {
        const char *from = a.q + b * a.q_batch + (row < rows ? t * a.q_token + head * a.q_head : h * a.group * a.q_head) + 16 * g;
#pragma unroll
        for (int p = 0; p < kSteps; ++p) q[p] = *reinterpret_cast<const u32x4 *>(from + 32 * p);
    }
    if (tiles > 0) {
        look_up(0);
        load_keys(even, 0);
        load_values(even, 0);
        look_up(std::min(1, tiles - 1));
        load_keys(odd, std::min(1, tiles - 1));
        load_values(odd, std::min(1, tiles - 1));
        look_up(std::min(2, tiles - 1));
    }
    if (tid == 0) not_finite = -1;
    float most = -INFINITY, l = 0.0f;
    f32x16 o[kBlocks];
#pragma unroll
    for (int m = 0; m < kBlocks; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] = 0.0f;

    // ---- a tile in LDS: scores, softmax, second product.  `sees`: bit j, the lane's row sees key j; looked at if `masked` ----
    auto work = [&](const Tile<kDim> &in, bool masked, uint64_t sees, auto ask, auto left_out) {
        f32x16 s[kHalves];
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[half][e] = 0.0f;
#pragma unroll
        for (int p = 0; p < kSteps; ++p)
#pragma unroll
            for (int half = 0; half < kHalves; ++half)
                s[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, in.k[Tile<kDim>::key_piece(32 * half + i, 2 * p + g)]),
                                                                  __builtin_bit_cast(bf16x8, q[p]), s[half], 0, 0, 0);
        read_ahead<kHalves * kSteps>();
        ask();
        if (masked) {
            const uint64_t own = sees >> (4 * g);
#pragma unroll
            for (int half = 0; half < kHalves; ++half)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if ((own >> (32 * half + e / 4 * 8 + e % 4) & 1ull) == 0ull) s[half][e] = -INFINITY;
        }
        float top = most;
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = __builtin_amdgcn_fmed3f(top, s[half][e], INFINITY);   // (a maximum that passes NaN over)
        top = halves_max(top);
        const bool above = (top - most) * a.c2 > kSlack;
        if (__any(above)) {
            // each row for itself: what a row gets must not depend on the rows it shares a wave with
            const float alpha = !above ? 1.0f : most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((most - top) * a.c2);
            most = above ? top : most;
            l *= alpha;
#pragma unroll
            for (int m = 0; m < kBlocks; ++m)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[m][e] *= alpha;
        }
        const float base = most == -INFINITY ? 0.0f : most * a.c2;
        bf16x8 p[kGroups];
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
            f32x8 w;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 2][k % 2 * 8 + e], a.c2, -base));
            l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            p[k] = __builtin_convertvector(w, bf16x8);   // (a choice: see the other kernel's)
        }
        left_out(p);
#pragma unroll
        for (int k = 0; k < kGroups; ++k)
#pragma unroll
            for (int m = 0; m < kBlocks; ++m)
                o[m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, in.v[Tile<kDim>::value_piece(32 * m + i, 2 * k + g)]), p[k], o[m],
                                                               0, 0, 0);
        read_ahead<kGroups * kBlocks>();
    };

    // The next tile goes to LDS, and the one two further on is asked for behind the scores (25 tokens over 8 x 9999 slots: 142 us with the loads in
    // front of the scores, 127 behind them; 102 where all loads hit the L2).  The two ways to ask, with and without rows, are compiled as two
    // blocks in line, either of which may have loads under way, and the registers just stored serve the scores: these wait for all or most loads of
    // the step before, so that a tile's loads have one step, not two, to land.  Behind the last tile it is loaded again, to no use: with a
    // load left out, the wait for the one before could not be told from one for all loads.
    auto step_of = [&](auto set, auto other, int tile) {
        const int left = n - (begin + tile) * kKeys, ahead = std::min(tile + 3, tiles - 1);
        auto ask = [&] {
            load_keys(other, ahead);
            load_values(other, ahead);
        };
        store(other, left - kKeys);
        if (active) work(buffer[set], left < kKeys, left < kKeys ? (1ull << left) - 1ull : ~0ull, ask, [](const bf16x8 *) {});
        else ask();
        look_up(std::min(tile + 4, tiles - 1));
        __syncthreads();
    };
    if (tiles > 0) {
        store(even, n - begin * kKeys);
        // (the wait for the queries is here, not at their use in the loop, where it would be one for the tiles on their way, too)
#pragma unroll
        for (int p = 0; p < kSteps; ++p) asm volatile("" : "+v"(q[p]));
        load_keys(even, std::min(2, tiles - 1));
        load_values(even, std::min(2, tiles - 1));
        look_up(std::min(3, tiles - 1));
        __syncthreads();
        // (no way out between the two steps: it would look like one from the first step to itself, and its waits would be longer)
        int tile = 0;
        for (; tile + 1 < tiles; tile += 2) {
            step_of(even, odd, tile);
            step_of(odd, even, tile + 1);
        }
        if (tile < tiles) step_of(even, odd, tile);
    }
    __syncthreads();
    for (int start = 0; start < drafted; start += kKeys) {
        const int here = std::min(kKeys, drafted - start);
        load_new(start);
        bool fine = true;
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    fine = fine && (finite_pair(value[0][r][j][w]) || 4 * (quad + r * kQuads) + j >= here);
                    value[0][r][j][w] = finite_part(value[0][r][j][w]);
                }
        if (!fine) not_finite = start;
        store(even, here);
        __syncthreads();
        uint64_t sees = 0ull;
        if (t < count) {
            if (a.tree != nullptr) {
                sees = a.tree[((int64_t)b * a.tokens + t) * a.words + (start >> 6)] >> (start & 63);
            } else {
                const int upto = t - start;
                sees = upto >= 63 ? ~0ull : upto < 0 ? 0ull : (2ull << upto) - 1ull;
            }
            if (here < 64) sees &= (1ull << here) - 1ull;
        }
        if (active) work(buffer[0], true, sees, [] {}, [&](const bf16x8 *p) {
            if (not_finite != start) return;
            // elements that were left out, for the rows that see their token (the others must not meet them, not even with a weight
            // of zero)
            for (int j = 0; j < here; ++j) {
                // key j: element 4 (j / 8) + j % 4 of lane half (j / 4) & 1
                float own = 0.0f;
#pragma unroll
                for (int x = 0; x < kKeys / 2; ++x)
                    if (x == j / 8 * 4 + j % 4) own = (float)p[x / 8][x % 8];
                const float w = __shfl(own, (j >> 2 & 1) * 32 + i);
                if ((sees >> j & 1ull) == 0ull) continue;
                const __bf16 *at = reinterpret_cast<const __bf16 *>(a.v + b * a.v_batch + (start + j) * a.v_token + h * a.v_head);
#pragma unroll
                for (int m = 0; m < kBlocks; ++m)
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const float element = (float)at[32 * m + x / 4 * 8 + 4 * g + x % 4];
                        if (!(fabsf(element) < INFINITY)) o[m][x] += w * element;
                    }
            }
        });
        __syncthreads();
    }

    l += __shfl_xor(l, 32);
    if (row >= rows) return;
    const int64_t at = ((int64_t)b * a.tokens + t) * a.q_heads + head;
    if (a.splits > 1) {
        float *to = a.part_o + (at * a.splits + split) * kDim + 4 * g;
#pragma unroll
        for (int m = 0; m < kBlocks; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<f32x4 *>(to + 32 * m + 8 * e) = f32x4{o[m][4 * e], o[m][4 * e + 1], o[m][4 * e + 2], o[m][4 * e + 3]};
        if (g == 0) {
            a.part_ml[(at * a.splits + split) * 2] = most;
            a.part_ml[(at * a.splits + split) * 2 + 1] = l;
        }
    } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        const float inverse = inverse_sum(l);
        const bool counts = t < count;
        __bf16 *to = reinterpret_cast<__bf16 *>(a.out + b * a.o_batch + t * a.o_token + head * a.o_head) + 4 * g;
#pragma unroll
        for (int m = 0; m < kBlocks; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bf16x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = (__bf16)(counts ? o[m][4 * e + j] * inverse : 0.0f);
                *reinterpret_cast<bf16x4 *>(to + 32 * m + 8 * e) = x;
            }
        if (g == 0) a.lse[at] = counts ? logsumexp(most, l, a.c2) : -INFINITY;
    }
}

template <int kDim>
void launch(const AttendArgs &a, int waves, const dim3 grid, hipStream_t st)
{
    if (waves == 4) attend_wide_kernel<kDim, 4><<<grid, 256, 0, st>>>(a);
    if constexpr (kDim != 256) {
        if (waves == 8) attend_wide_kernel<kDim, 8><<<grid, 512, 0, st>>>(a);
    }
}

}  // namespace

void attend_wide(const AttendArgs &a, int waves, uint32_t workgroups, hipStream_t st)
{
    if (a.c.head_dim == 64) launch<64>(a, waves, dim3(workgroups), st);
    else if (a.c.head_dim == 128) launch<128>(a, waves, dim3(workgroups), st);
    else launch<256>(a, waves, dim3(workgroups), st);
}

}  // namespace fgmp
