// Attention of new tokens over a cache and over each other.
//
// The query heads that share a key head, for all new tokens of a sequence, are the rows of one product with that head's keys:
// row r = token * group + head of the group.  A wave holds 16 kRows of them in registers and walks over the keys in tiles, each
// wave tiles of its own, with the running maximum and sum of the softmax (one pass over keys and values):
//   S^T = K Q^T    a 16 x 16 tile of matrix instructions has keys along the registers and rows along the lanes, so that
//   O^T += V^T P^T takes the weights P from the registers they were computed in, with no exchange between lanes: the order of the keys
//                  in the k index of a matrix instruction is free, as long as both operands have the same.
// Lane l = 16 g + i then holds, of the weights, row i and keys 4 g .. 4 g + 3 of each 16, and of V the same keys and the
// elements d = n i .. n i + n - 1 (n = head_dim / 16): 16 lanes load a whole row of V, and BF16 values change places within the
// lane's registers (32 v_perm for 8 keys x 8 elements).  K is loaded in operand order: 16 rows x 64 bytes an instruction.
#include "fgmp_attention.hpp"

namespace fgmp {

namespace {

constexpr int kFewWaves = 4, kManyWaves = 8;   // of a workgroup
constexpr int kMaxTokens = 1024;

template <bool kF32>
struct Elem;
template <>
struct Elem<false> {
    static constexpr int kSize = 2, kKeys = 32;   // keys of a tile: one matrix instruction's k index in the second product
};
template <>
struct Elem<true> {
    static constexpr int kSize = 4, kKeys = 16;
};

// Keys (or queries) of 16 rows as an operand: lane 16 g + i holds row i, and of every 64 bytes of it the g-th 16.
template <bool kF32, int kDim>
struct Operand {
    static constexpr int kPieces = kDim * Elem<kF32>::kSize / 64;
    u32x4 x[kPieces];
    __device__ __forceinline__ void load(const char *row_and_lane)   // the lane's row + 16 g bytes
    {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) x[p] = *reinterpret_cast<const u32x4 *>(row_and_lane + 64 * p);
    }
    // in the order that keys of 8 bits have: of every 64 elements the g-th 16, in two pieces; the lane's row + 32 g bytes
    __device__ __forceinline__ void load_by_64(const char *row_and_lane)
    {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) x[p] = *reinterpret_cast<const u32x4 *>(row_and_lane + 128 * (p / 2) + 16 * (p % 2));
    }
};

// The same of keys in 8 bits: a load is 16 elements, which become two pieces of BF16 (exactly: a code has 4 bits, its scale is a power of two).
template <int kDim>
struct KeyCodes {
    u32x4 x[kDim / 64];
    uint32_t scale;
    __device__ __forceinline__ void load(const char *row_and_lane, const uint8_t *row_scale)
    {
#pragma unroll
        for (int p = 0; p < kDim / 64; ++p) x[p] = *reinterpret_cast<const u32x4 *>(row_and_lane + 64 * p);
        scale = *row_scale;
    }
    __device__ __forceinline__ Operand<false, kDim> values() const
    {
        Operand<false, kDim> k;
        const float s = scale_of(scale);
#pragma unroll
        for (int p = 0; p < kDim / 32; ++p)
#pragma unroll
            for (int w = 0; w < 4; ++w) k.x[p][w] = values_of(x[p / 2][2 * (p % 2) + w / 2], s, w % 2);
        return k;
    }
};

template <bool kF32, int kDim>
__device__ __forceinline__ f32x4 scores(const Operand<kF32, kDim> &a, const Operand<kF32, kDim> &b)
{
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < Operand<kF32, kDim>::kPieces; ++p) {
        if constexpr (kF32) {
            const f32x4 x = __builtin_bit_cast(f32x4, a.x[p]), y = __builtin_bit_cast(f32x4, b.x[p]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], s, 0, 0, 0);
        } else {
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.x[p]), __builtin_bit_cast(bf16x8, b.x[p]), s, 0, 0, 0);
        }
    }
    return s;
}

// Values of a tile's keys: lane 16 g + i holds elements n i .. n i + n - 1 of its 4 (FP32) or 8 (BF16) keys.
template <bool kF32, int kDim>
struct Values {
    static constexpr int kPer = kDim / 16, kLaneKeys = kF32 ? 4 : 8, kWords = kPer * Elem<kF32>::kSize / 4;
    uint32_t x[kLaneKeys][kWords];
    __device__ __forceinline__ void load(int key, const char *at)
    {
        if constexpr (kWords == 2) {
            const u32x2 t = *reinterpret_cast<const u32x2 *>(at);
            x[key][0] = t[0], x[key][1] = t[1];
        } else {
#pragma unroll
            for (int p = 0; p < kWords / 4; ++p) {
                const u32x4 t = *reinterpret_cast<const u32x4 *>(at + 16 * p);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[key][4 * p + e] = t[e];
            }
        }
    }
    __device__ __forceinline__ void clear(int key)
    {
#pragma unroll
        for (int w = 0; w < kWords; ++w) x[key][w] = 0u;
    }
    static __device__ __forceinline__ bool finite(uint32_t w)
    {
        return kF32 ? (w & 0x7F800000u) != 0x7F800000u : (w & 0x7F800000u) != 0x7F800000u && (w & 0x7F80u) != 0x7F80u;
    }
    __device__ __forceinline__ bool all_finite() const
    {
        bool fine = true;
#pragma unroll
        for (int j = 0; j < kLaneKeys; ++j)
#pragma unroll
            for (int w = 0; w < kWords; ++w) fine = fine && finite(x[j][w]);
        return fine;
    }
    // zeros in place of elements that are not finite
    __device__ __forceinline__ void clear_non_finite()
    {
#pragma unroll
        for (int j = 0; j < kLaneKeys; ++j)
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                const uint32_t t = x[j][w];
                if constexpr (kF32) x[j][w] = finite(t) ? t : 0u;
                else x[j][w] = ((t & 0x7F80u) != 0x7F80u ? t & 0xFFFFu : 0u) | ((t & 0x7F800000u) != 0x7F800000u ? t & 0xFFFF0000u : 0u);
            }
    }
    // the m-th element of all the lane's keys, as the operand of the second product
    __device__ __forceinline__ bf16x8 column(int m) const
    {
        u32x4 t;
#pragma unroll
        for (int p = 0; p < 4; ++p)
            t[p] = __builtin_amdgcn_perm(x[2 * p + 1][m / 2], x[2 * p][m / 2], (m & 1) != 0 ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(bf16x8, t);
    }
};

// The same of values in 8 bits: lane 16 g + i holds elements n i .. n i + n - 1 of keys 4 g .. 4 g + 3 of each 16, whose scales are a word.
template <int kDim>
struct ValueCodes {
    static constexpr int kWords = kDim / 64;
    uint32_t x[8][kWords], scale[2];
    __device__ __forceinline__ void load(int key, const char *at)
    {
        if constexpr (kWords == 1) {
            x[key][0] = *reinterpret_cast<const uint32_t *>(at);
        } else if constexpr (kWords == 2) {
            const u32x2 t = *reinterpret_cast<const u32x2 *>(at);
            x[key][0] = t[0], x[key][1] = t[1];
        } else {
            const u32x4 t = *reinterpret_cast<const u32x4 *>(at);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[key][e] = t[e];
        }
    }
    __device__ __forceinline__ void values(Values<false, kDim> &v) const
    {
#pragma unroll
        for (int key = 0; key < 8; ++key) {
            const float s = scale_of(scale[key / 4] >> (8 * (key % 4)) & 0xFFu);
#pragma unroll
            for (int w = 0; w < 2 * kWords; ++w) v.x[key][w] = values_of(x[key][w / 2], s, w % 2);
        }
    }
};

// Online softmax state and results of 16 rows: lane 16 g + i has row i; o[m][j] is element n (4 g + j) + m.
template <int kDim>
struct RowState {
    float m, l;   // maximum (of unscaled scores), sum of the weights (of the lane's keys)
    f32x4 o[kDim / 16];
};

// Over the four lanes of a row (lanes apart by 16), the same in all of them: halves of the wave change places, then rows of 16 lanes.
__device__ __forceinline__ float over_groups_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    x = fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    const auto q = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)q[0]), __builtin_bit_cast(float, (uint32_t)q[1]));
}
__device__ __forceinline__ float over_groups_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    x = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    const auto q = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return __builtin_bit_cast(float, (uint32_t)q[0]) + __builtin_bit_cast(float, (uint32_t)q[1]);
}

// The softmax of one tile: s[sub][j] are the lane's scores (masked ones -inf); p: the weights as the operand of the second product,
// relative to st.m, the maximum until it is exceeded by a
// factor of 2^kSlack: then the state is scaled to the new one.
template <bool kF32, int kDim>
struct Weights;
template <int kDim>
struct Weights<false, kDim> { bf16x8 p; };
template <int kDim>
struct Weights<true, kDim> { float p[4]; };

template <bool kF32, int kDim>
__device__ __forceinline__ void weigh(RowState<kDim> &st, const f32x4 *s, Weights<kF32, kDim> &w, float c2)
{
    constexpr int kSubs = kF32 ? 1 : 2, kPer = kDim / 16;
    float most = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
    if constexpr (kSubs == 2) most = fmaxf(most, fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    most = fmaxf(over_groups_max(most), st.m);
    // (-inf - -inf is not above it: nothing has been seen yet)
    const bool above = (most - st.m) * c2 > kSlack;
    if (__any(above)) {
        // each row for itself: what a row gets must not depend on the rows it shares a wave with
        const float alpha = !above ? 1.0f : st.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((st.m - most) * c2);
        st.m = above ? most : st.m;
        st.l *= alpha;
#pragma unroll
        for (int m = 0; m < kPer; ++m) st.o[m] *= alpha;
    }
    const float base = st.m == -INFINITY ? 0.0f : st.m * c2;
    float p[4 * kSubs];
#pragma unroll
    for (int i = 0; i < 4 * kSubs; ++i) {
        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], c2, -base));
        st.l += p[i];
    }
    if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w.p[i] = p[i];
    } else {
        // (BF16 is what the matrix instruction takes.  A weight is off by up to 2^-8 of itself, in either direction, and their sum is of the
        // unrounded ones; results' errors against 64 bits are 0.0017 of their size with these weights and with FP32 ones, which is
        // what their own rounding to BF16 makes)
#pragma unroll
        for (int i = 0; i < 8; ++i) w.p[i] = (__bf16)p[i];
    }
}

template <bool kF32, int kDim>
__device__ __forceinline__ void add_values(RowState<kDim> &st, const Weights<kF32, kDim> &w, const Values<kF32, kDim> &v, const bf16x8 *columns)
{
#pragma unroll
    for (int m = 0; m < kDim / 16; ++m) {
        if constexpr (kF32) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                st.o[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, v.x[j][m]), w.p[j], st.o[m], 0, 0, 0);
        } else {
            st.o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(columns[m], w.p, st.o[m], 0, 0, 0);
        }
    }
}

// What add_values() left out of a tile of new tokens: elements of V that are not finite, which rows that do not see their token must
// not meet, not even with a weight of zero.  `v` points at the tile's first token.
template <bool kF32, int kDim>
__device__ __forceinline__ void add_non_finite(RowState<kDim> &st, const f32x4 *s, uint32_t sees, const char *v, int64_t v_token, int keys, float c2)
{
    constexpr int kPer = kDim / 16;
    const int lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    const float base = st.m == -INFINITY ? 0.0f : st.m * c2;
    for (int key = 0; key < keys; ++key) {
        const f32x4 mine = kF32 || key < 16 ? s[0] : s[1];
        const float own = key % 4 == 0 ? mine[0] : key % 4 == 1 ? mine[1] : key % 4 == 2 ? mine[2] : mine[3];
        float p = __builtin_amdgcn_exp2f(__builtin_fmaf(__shfl(own, key % 16 / 4 * 16 + i), c2, -base));
        if (!kF32) p = (float)(__bf16)p;
        if ((sees >> key & 1u) == 0u) continue;
        const char *at = v + key * v_token;
#pragma unroll
        for (int m = 0; m < kPer; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = kPer * (4 * g + j) + m;
                const float x = kF32 ? reinterpret_cast<const float *>(at)[d] : (float)reinterpret_cast<const __bf16 *>(at)[d];
                if (!(fabsf(x) < INFINITY)) st.o[m][j] += p * x;
            }
    }
}

// kRows: groups of 16 rows that a workgroup's waves hold, every wave all of them.  A tile of keys and values is asked for while the one
// before is worked on: the keys as soon as its scores are there, the values as soon as they have changed places.
// kEight: a cache in 8 bits, all else BF16; codes become BF16 when their tile is worked on.
template <bool kF32, int kDim, int kRows, bool kEight = false, int kWaves = kFewWaves>
__global__ void __launch_bounds__(64 * kWaves, kRows > 1 ? 2 : 1) attend_kernel(ArgsOf<kEight> a)
{
    static_assert(!(kF32 && kEight), "new tokens, results and weights are BF16 where the cache is in 8 bits");
    constexpr int kSize = Elem<kF32>::kSize, kKeys = Elem<kF32>::kKeys, kSubs = kKeys / 16, kPer = kDim / 16;
    constexpr int kLaneKeys = Values<kF32, kDim>::kLaneKeys;
    __shared__ float merge_o[kWaves][kRows * kPer * 4 * 64];
    __shared__ float merge_ml[kWaves][kRows][2][16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, i = lane & 15;
    const AttendPlace place(a);
    if (!place.there) return;
    const int split = place.split, block = place.block, h = place.h, b = place.b;

    const int32_t n = a.c.length(b), count = a.count(b);
    const int rows = a.tokens * a.group, first = block * (16 * kRows);
    const bool empty = first >= count * a.group;         // no row of this block belongs to a token that counts
    if (empty && a.splits > 1) return;                   // (written by the launch that joins the ranges)
    const int drafted = a.k != nullptr ? count : 0;

    // this workgroup's tiles; the new tokens' go with the last range
    const int per = a.range(n), used = a.ranges(n);
    if (split >= used) return;
    const int end = std::min(a.tiles(n), (split + 1) * per);
    const int draft_tiles = split == used - 1 ? (drafted + kKeys - 1) / kKeys : 0;

    Operand<kF32, kDim> kt[kSubs];
    Values<kF32, kDim> vt;
    KeyCodes<kDim> kc[kSubs];                            // (kEight)
    ValueCodes<kDim> vc;
    const uint32_t dv = i * kPer * (kEight ? 1 : kSize);
    const uint8_t *k_scale_at[kSubs], *v_scale_at[kSubs];
    const uint32_t step = (uint32_t)a.c.token_stride;    // (16 rows: less than 2^32 bytes)
    const char *k_at[kSubs], *v_at[kSubs];               // of the tile to be loaded next
    auto locate = [&](int tile) {
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) {
            // (the group of slots behind the last one in use may have no page: read as the one in use)
            if constexpr (kEight) {
                uint32_t row;
                const uint32_t entry = a.c.entry_of((uint32_t)std::min(kSubs * tile + sub, (n - 1) / 16), &row), page = a.c.page_of(b, entry);
                const int64_t at = a.c.offset(page, row, h), scale = a.scale_at(page, row, h);
                k_at[sub] = a.c.k + at;
                v_at[sub] = a.c.v + at;
                k_scale_at[sub] = a.k_scales + scale;
                v_scale_at[sub] = a.v_scales + scale;
                continue;
            }
            const int64_t at = a.c.group_offset(b, (uint32_t)std::min(kSubs * tile + sub, (n - 1) / 16), h);
            k_at[sub] = a.c.k + at;
            v_at[sub] = a.c.v + at;
        }
    };
    auto load_key = [&](int sub, int row) {
        if constexpr (kEight) kc[sub].load(k_at[sub] + ((uint32_t)row * step + 16u * g), k_scale_at[sub] + (uint32_t)row);
        else kt[sub].load(k_at[sub] + ((uint32_t)row * step + 16u * g));
    };
    auto load_value = [&](int sub, int j, int row) {
        if constexpr (kEight) vc.load(4 * sub + j, v_at[sub] + ((uint32_t)row * step + dv));
        else vt.load(4 * sub + j, v_at[sub] + ((uint32_t)row * step + dv));
    };
    // rows behind the last slot in use are read as the last one
    auto load_keys = [&](int tile) {
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) {
            if ((tile + 1) * kKeys <= n) {
                load_key(sub, i);
            } else {
                const int last = std::min(15, n - 1 - 16 * std::min(kSubs * tile + sub, (n - 1) / 16));
                load_key(sub, std::min(i, last));
            }
        }
    };
    auto load_values = [&](int tile) {
#pragma unroll
        for (int sub = 0; sub < kSubs; ++sub) {
            if ((tile + 1) * kKeys <= n) {
#pragma unroll
                for (int j = 0; j < 4; ++j) load_value(sub, j, 4 * g + j);
            } else {
                const int last = std::min(15, n - 1 - 16 * std::min(kSubs * tile + sub, (n - 1) / 16));
#pragma unroll
                for (int j = 0; j < 4; ++j) load_value(sub, j, std::min(4 * g + j, last));
            }
            // (of slots behind the last one the scales may be anything: their values are cleared)
            if constexpr (kEight) vc.scale[sub] = *reinterpret_cast<const uint32_t *>(v_scale_at[sub] + 4 * g);
        }
    };

    const int begin = empty ? end : split * per + wave;
    if (begin < end) {
        locate(begin);
        load_keys(begin);
        load_values(begin);
    }
    int token[kRows];
    Operand<kF32, kDim> q[kRows];
    RowState<kDim> st[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int row = first + 16 * r + i, t = row / a.group;
        token[r] = t < count ? t : -1;                   // (no row: sees nothing)
        const int at = row < rows ? t : 0, head = h * a.group + (row < rows ? row - t * a.group : 0);
        if constexpr (kEight) q[r].load_by_64(a.q + b * a.q_batch + at * a.q_token + head * a.q_head + 32 * g);
        else q[r].load(a.q + b * a.q_batch + at * a.q_token + head * a.q_head + 16 * g);
        st[r].m = -INFINITY;
        st[r].l = 0.0f;
#pragma unroll
        for (int m = 0; m < kPer; ++m) st[r].o[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto new_tokens = [&] {
        // (the first of them to the wave behind the one that had the last tile of the range)
        for (int tile = empty ? draft_tiles : (wave + kWaves - (end - split * per) % kWaves) % kWaves; tile < draft_tiles; tile += kWaves) {
            const int start = tile * kKeys, last = drafted - 1 - start;
#pragma unroll
            for (int sub = 0; sub < kSubs; ++sub) {
                const char *const key = a.k + b * a.k_batch + (start + std::min(16 * sub + i, last)) * a.k_token + h * a.k_head;
                if constexpr (kEight) kt[sub].load_by_64(key + 32 * g);
                else kt[sub].load(key + 16 * g);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    vt.load(4 * sub + j, a.v + b * a.v_batch + (start + std::min(16 * sub + 4 * g + j, last)) * a.v_token + h * a.v_head + i * kPer * kSize);
            }
#pragma unroll
            for (int j = 0; j < kLaneKeys; ++j)
                if (16 * (j / 4) + 4 * g + j % 4 > last) vt.clear(j);
            const bool finite = __all(vt.all_finite());
            if (!finite) vt.clear_non_finite();
            bf16x8 columns[kPer];
            if constexpr (!kF32) {
#pragma unroll
                for (int m = 0; m < kPer; ++m) columns[m] = vt.column(m);
            }
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                // bit j: the lane's row sees new token start + j
                uint32_t sees = 0u;
                if (token[r] >= 0) {
                    if (a.tree != nullptr) {
                        const uint64_t word = a.tree[((int64_t)b * a.tokens + token[r]) * a.words + (start >> 6)];
                        sees = (uint32_t)(word >> (start & 63));
                    } else {
                        const int upto = token[r] - start;
                        sees = upto >= 31 ? 0xFFFFFFFFu : upto < 0 ? 0u : (2u << upto) - 1u;
                    }
                    if (last < 31) sees &= (2u << last) - 1u;
                }
                f32x4 s[kSubs];
#pragma unroll
                for (int sub = 0; sub < kSubs; ++sub) {
                    s[sub] = scores<kF32, kDim>(kt[sub], q[r]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if ((sees >> (16 * sub + 4 * g + j) & 1u) == 0u) s[sub][j] = -INFINITY;
                }
                Weights<kF32, kDim> w;
                weigh<kF32, kDim>(st[r], s, w, a.c2);
                add_values<kF32, kDim>(st[r], w, vt, columns);
                if (!finite)
                    add_non_finite<kF32, kDim>(st[r], s, sees, a.v + b * a.v_batch + start * a.v_token + h * a.v_head, a.v_token,
                                               std::min(kKeys, last + 1), a.c2);
            }
        }
    };
    // (over a short cache in 8 bits they come first: their loads and the first tile's, which has registers of its own, are waited for together.  8 x 8 heads of 1024 slots 14.8 ->
    // 13.6 us; with head_dim 64, and with four waves over 2048 and 4096 slots, it is 0.2 to 1 slower)
    constexpr bool kNewFirst = kEight && kWaves == kManyWaves && kDim == 128;
    if constexpr (kNewFirst) new_tokens();

    for (int tile = begin; tile < end; tile += kWaves) {
        const int next = tile + kWaves, left = n - tile * kKeys;
        if (next < end) locate(next);
        f32x4 s[kRows][kSubs];
        if constexpr (kEight) {
#pragma unroll
            for (int sub = 0; sub < kSubs; ++sub) kt[sub] = kc[sub].values();
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int sub = 0; sub < kSubs; ++sub) s[r][sub] = scores<kF32, kDim>(kt[sub], q[r]);
        if (next < end) load_keys(next);
        if constexpr (kEight) {
            vc.values(vt);
            if (next < end) load_values(next);
        }
        if (left < kKeys) {
            // what lies behind the sequence must not meet a weight of zero: it might not be finite
#pragma unroll
            for (int j = 0; j < kLaneKeys; ++j) {
                if (16 * (j / 4) + 4 * g + j % 4 < left) continue;
                vt.clear(j);
#pragma unroll
                for (int r = 0; r < kRows; ++r) s[r][j / 4][j % 4] = -INFINITY;
            }
        }
        Weights<kF32, kDim> w[kRows];
        if constexpr (kF32) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) weigh<kF32, kDim>(st[r], s[r], w[r], a.c2);
#pragma unroll
            for (int r = 0; r < kRows; ++r) add_values<kF32, kDim>(st[r], w[r], vt, nullptr);
            if (next < end) load_values(next);
        } else if constexpr (kRows > 1) {
            // (no registers for the values in both orders)
#pragma unroll
            for (int r = 0; r < kRows; ++r) weigh<kF32, kDim>(st[r], s[r], w[r], a.c2);
#pragma unroll
            for (int m = 0; m < kPer; ++m) {
                const bf16x8 column = vt.column(m);
#pragma unroll
                for (int r = 0; r < kRows; ++r) st[r].o[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(column, w[r].p, st[r].o[m], 0, 0, 0);
            }
            if (!kEight && next < end) load_values(next);
        } else {
            bf16x8 columns[kPer];
#pragma unroll
            for (int m = 0; m < kPer; ++m) columns[m] = vt.column(m);
            if (!kEight && next < end) load_values(next);
#pragma unroll
            for (int r = 0; r < kRows; ++r) weigh<kF32, kDim>(st[r], s[r], w[r], a.c2);
#pragma unroll
            for (int r = 0; r < kRows; ++r) add_values<kF32, kDim>(st[r], w[r], vt, columns);
        }
    }
    if constexpr (!kNewFirst) new_tokens();

    // join the waves: every one holds all rows over keys of its own
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const float l = over_groups_sum(st[r].l);
        if (g == 0) {
            merge_ml[wave][r][0][i] = st[r].m;
            merge_ml[wave][r][1][i] = l;
        }
#pragma unroll
        for (int m = 0; m < kPer; ++m)
            *reinterpret_cast<f32x4 *>(&merge_o[wave][((r * kPer + m) * 64 + lane) * 4]) = st[r].o[m];
    }
    __syncthreads();
    // wave w adds up elements m = w, w + 4, ... of each lane's rows
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int row = first + 16 * r + i;
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, merge_ml[w][r][0][i]);
        float f[kWaves], l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float m = merge_ml[w][r][0][i];
            f[w] = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - most) * a.c2);
            l += merge_ml[w][r][1][i] * f[w];
        }
        const int t = row / a.group, head = h * a.group + row - t * a.group;
        const int64_t at = ((int64_t)b * a.tokens + t) * a.q_heads + head;   // (of rows that exist)
        const float inverse = inverse_sum(l);
#pragma unroll
        for (int m4 = 0; m4 < (kPer + kWaves - 1) / kWaves; ++m4) {
            const int m = kPer < kWaves ? wave : wave * (kPer / kWaves) + m4;
            if (kPer < kWaves && wave >= kPer) continue;
            f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) o += *reinterpret_cast<const f32x4 *>(&merge_o[w][((r * kPer + m) * 64 + lane) * 4]) * f[w];
            if (row < rows) {
                if (a.splits > 1) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) a.part_o[(at * a.splits + split) * kDim + kPer * (4 * g + j) + m] = o[j];
                } else {
                    char *to = a.out + b * a.o_batch + t * a.o_token + head * a.o_head;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int d = kPer * (4 * g + j) + m;
                        const float x = t < count ? o[j] * inverse : 0.0f;
                        if constexpr (kF32) reinterpret_cast<float *>(to)[d] = x;
                        else reinterpret_cast<__bf16 *>(to)[d] = (__bf16)x;
                    }
                }
            }
        }
        if (wave == 0 && g == 0 && row < rows) {
            if (a.splits > 1) {
                float *ml = a.part_ml + (at * a.splits + split) * 2;
                ml[0] = most;
                ml[1] = l;
            } else {
                a.lse[at] = t < count ? logsumexp(most, l, a.c2) : -INFINITY;
            }
        }
    }
}

// Over rows of 16 lanes, the same in all of them: neighbours, then pairs, quads, eights.
template <typename Op>
__device__ __forceinline__ float over_16(float x, Op op)
{
    auto step = [&](auto control) {
        x = op(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(control)::value, 0xF, 0xF, true)));
    };
    step(std::integral_constant<int, 0xB1>());    // lane ^ 1
    step(std::integral_constant<int, 0x4E>());    // lane ^ 2
    step(std::integral_constant<int, 0x141>());   // 7 - lane of eight
    step(std::integral_constant<int, 0x140>());   // 15 - lane of a row
    return x;
}

template <int kN>
struct FloatsOf {
    typedef float type __attribute__((ext_vector_type(kN)));
};

template <bool kF32, int kN>
__device__ __forceinline__ void store_joined(char *to, int lane, typename FloatsOf<kN>::type o)
{
#pragma unroll
    for (int e = 0; e < kN; ++e) {
        if constexpr (kF32) reinterpret_cast<float *>(to)[lane * kN + e] = o[e];
        else reinterpret_cast<__bf16 *>(to)[lane * kN + e] = (__bf16)o[e];
    }
}

// Joins up to kFewRanges ranges of keys: kDim / 4 lanes have a row, 16 of them each the maximum and sum of a range.  What the first four ranges hold is
// asked for before it is known how many are in use: one trip to memory for all
// (12800 rows of 4 ranges, head_dim 128: 7.4 us, 9.2 with a wave to a row that asks for ranges in use; four waves to a row had hardly anything to do, 20).
constexpr int kFewRanges = 16;
template <bool kF32, int kDim>
__global__ void __launch_bounds__(256) join_few_kernel(AttendArgs a, uint32_t rows)
{
    constexpr int kLanes = kDim / 4, kRowsHere = 256 / kLanes, kAtATime = 4;
    const int lane = threadIdx.x % kLanes, range = threadIdx.x % kFewRanges, first_lane = (threadIdx.x & 63) / kLanes * kLanes;
    const uint32_t place = blockIdx.x * kRowsHere + threadIdx.x / kLanes, at = std::min(place, rows - 1u);
    const f32x4 *po = reinterpret_cast<const f32x4 *>(a.part_o + (int64_t)at * a.splits * kDim) + lane;
    f32x4 x[kAtATime];
    auto load = [&](int from) {
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) x[j] = po[std::min(from + j, a.splits - 1) * kLanes];
    };
    load(0);
    const float2 ml = reinterpret_cast<const float2 *>(a.part_ml)[(int64_t)at * a.splits + std::min(range, a.splits - 1)];
    const int head = (int)(at % (uint32_t)a.q_heads);
    const uint32_t bt = at / (uint32_t)a.q_heads;
    const int t = (int)(bt % (uint32_t)a.tokens), b = (int)(bt / (uint32_t)a.tokens);
    const int used = t < a.count(b) ? a.ranges(a.c.length(b)) : 0;
    const float m = range < used ? ml.x : -INFINITY, most = over_16(m, [](float p, float q) { return fmaxf(p, q); });
    const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - most) * a.c2);
    const float l = over_16(range < used ? ml.y * f : 0.0f, [](float p, float q) { return p + q; });
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int first = 0; first < a.splits; first += kAtATime) {
        if (first > 0) load(first);
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) {
            const float factor = __shfl(f, first_lane + first + j);
            if (first + j < used) o += x[j] * factor;
        }
    }
    if (place >= rows) return;
    o *= inverse_sum(l);
    store_joined<kF32, 4>(a.out + b * a.o_batch + t * a.o_token + head * a.o_head, lane, o);
    if (lane == 0) a.lse[at] = logsumexp(most, l, a.c2);
}

// Joins more of them, a workgroup to a row: a lane holds the maximum and sum of one range (of every 64), and each wave adds up every fourth
// range, the first of them asked for before it is known how many are in use (128 rows of 32 ranges: 4.8 us, 5.2 asked for later; 64 rows of 64 took one wave a
// row 36 us, four 7).
template <bool kF32, int kDim>
__global__ void __launch_bounds__(256) join_many_kernel(AttendArgs a)
{
    constexpr int kPer = kDim / 64, kWavesPerRow = 4, kAtATime = 8;
    using part = typename FloatsOf<kPer>::type;
    __shared__ part sums[kWavesPerRow][64];
    const int lane = threadIdx.x & 63, share = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t at = blockIdx.x;
    const part *po = reinterpret_cast<const part *>(a.part_o + (int64_t)at * a.splits * kDim) + lane;
    part x[kAtATime];
    auto load = [&](int from) {
#pragma unroll
        for (int j = 0; j < kAtATime; ++j) x[j] = po[std::min(from + kWavesPerRow * j, a.splits - 1) * 64];
    };
    load(share);
    const float *ml = a.part_ml + (int64_t)at * a.splits * 2;
    const int head = (int)(at % (uint32_t)a.q_heads);
    const uint32_t bt = at / (uint32_t)a.q_heads;
    const int t = (int)(bt % (uint32_t)a.tokens), b = (int)(bt / (uint32_t)a.tokens);
    const int used = t < a.count(b) ? a.ranges(a.c.length(b)) : 0;
    float most = -INFINITY;
    for (int s = lane; s < used; s += 64) most = fmaxf(most, ml[2 * s]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    float l = 0.0f;
    part o = {};
    for (int start = 0; start < used; start += 64) {
        float f = 0.0f;
        if (start + lane < used) {
            const float m = ml[2 * (start + lane)];
            f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - most) * a.c2);
            l += ml[2 * (start + lane) + 1] * f;
        }
        const int here = std::min(64, used - start);
        for (int first = share; first < here; first += kAtATime * kWavesPerRow) {
            if (start + first > share) load(start + first);
#pragma unroll
            for (int j = 0; j < kAtATime; ++j) {
                const float factor = __shfl(f, first + kWavesPerRow * j);
                if (first + kWavesPerRow * j < here) o += x[j] * factor;
            }
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
    sums[share][lane] = o;
    __syncthreads();
    if (share != 0) return;
    o = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    o *= inverse_sum(l);
    store_joined<kF32, kPer>(a.out + b * a.o_batch + t * a.o_token + head * a.o_head, lane, o);
    if (lane == 0) a.lse[at] = logsumexp(most, l, a.c2);
}

// ---- attention weights of accepted tokens ----
//
// The first product alone, S = Q K^T, with rows along the registers: the sum over rows is then within a lane, but for its last
// step over the four lane groups.  A wave holds 16 kWeightKeys keys in registers, asks for its next ones, and walks over the accepted rows,
// which the workgroup stages in LDS in operand order: once where they are no more than kStage, for every block of keys else.  No sum is
// shared between waves: the order of additions is fixed.

// Workgroups asked for, more than the chip holds at a time (1280 or 1024 with head_dim 64, 1024 with 128, 512 with 256; FP32 512 with 128, 256 with
// 256): 2 x 8 heads of 65537 slots, at 256 / 512 / 1024 / 2048: BF16 57 / 38 / 29 / 30 us with head_dim 64, 78 / 64 / 58 / 54 with 128, 112 / 102 / 104 / 115
// with 256; FP32 83 / 65 / 58 / 56, 124 / 104 / 107 / 123, 200 / 204 / 215 / 256.
constexpr int kWeightKeys = 2, kStage = 64, kWeightWorkgroups = 2048;

struct WeightArgs {
    CacheView c;
    const char *q;
    const float *lse;
    int64_t q_batch, q_token, q_head;   // bytes
    const int32_t *rows, *counts;
    int32_t tokens, accepted, q_heads, group, blocks;
    float c2;
    const float *weights;
    float *out;
    int64_t stride;
};

template <bool kF32, int kDim>
__global__ void __launch_bounds__(64 * kFewWaves) weights_kernel(WeightArgs a)
{
    constexpr int kPieces = Operand<kF32, kDim>::kPieces, kBlock = 16 * kWeightKeys * kFewWaves;
    __shared__ u32x4 stage[kStage / 16][kPieces][64];
    __shared__ float stage_lse[kStage];   // log2 of the row's sum; +inf: a row that adds nothing
    __shared__ int32_t stage_end[kStage]; // slots that the row sees
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x;
    const int g = lane >> 4, i = lane & 15;
    uint32_t id = blockIdx.x;
    const int block = id % a.blocks;
    id /= a.blocks;
    const int h = id % a.c.heads, b = id / a.c.heads;
    const int32_t n = a.c.length(b);
    int32_t count = a.counts != nullptr ? a.counts[b] : a.accepted;
    count = count < 0 ? 0 : count > a.accepted ? a.accepted : count;
    const int rows = count * a.group;
    // rows start .. start + kStage - 1; of those that there are not, whole groups of 16 are left as they are
    auto put = [&](int start) {
        for (int p = tid; p < kStage / 16 * kPieces * 64; p += 64 * kFewWaves) {
            if (start + p / (kPieces * 64) * 16 >= rows) break;
            const int r = start + p / (kPieces * 64) * 16 + (p & 15);
            u32x4 x = {0u, 0u, 0u, 0u};
            if (r < rows) {
                const int t = r / a.group, row = a.rows != nullptr ? a.rows[b * (int64_t)a.accepted + t] : t;
                if ((uint32_t)row < (uint32_t)a.tokens)
                    x = *reinterpret_cast<const u32x4 *>(a.q + b * a.q_batch + row * a.q_token + (h * a.group + r - t * a.group) * a.q_head +
                                                         p / 64 % kPieces * 64 + (p / 16 & 3) * 16);
            }
            stage[p / (kPieces * 64)][p / 64 % kPieces][p & 63] = x;
        }
        if (tid < kStage) {
            const int r = start + tid, t = r / a.group;
            float lse = INFINITY;
            if (r < rows) {
                const int row = a.rows != nullptr ? a.rows[b * (int64_t)a.accepted + t] : t;
                if ((uint32_t)row < (uint32_t)a.tokens) lse = a.lse[((int64_t)b * a.tokens + row) * a.q_heads + h * a.group + r - t * a.group] * kLog2e;
                if (lse == -INFINITY) lse = INFINITY;   // (a row that saw nothing has no weights)
            }
            stage_lse[tid] = lse;
            stage_end[tid] = n - count + t + 1;
        }
    };
    auto load = [&](int first, Operand<kF32, kDim> *k) {
#pragma unroll
        for (int s = 0; s < kWeightKeys; ++s) {
            const int u = std::min(first / 16 + wave * kWeightKeys + s, (n - 1) / 16), last = std::min(15, n - 1 - 16 * u);
            k[s].load(a.c.k + a.c.group_offset(b, (uint32_t)u, h) + ((uint32_t)std::min(i, last) * (uint32_t)a.c.token_stride + 16u * g));
        }
    };
    const bool once = rows <= kStage;
    Operand<kF32, kDim> kt[kWeightKeys];
    if (block * kBlock < n) load(block * kBlock, kt);
    if (once) {
        put(0);
        __syncthreads();
    }
    for (int first = block * kBlock; first < n; first += a.blocks * kBlock) {
        const int mine = first + wave * 16 * kWeightKeys, next = first + a.blocks * kBlock;
        Operand<kF32, kDim> ahead[kWeightKeys];
        if (next < n) load(next, ahead);
        // (what the slots have is on its way meanwhile, too)
        const int64_t at = ((int64_t)b * a.c.heads + h) * a.stride + mine + i;
        float have[kWeightKeys], sum[kWeightKeys] = {};
#pragma unroll
        for (int s = 0; s < kWeightKeys; ++s) have[s] = g == 0 && mine + 16 * s + i < n ? a.weights[at + 16 * s] : 0.0f;
        for (int start = 0; start < rows; start += kStage) {
            if (!once) {
                __syncthreads();
                put(start);
                __syncthreads();
            }
#pragma unroll 1
            for (int r = 0; r < kStage / 16 && start + 16 * r < rows; ++r) {
                Operand<kF32, kDim> q;
#pragma unroll
                for (int p = 0; p < kPieces; ++p) q.x[p] = stage[r][p][lane];
                const f32x4 lse = *reinterpret_cast<const f32x4 *>(&stage_lse[16 * r + 4 * g]);
                const int4 ends = *reinterpret_cast<const int4 *>(&stage_end[16 * r + 4 * g]);
#pragma unroll
                for (int s = 0; s < kWeightKeys; ++s) {
                    const f32x4 x = scores<kF32, kDim>(q, kt[s]);
                    const int slot = mine + 16 * s + i;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], a.c2, -lse[j]));
                        sum[s] += slot < (j == 0 ? ends.x : j == 1 ? ends.y : j == 2 ? ends.z : ends.w) && lse[j] != INFINITY ? w : 0.0f;
                    }
                }
            }
        }
#pragma unroll
        for (int s = 0; s < kWeightKeys; ++s) {
            const float total = over_groups_sum(sum[s]);
            if (g == 0 && mine + 16 * s + i < n) a.out[at + 16 * s] = have[s] + total;
        }
#pragma unroll
        for (int s = 0; s < kWeightKeys; ++s) kt[s] = ahead[s];
    }
}

// How a call is shared out.  Up to 32 rows (16 with head_dim 256), and in FP32, a workgroup's waves all have the same rows; those of the kernel
// for many rows have 32 each.  The one / the other, 4 x 4 heads of 30000 slots: head_dim 128, 32 rows 61 / 67 us, 40 rows 71 / 69, 80 rows 100 / 73; head_dim
// 256, 16 rows 110 / 134, 32 rows 135 / 135, 40 rows 189 / 132 (8 x 8 heads of 5000: 32 rows 105 / 96); head_dim 64, 32 rows 30 / 29, 80 rows 57 / 34.
struct AttendPlan {
    int waves_of_rows;      // of the kernel for many rows; 0: the other one
    int row_groups;         // groups of 16 rows, of the other one
    int waves;              // of a workgroup of the other one
    int tile_keys, min_tiles;
    int64_t row_blocks, splits;
    int64_t units, workgroups;   // ranges of all heads and sequences; in eights, and for each row block
};

AttendPlan attend_plan(int64_t batch, int64_t tokens, int64_t q_heads, int64_t heads, int64_t head_dim, bool f32, int64_t max_length, bool eight = false)
{
    AttendPlan p = {};
    const int64_t groups = (tokens * (q_heads / heads) + 15) / 16;
    int64_t want;   // workgroups asked for, by making ranges
    // The kernel for many rows begins with three groups (two with head_dim 256).  Over a short cache in 8 bits it is not worth its stages below five: one sequence of 1000
    // slots, 8 heads, three groups, with it / without: 13.3 / 12.1 us with head_dim 64, 18.0 / 15.9 with 128, 16 of 1500 23.9 / 22.3 and 35.1 / 32.4, 3 of 4000 24.0 / 23.2
    // and 33.8 / 33.4, 2 of 30000 32.5 / 36.4 and 53.0 / 58.7; 4 heads of 256: one of 1000 24.7 / 17.7, 3 of 4000 49.5 / 39.4, 16 of 1500 42.7 / 51.6, 2 of 30000 85 / 127.
    const bool few = eight && groups <= 4 && (head_dim == 256 ? max_length <= 4096 && batch * heads * groups < 128 : max_length <= 2048);
    if (!f32 && !few && groups > (head_dim == 256 ? 1 : 2)) {
        p.waves_of_rows = groups <= 8 || head_dim == 256 ? 4 : 8;
        p.row_blocks = (groups + 2 * p.waves_of_rows - 1) / (2 * p.waves_of_rows);
        p.tile_keys = wide_keys((int)head_dim);
        p.min_tiles = 128 / p.tile_keys;
        want = p.waves_of_rows == 8 || head_dim == 256 ? 256 : 512;   // (as many as the chip holds at a time)
    } else {
        // as many rows as the registers of a wave hold, in blocks of equal size
        const int64_t most = head_dim == 256 ? 1 : 2;
        p.row_blocks = (groups + most - 1) / most;
        p.row_groups = (int)((groups + p.row_blocks - 1) / p.row_blocks);
        p.tile_keys = f32 ? Elem<true>::kKeys : Elem<false>::kKeys;
        p.min_tiles = 128 / p.tile_keys;
        // One row group: more than the chip holds at a time but for FP32 and head_dim 64 (768 with BF16 and 64, 512 with 128, 256 with 256), which
        // evens out their ends over long sequences and is paid for by joining over short ones.  2 x 8 heads of 65537 slots at 256 / 512 / 1024 / 2048:
        // BF16 63 / 63 / 56 / 58 us with head_dim 64, 110 / 105 / 105 / 107 with 128, 184 / 181 / 184 / 205 with 256; 4 x 8 of 16000: 27 / 31 / 28 / 29,
        // 56 / 58 / 57 / 57, 94 / 100 / 104 / 125.  Two, 2 x 8 of 65537: 62 / 68 / 63 / 71, 114 / 112 / 116 / 129; FP32 130 / 109 / 122 / 127, 201 / 204 / 217 / 257.
        // Over 8 bits, whose ranges are read in half the time, as many as the chip holds: 2 x 8 heads of 131071 slots at 512 / 1024: 110 / 113 us, of 65537 63 / 68, one sequence's
        // 8 of 32000 21.7 / 30.5, 32 of 4096 19.5 / 22.6, 32 x 8 of up to 4000 55 / 54; 256 with head_dim 256: 2 of 30000 21.2 / 32.0.
        want = p.row_groups != 1 ? 512 : !eight ? 1024 : head_dim == 256 ? 256 : 512;
    }
    const int64_t whole = batch * heads * p.row_blocks, least = (int64_t)p.tile_keys * p.min_tiles;
    p.splits = std::max<int64_t>(1, std::min((max_length + least - 1) / least, (want + whole - 1) / whole));
    p.waves = kFewWaves;
    // A short cache in 8 bits is not cut: twice the waves, and no launch to join.  One sequence's 32 heads of 517 / 1024 / 2048 slots, cut / not: 10.8 / 9.6, 11.9 / 12.2,
    // 16.2 / 21.7 us; 8 x 8 heads 12.3 / 9.9, 15.7 / 13.6, 18.6 / 20.0; 16 x 8 13.7 / 10.8, 17.4 / 13.6, 21.6 / 20.0 (head_dim 256 has no registers for so many waves)
    if (eight && p.row_groups == 1 && head_dim != 256 && p.splits > 1 && max_length <= (whole >= 128 ? 2048 : 1024)) p.splits = 1, p.waves = kManyWaves;
    p.units = batch * heads * p.splits;
    p.workgroups = (p.units + 7) / 8 * 8 * p.row_blocks;
    return p;
}

size_t attend_bytes(const AttendPlan &p, int64_t rows, int64_t head_dim)
{
    return p.splits > 1 ? (size_t)(rows * p.splits * (head_dim + 2) * 4) : 0;
}

template <bool kF32, int kDim, bool kEight = false>
void attend_launch(const ArgsOf<kEight> &a, const AttendPlan &p, hipStream_t st)
{
    const dim3 grid((unsigned)p.workgroups);
    if (p.waves_of_rows > 0) attend_wide(a, p.waves_of_rows, (uint32_t)p.workgroups, st);
    else if (p.row_groups == 1 && (!kEight || p.waves == kFewWaves)) attend_kernel<kF32, kDim, 1, kEight><<<grid, 64 * kFewWaves, 0, st>>>(a);
    if constexpr (kEight) {
        if constexpr (kDim != 256)
            if (p.row_groups == 1 && p.waves == kManyWaves) attend_kernel<kF32, kDim, 1, kEight, kManyWaves><<<grid, 64 * kManyWaves, 0, st>>>(a);
    }
    if constexpr (kDim != 256) {
        if (p.row_groups == 2) attend_kernel<kF32, kDim, 2, kEight><<<grid, 64 * kFewWaves, 0, st>>>(a);
    }
    const int64_t rows = (int64_t)a.c.batch * a.tokens * a.q_heads;
    if (p.splits > kFewRanges) join_many_kernel<kF32, kDim><<<dim3((unsigned)rows), 256, 0, st>>>(a);
    else if (p.splits > 1) join_few_kernel<kF32, kDim><<<dim3((unsigned)((rows + 1024 / kDim - 1) / (1024 / kDim))), 256, 0, st>>>(a, (uint32_t)rows);
}

}  // namespace

}  // namespace fgmp

using namespace fgmp;

// What both calls check and do; the cache is in a already.
template <bool kEight>
static fgmp_status_t attend(ArgsOf<kEight> &a, fgmp_dtype_t dtype, const fgmp_heads_t *q, const fgmp_heads_t *k, const fgmp_heads_t *v, int64_t tokens,
                            int64_t q_heads, const uint64_t *tree, const int32_t *counts, float scale, int64_t max_length, const fgmp_heads_t *out,
                            float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    fgmp_status_t rc;
    if (tokens <= 0 || q_heads <= 0 || lse == nullptr || (k == nullptr) != (v == nullptr) || !(scale > 0.0f) || !(scale < INFINITY) || max_length < 0)
        return FGMP_ERR_INVALID_ARG;
    if (q_heads % a.c.heads != 0) return FGMP_ERR_BAD_SHAPE;
    if (tokens > kMaxTokens || q_heads > 65535) return FGMP_ERR_UNSUPPORTED;
    const int size = dtype_size(dtype), dim = a.c.head_dim;
    if ((rc = check_heads(q, a.c.batch, tokens, q_heads, dim, size, false)) != FGMP_OK) return rc;
    if ((rc = check_heads(out, a.c.batch, tokens, q_heads, dim, size, true)) != FGMP_OK) return rc;
    if (k != nullptr) {
        if ((rc = check_heads(k, a.c.batch, tokens, a.c.heads, dim, size, false)) != FGMP_OK) return rc;
        if ((rc = check_heads(v, a.c.batch, tokens, a.c.heads, dim, size, false)) != FGMP_OK) return rc;
    }
    if (max_length == 0 || max_length > a.c.slots) max_length = a.c.slots;
    const AttendPlan p = attend_plan(a.c.batch, tokens, q_heads, a.c.heads, dim, dtype == FGMP_F32, max_length, kEight);
    const int64_t rows = a.c.batch * tokens * q_heads;
    const size_t need = attend_bytes(p, rows, dim);
    if (need > 0) {
        if (workspace == nullptr) return FGMP_ERR_INVALID_ARG;
        if (!aligned16(workspace)) return FGMP_ERR_BAD_ALIGN;
        if (workspace_bytes < need) return FGMP_ERR_BUFFER_TOO_SMALL;
    }
    // (ranges are joined only where heads and row blocks are fewer than 1024, of 256 rows at most: that launch stays small)
    if (!launch_counts(p.workgroups, 64 * (p.waves_of_rows > 0 ? p.waves_of_rows : p.waves)) || rows >= (int64_t)1 << 31) return FGMP_ERR_UNSUPPORTED;
    a.q = static_cast<const char *>(q->data);
    a.q_batch = q->batch_stride * size, a.q_token = q->token_stride * size, a.q_head = q->head_stride * size;
    a.out = static_cast<char *>(out->data);
    a.o_batch = out->batch_stride * size, a.o_token = out->token_stride * size, a.o_head = out->head_stride * size;
    if (k != nullptr) {
        a.k = static_cast<const char *>(k->data);
        a.k_batch = k->batch_stride * size, a.k_token = k->token_stride * size, a.k_head = k->head_stride * size;
        a.v = static_cast<const char *>(v->data);
        a.v_batch = v->batch_stride * size, a.v_token = v->token_stride * size, a.v_head = v->head_stride * size;
    }
    a.lse = lse;
    a.tree = tree;
    a.counts = counts;
    a.tokens = (int32_t)tokens;
    a.q_heads = (int32_t)q_heads;
    a.group = (int32_t)(q_heads / a.c.heads);
    a.words = (int32_t)((tokens + 63) / 64);
    a.row_blocks = (uint32_t)p.row_blocks;
    a.units = (uint32_t)p.units;
    a.splits = (int32_t)p.splits;
    a.tile_keys = p.tile_keys;
    a.min_tiles = p.min_tiles;
    a.c2 = scale * kLog2e;
    a.part_o = static_cast<float *>(workspace);
    a.part_ml = a.part_o + rows * p.splits * dim;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if constexpr (kEight) {
        if (dim == 64) attend_launch<false, 64, true>(a, p, st);
        else if (dim == 128) attend_launch<false, 128, true>(a, p, st);
        else attend_launch<false, 256, true>(a, p, st);
    } else if (dtype == FGMP_F32) {
        if (dim == 64) attend_launch<true, 64>(a, p, st);
        else if (dim == 128) attend_launch<true, 128>(a, p, st);
        else attend_launch<true, 256>(a, p, st);
    } else {
        if (dim == 64) attend_launch<false, 64>(a, p, st);
        else if (dim == 128) attend_launch<false, 128>(a, p, st);
        else attend_launch<false, 256>(a, p, st);
    }
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

extern "C" {

size_t fgmp_tree_attention_workspace_bytes(int64_t batch, int64_t tokens, int64_t q_heads, int64_t heads, int64_t head_dim, int64_t max_length)
{
    if (batch <= 0 || tokens <= 0 || tokens > kMaxTokens || heads <= 0 || q_heads <= 0 || q_heads % heads != 0 || batch > 65535 ||
        q_heads > 65535 || max_length < 0 || max_length > (int64_t)1 << 30 || (head_dim != 64 && head_dim != 128 && head_dim != 256))
        return 0;
    // (the cache's type is not known here: whichever needs more)
    const AttendPlan p = attend_plan(batch, tokens, q_heads, heads, head_dim, false, max_length);
    const AttendPlan f = attend_plan(batch, tokens, q_heads, heads, head_dim, true, max_length);
    const int64_t rows = batch * tokens * q_heads;
    return std::max<size_t>(16, std::max(attend_bytes(p, rows, head_dim), attend_bytes(f, rows, head_dim)));
}

fgmp_status_t fgmp_tree_attention(const fgmp_heads_t *q, const fgmp_heads_t *k, const fgmp_heads_t *v, int64_t tokens, int64_t q_heads,
                                  const fgmp_cache_t *cache, const uint64_t *tree, const int32_t *counts, float scale, int64_t max_length,
                                  const fgmp_heads_t *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    AttendArgs a = {};
    const fgmp_status_t rc = check_cache(cache, &a.c);
    if (rc != FGMP_OK) return rc;
    return attend<false>(a, cache->dtype, q, k, v, tokens, q_heads, tree, counts, scale, max_length, out, lse, workspace, workspace_bytes, stream);
}

fgmp_status_t fgmp_quant_cache_attention(const fgmp_heads_t *q, const fgmp_heads_t *k, const fgmp_heads_t *v, int64_t tokens, int64_t q_heads,
                                         const fgmp_quant_cache_t *cache, const uint64_t *tree, const int32_t *counts, float scale, int64_t max_length,
                                         const fgmp_heads_t *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    QuantAttendArgs a = {};
    QuantCacheView c;
    const fgmp_status_t rc = check_quant_cache(cache, &c);
    if (rc != FGMP_OK) return rc;
    a.c = c.c;
    a.k_scales = c.k_scales, a.v_scales = c.v_scales;
    a.scale_page = c.scale_page, a.scale_head = c.scale_head;
    return attend<true>(a, FGMP_BF16, q, k, v, tokens, q_heads, tree, counts, scale, max_length, out, lse, workspace, workspace_bytes, stream);
}

fgmp_status_t fgmp_attention_weights(const fgmp_heads_t *q, const float *lse, int64_t tokens, int64_t q_heads, const fgmp_cache_t *cache,
                                     const int32_t *rows, int64_t accepted, const int32_t *counts, float scale, int64_t max_length,
                                     const float *weights, float *out, int64_t weights_stride, void *stream)
{
    WeightArgs a = {};
    fgmp_status_t rc = check_cache(cache, &a.c);
    if (rc != FGMP_OK) return rc;
    if (tokens <= 0 || accepted <= 0 || q_heads <= 0 || lse == nullptr || weights == nullptr || out == nullptr || !(scale > 0.0f) ||
        !(scale < INFINITY) || max_length < 0)
        return FGMP_ERR_INVALID_ARG;
    if (q_heads % a.c.heads != 0 || (rows == nullptr && accepted > tokens) || weights_stride < a.c.slots) return FGMP_ERR_BAD_SHAPE;
    if (tokens > kMaxTokens || accepted > kMaxTokens || q_heads > 65535) return FGMP_ERR_UNSUPPORTED;
    const int size = dtype_size(cache->dtype), dim = a.c.head_dim;
    if ((rc = check_heads(q, a.c.batch, tokens, q_heads, dim, size, false)) != FGMP_OK) return rc;
    if (max_length == 0 || max_length > a.c.slots) max_length = a.c.slots;
    constexpr int kBlock = 16 * kWeightKeys * kFewWaves;
    const int64_t pairs = (int64_t)a.c.batch * a.c.heads;
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>((max_length + kBlock - 1) / kBlock, (kWeightWorkgroups + pairs - 1) / pairs));
    if (!launch_counts(pairs * blocks, 64 * kFewWaves)) return FGMP_ERR_UNSUPPORTED;
    a.q = static_cast<const char *>(q->data);
    a.q_batch = q->batch_stride * size, a.q_token = q->token_stride * size, a.q_head = q->head_stride * size;
    a.lse = lse;
    a.rows = rows;
    a.counts = counts;
    a.tokens = (int32_t)tokens;
    a.accepted = (int32_t)accepted;
    a.q_heads = (int32_t)q_heads;
    a.group = (int32_t)(q_heads / a.c.heads);
    a.blocks = (int32_t)blocks;
    a.c2 = scale * kLog2e;
    a.weights = weights;
    a.out = out;
    a.stride = weights_stride;
    const dim3 grid((unsigned)(pairs * blocks));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (cache->dtype == FGMP_F32) {
        if (dim == 64) weights_kernel<true, 64><<<grid, 64 * kFewWaves, 0, st>>>(a);
        else if (dim == 128) weights_kernel<true, 128><<<grid, 64 * kFewWaves, 0, st>>>(a);
        else weights_kernel<true, 256><<<grid, 64 * kFewWaves, 0, st>>>(a);
    } else {
        if (dim == 64) weights_kernel<false, 64><<<grid, 64 * kFewWaves, 0, st>>>(a);
        else if (dim == 128) weights_kernel<false, 128><<<grid, 64 * kFewWaves, 0, st>>>(a);
        else weights_kernel<false, 256><<<grid, 64 * kFewWaves, 0, st>>>(a);
    }
    return hipGetLastError() == hipSuccess ? FGMP_OK : FGMP_ERR_HIP;
}

}  // extern "C"
