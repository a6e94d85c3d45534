// usp_attention.h -- what the attention kernels share (include/usp.h, usp_attention).
//
// Both kernels take a tile of columns (a column: one head of one row, all columns of a tile
// reading one head of the cache) through the blocks of 32 keys that it sees, once, with the
// running maximum m and sum l of each column's softmax:
//
//     S^T = K Q^T     (keys x columns; rows of K are the matrix unit's A operand)
//     p = exp2(s - m),  l = l exp2(m_old - m) + sum p
//     O^T = O^T exp2(m_old - m) + V^T P^T    (channels x columns; rows of V^T are A)
//
// S^T leaves a lane the scores of one column, and with the cache's order of a block's
// keys they are the 8 consecutive keys of which it hands over P^T's B operand: softmax and
// P stay in registers, without an exchange but the maximum over the lanes of a column. K and V
// are read in the order that they lie in (usp_cache.h).
#pragma once
#include "usp_cache.h"
#include "usp_device.h"

namespace usp {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t v2u32 __attribute__((ext_vector_type(2)));
typedef _Float16 half2a __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNothing = -__builtin_inff();

// Weights in fp16 are 2^(score - m), m being the largest score less one of these: the larger below kLargeScore, where m's
// rounding moves it by 2 at most, and one that rounds to 8 at most beyond, so that no weight passes fp16's 65504.
constexpr float kLift = 13.f, kLargeLift = 7.f, kLargeScore = 0x1.fp25f;

struct AttendArgs {
    CacheView c;
    RowsView r;
    const int32_t *first, *last;
    const uint16_t *q;
    uint16_t *out;
    const float *slopes;
    int64_t ld_q, head_q, ld_out, head_out;
    float scale;           // score of q . K in the exponent of 2, or the argument of the cap's exponential
    float cap;             // in the exponent of 2; 0: none
    float cap_inv;         // of a large cap 1 / cap (scale is then the score's), else 0
    int heads, group, window;
    int tiles;             // tiles of 16 heads of a row (rows kernel)
    int q_vec, out_vec;
    int split;             // whether tiles are cut into pieces (rows kernel)
    int pieces;            // most pieces of a tile (tiles kernel)
    int pieces_bits;       // 2^pieces_bits pieces of all tiles and heads together are aimed at (rows kernel)
    int min_blocks;        // of a piece at least (rows kernel)
    int limit, slot_limit; // items of a head in the grid, and slots of a head in the workspace
    uint32_t *counters;
    float *partials;
};

__device__ inline float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }
__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// The larger of a value and what the lanes 16 (32) away hold.
__device__ inline float max_16(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}
__device__ inline float max_32(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}
__device__ inline float sum_16(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
}
__device__ inline float sum_32(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
}

// Eight codes as fp16: the byte 128 + c under the exponent of 1024 is 1152 + c, exactly.
__device__ inline half8 halves_of(v2u32 codes) {
    const half2a bias = {(_Float16)-1152.f, (_Float16)-1152.f};
    v4u32 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t u = codes[i / 2] ^ 0x80808080u;
        const uint32_t w = __builtin_amdgcn_perm(0x64646464u, u, i % 2 ? 0x07030602u : 0x05010400u);
        out[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2a, w) + bias);
    }
    return __builtin_bit_cast(half8, out);
}

// Eight channels d .. d + 7 of a head of q, zeros behind head_dim and where there is no column.
__device__ inline half8 load_q8(const AttendArgs &a, int t, int head, int d, bool there) {
    half8 x = {};
    if (!there || d >= a.c.head_dim) return x;
    const uint16_t *from = a.q + (int64_t)t * a.ld_q + (int64_t)head * a.head_q + d;
    if (a.q_vec) return *reinterpret_cast<const half8 *>(from);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(_Float16, from[i]);
    return x;
}

// Channels d .. d + 3 of an output.
__device__ inline void store_out4(const AttendArgs &a, int t, int head, int d, floatx4 v) {
    uint16_t *to = a.out + (int64_t)t * a.ld_out + (int64_t)head * a.head_out + d;
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(uint16_t, (_Float16)v[i]);
    if (a.out_vec) {
        *reinterpret_cast<uint2 *>(to) = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = h[i];
    }
}

// The keys lo <= k < hi that row t, token p of a sequence of len, sees.
__device__ inline void span_of(const AttendArgs &a, int t, int p, int len, int &lo, int &hi) {
    lo = a.first ? a.first[t] : 0;
    if (a.window && p - a.window + 1 > lo) lo = p - a.window + 1;
    if (lo < 0) lo = 0;
    hi = a.last ? a.last[t] : p + 1;
    if (hi > len) hi = len;
    if (p < 0) hi = 0;
}

// Scores in the exponent of 2, from q . K: scaled, capped, biased. key(i): the key of x[i], less `key0`. (One branch for
// all of them: behind a branch for each, their exponentials waited for one another.)
template <class Scores, class Key>
__device__ inline void modify_scores(const AttendArgs &a, Scores &x, int n, float slope, int p, int key0, Key key) {
#pragma unroll
    for (int i = 0; i < n; ++i) x[i] *= a.scale;
    if (a.cap_inv > 0.f) {
        // The form below is off by some 2^-22 of the cap, however small the score. Here x is the score, y = x / cap, and
        // tanh(y) for |y| < 1 / 8 the series to y^7, off by 2^-29 of itself.
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float y = x[i] * a.cap_inv, z = y * y;
            const float series = fmaf(x[i] * z, fmaf(z, fmaf(z, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), x[i]);
            const float whole = fmaf(-2.f * a.cap, __builtin_amdgcn_rcpf(1.f + exp2_of(2.f * kLog2e * y)), a.cap);
            x[i] = fabsf(y) < 0.125f ? series : whole;
        }
    } else if (a.cap > 0.f) {  // cap tanh(y) is cap (1 - 2 / (1 + exp(2 y))); x is 2 y in the exponent of 2
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = fmaf(-2.f * a.cap, __builtin_amdgcn_rcpf(1.f + exp2_of(x[i])), a.cap);
    }
    if (a.slopes) {
        const float away = (float)(p - key0);  // and the differences are exact below 2^24
#pragma unroll
        for (int i = 0; i < n; ++i) x[i] = fmaf(-slope, fabsf(away - (float)key(i)), x[i]);
    }
}

}  // namespace

constexpr int kTileWaves = 4;
int tile_columns(int width);
int64_t tile_slot_floats(int width);  // of a piece's partial result
int launch_tiles(const void *args, int width, int value_bytes, bool modified, int64_t grid, void *stream);  // args: an AttendArgs

}  // namespace usp
