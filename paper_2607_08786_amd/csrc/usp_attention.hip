// usp_attention.hip -- attention of a step's rows over a paged cache: the planner, and the kernel
// for few rows of each sequence (single tokens).
//
// Bound by the cache's bytes, each read once: one token over 131072, 8 heads of 128 for 64 of q's, 537 MB, takes 93 us
// (5.8 TB/s; a 2 GB copy moves 5.1); 64 sequences of 1024 to 8191 tokens in 8 bits, 633 MB with the scales, 129 us (4.9);
// 16 sequences of up to 1023 tokens, 40 heads each, 199 MB, 34 us (5.8, part of it from the 256 MB cache). So K and V go
// from memory to the matrix unit's operands with nothing between, 16 KB a wavefront under way, eight wavefronts a CU; a
// tile fills 16 of the unit's columns with as many heads as share a head of the cache, down to one, which costs
// nothing: the unit idles. Loads that pass L2 by (43.9 -> 39.4 us for the 16 sequences) and one test for all of a
// block's masks, caps and biases instead of one a key (8 bits: 160 -> 129) brought most. The smallest calls are launch,
// the lengths, the table, the keys, one after the other: 4.9 us for one sequence of 101 tokens.
#include "usp_attention.h"

#include <algorithm>
#include <cmath>

namespace usp {
namespace {

// ---- Few rows of each sequence: one tile of up to 16 heads of a row at a time.

constexpr int kRowWaves = 4;
constexpr int kMostPieces = 256;  // of a tile: the join's weights lie in LDS

// What a workgroup does: piece `piece` of at most `pieces`, of `blocks` blocks each, of tile `tile` of row t.
struct Item {
    int s, t, tile, piece, pieces, blocks;
    int p, len;   // the row's token, and its sequence's
    int slot;     // of the tile's first piece
    int counter;
};

// Blocks that a row of a sequence may see.
__device__ inline int most_blocks(const AttendArgs &a, int len) {
    const int all = (len + kBlockTokens - 1) / kBlockTokens;
    return a.window && !a.last ? min(all, (a.window - 1 + kBlockTokens - 1) / kBlockTokens + 1) : all;
}

// Lane by lane sums over a wavefront by DPP row shifts and broadcasts; the last lane has the whole.
template <int CTRL, int ROWS>
__device__ inline uint32_t dpp_add(uint32_t v) {
    return v + __builtin_amdgcn_update_dpp(0u, v, CTRL, ROWS, 0xF, ROWS == 0xF);
}
__device__ inline uint32_t scan_lanes(uint32_t v) {
    v = dpp_add<0x111, 0xF>(v);  // row_shr:1
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    v = dpp_add<0x118, 0xF>(v);
    v = dpp_add<0x142, 0xA>(v);  // row_bcast:15
    return dpp_add<0x143, 0xC>(v);  // row_bcast:31
}
template <int CTRL, int ROWS>
__device__ inline float dpp_add(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0u, __builtin_bit_cast(uint32_t, v), CTRL, ROWS, 0xF, ROWS == 0xF));
}
__device__ inline float sum_lanes(float v) {
    v = dpp_add<0x111, 0xF>(v);
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    v = dpp_add<0x118, 0xF>(v);
    v = dpp_add<0x142, 0xA>(v);
    v = dpp_add<0x143, 0xC>(v);
    return __builtin_bit_cast(float, (uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kLanes - 1));
}

// Item number `item` of a head. Where tiles are cut, a piece has as many blocks as make
// 2^pieces_bits pieces of all of them, and every wavefront finds its item by itself: each
// lane counts the pieces of as many sequences as it takes. False: there is no such item.
__device__ inline bool find_item(const AttendArgs &a, int item, Item &it) {
    const int S = a.r.sequences, lane = threadIdx.x & (kLanes - 1);
    if (!a.split) {
        it.t = item / a.tiles;
        it.tile = item - it.t * a.tiles;
        if (it.t >= a.r.rows) return false;
        it.s = sequence_of(a.r, it.t);
        if (it.s >= S || offset_of(a.r, it.s) > it.t) return false;
        it.len = length_of(a.r, it.s);
        it.p = it.len - (offset_of(a.r, it.s + 1) - it.t);
        it.piece = 0;
        it.pieces = 1;
        it.blocks = 0;
        it.slot = it.counter = 0;
        return true;
    }
    // The lane's sequences s0 .. s0 + per - 1; the first one's figures stay at hand.
    const int per = (S + kLanes - 1) / kLanes, s0 = lane * per;
    auto figures = [&](int s, int &off, int &n, int &len) {
        off = n = len = 0;
        if (s >= S) return;
        off = offset_of(a.r, s);
        n = max(0, offset_of(a.r, s + 1) - off);
        len = length_of(a.r, s);
    };
    int off0, n0, len0;
    figures(s0, off0, n0, len0);
    float total = (float)n0 * (float)most_blocks(a, len0);
    for (int i = 1; i < per; ++i) {
        int off, n, len;
        figures(s0 + i, off, n, len);
        total += (float)n * (float)most_blocks(a, len);
    }
    // The sum's roundings are fewer than 128, of 2^-24 each: 2^-16 more, and the pieces are no more than were made room for.
    total = sum_lanes(total) * (float)(a.tiles * a.c.kv_heads) * (1.f + 1.f / 65536.f);
    const int blocks = (int)fminf(1e9f, fmaxf((float)a.min_blocks, ceilf(ldexpf(total, -a.pieces_bits))));
    auto pieces_of = [&](int len) {
        return min(kMostPieces, max(1, (most_blocks(a, len) + blocks - 1) / blocks));
    };
    constexpr uint32_t kFull = 1u << 24;  // more items than a grid has
    // n tiles is at most 16384 where tiles are cut, so of one sequence there are fewer than 2^23 items.
    const uint32_t items0 = (uint32_t)n0 * (uint32_t)a.tiles * (uint32_t)pieces_of(len0);
    uint32_t items = items0, slots = pieces_of(len0) > 1 ? items0 : 0;
    for (int i = 1; i < per; ++i) {
        int off, n, len;
        figures(s0 + i, off, n, len);
        const uint32_t of_s = (uint32_t)n * (uint32_t)a.tiles * (uint32_t)pieces_of(len);
        items = min(kFull, items + of_s);
        if (pieces_of(len) > 1) slots = min(kFull, slots + of_s);
    }
    const uint32_t items_end = scan_lanes(items), slots_end = scan_lanes(slots);
    const uint64_t has = __ballot((uint32_t)item < items_end);
    if (!has) return false;
    const int owner = __ffsll((unsigned long long)has) - 1;
    uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)(items_end - items), owner);
    uint32_t slot = (uint32_t)__builtin_amdgcn_readlane((int)(slots_end - slots), owner);
    for (int i = 0; i < per; ++i) {
        const int s = owner * per + i;
        if (s >= S) break;
        int off, n, len;
        if (i == 0) {
            off = __builtin_amdgcn_readlane(off0, owner);
            n = __builtin_amdgcn_readlane(n0, owner);
            len = __builtin_amdgcn_readlane(len0, owner);
        } else {
            figures(s, off, n, len);
        }
        const int pieces = pieces_of(len);
        const uint32_t of_s = (uint32_t)n * (uint32_t)a.tiles * (uint32_t)pieces;
        if ((uint32_t)item - at < of_s) {
            const int in = item - (int)at, tile = in / pieces;
            it.s = s;
            it.piece = in - tile * pieces;
            it.t = off + tile / a.tiles;
            it.tile = tile % a.tiles;
            it.len = len;
            it.p = len - n + tile / a.tiles;
            it.pieces = pieces;
            it.blocks = blocks;
            it.slot = (int)slot + tile * pieces;
            it.counter = (int)at + tile * pieces;
            // Offsets that decrease may give more items than the grid and the workspace were made for.
            return it.counter + pieces <= a.limit && (pieces == 1 || it.slot + pieces <= a.slot_limit);
        }
        at += of_s;
        if (pieces > 1) slot += of_s;
    }
    return false;
}

// Floats of a piece's partial result: maxima, sums, and the output of each of its columns.
__host__ __device__ inline int partial_floats(int columns, int width) { return 32 + columns * width; }

// MOD: scores are capped, biased or not scaled by a positive number.
template <int DS, int VB, bool MOD>
__global__ __launch_bounds__(kRowWaves *kLanes) void attend_rows_kernel(AttendArgs a) {
    constexpr int W = 32 * DS, kBlockBytes = (int)cache_block_bytes(W, VB);
    constexpr int kStride = W + 4;
    constexpr int kJoinFloats = kMostPieces * 32;
    constexpr int kShared = kRowWaves * 16 * kStride > kJoinFloats ? kRowWaves * 16 * kStride : kJoinFloats;
    __shared__ __attribute__((aligned(16))) float so[kShared];
    __shared__ float sm[kRowWaves][16], sl[kRowWaves][16];
    __shared__ uint32_t arrived;

    const int h = blockIdx.x % a.c.kv_heads;
    Item it;
    if (!find_item(a, blockIdx.x / a.c.kv_heads, it)) return;
    const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes;
    const int r = lane & 15, g = lane >> 4;
    const int columns = min(16, a.group - 16 * it.tile), head0 = h * a.group + 16 * it.tile;

    int lo, hi;
    span_of(a, it.t, it.p, it.len, lo, hi);
    int b0 = lo / kBlockTokens, b1 = (hi + kBlockTokens - 1) / kBlockTokens;
    if (hi <= lo) b0 = b1 = 0;
    int pieces = 1;
    if (it.pieces > 1) {
        const int want = min(it.pieces, max(1, (b1 - b0 + it.blocks - 1) / it.blocks));
        const int each = max(1, (b1 - b0 + want - 1) / want);
        pieces = max(1, (b1 - b0 + each - 1) / each);
        if (it.piece >= pieces) return;
        b0 += it.piece * each;
        b1 = min(b1, b0 + each);
    }

    half8 q[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s) q[s] = load_q8(a, it.t, head0 + r, 32 * s + 8 * g, r < columns);
    const float slope = MOD && a.slopes && r < columns ? a.slopes[head0 + r] * kLog2e : 0.f;

    floatx4 o[2 * DS];
#pragma unroll
    for (int d = 0; d < 2 * DS; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = kNothing, l = 0.f;  // l: of this lane's keys alone
    float unit = 1e-30f;          // 8 bits: the largest scale of values so far; o is in 2^-14 of it
    const uint8_t *head_base = a.c.base + (int64_t)h * a.c.page_blocks * kBlockBytes;
    const int32_t *table = a.r.table + (int64_t)it.s * a.r.ld_table;

    int pages = 0, places = 0;  // lane i: page, and block in it, of this wavefront's i-th block from here
    for (int n = 0, b = b0 + wave; b < b1; ++n, b += kRowWaves) {
        if (n % kLanes == 0) {
            const int mine = b + kRowWaves * lane;
            if (mine < b1) {
                const int in = mine / a.c.page_blocks;
                pages = table[in];
                places = mine - in * a.c.page_blocks;
            }
        }
        const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages, n % kLanes);
        if (page >= a.c.pages) continue;
        const uint8_t *block = head_base + (int64_t)page * a.c.page_bytes + (int64_t)__builtin_amdgcn_readlane(places, n % kLanes) * kBlockBytes;

        half8 k[DS][2], v[2 * DS];
        floatx4 ks[2], vs[2];
#pragma unroll
        for (int s = 0; s < DS; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int unit8 = (4 * s + g) * kBlockTokens + 16 * (r / 8) + 8 * i + r % 8;
                if (VB == 2)
                    k[s][i] = __builtin_nontemporal_load(reinterpret_cast<const half8 *>(block) + unit8);
                else
                    k[s][i] = halves_of(__builtin_nontemporal_load(reinterpret_cast<const v2u32 *>(block) + unit8));
            }
#pragma unroll
        for (int d = 0; d < 2 * DS; ++d) {
            const int unit8 = W / 8 * kBlockTokens + g * W + 16 * d + r;
            if (VB == 2)
                v[d] = __builtin_nontemporal_load(reinterpret_cast<const half8 *>(block) + unit8);
            else
                v[d] = halves_of(__builtin_nontemporal_load(reinterpret_cast<const v2u32 *>(block) + unit8));
        }
        if (VB == 1) {
            const floatx4 *scales = reinterpret_cast<const floatx4 *>(block + 2 * kBlockTokens * W);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                ks[i] = scales[2 * g + i];
                vs[i] = scales[kBlockTokens / 4 + 2 * g + i];
            }
        }

        floatx4 st[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int s = 0; s < DS; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) st[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[s][i], q[s], st[i], 0, 0, 0);

        // The scores of keys key0 .. key0 + 7.
        const int key0 = b * kBlockTokens + 8 * g;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = st[j / 4][j % 4];
            if (VB == 1) x[j] *= ks[j / 4][j % 4];
        }
        // Scores are scaled and rounded before their maximum is taken, so a maximum that stays fades nothing, whatever the
        // scores. (Scaled in the exponent's sum instead, the maximum's own rounding came in at every block.)
        if (MOD) {
            modify_scores(a, x, 8, slope, it.p, key0, [](int j) { return j; });
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= a.scale;
        }
        if (b * kBlockTokens < lo || (b + 1) * kBlockTokens > hi) {
            // What the row does not see may hold anything, and nothing times infinity is not nothing.
            uint32_t keep[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool seen = key0 + j >= lo && key0 + j < hi;
                keep[j] = seen ? 0xFFFFu : 0u;
                x[j] = seen ? x[j] : kNothing;
                if (VB == 1) vs[j / 4][j % 4] = seen ? vs[j / 4][j % 4] : 0.f;
            }
            if (VB == 2) {
                const v4u32 both = {keep[0] | keep[1] << 16, keep[2] | keep[3] << 16, keep[4] | keep[5] << 16, keep[6] | keep[7] << 16};
#pragma unroll
                for (int d = 0; d < 2 * DS; ++d) v[d] = __builtin_bit_cast(half8, __builtin_bit_cast(v4u32, v[d]) & both);
            }
        }
        float top = x[0], top_scale = VB == 1 ? vs[0][0] : 0.f;
#pragma unroll
        for (int j = 1; j < 8; ++j) {
            top = fmaxf(top, x[j]);
            if (VB == 1) top_scale = fmaxf(top_scale, vs[j / 4][j % 4]);
        }
        top = max_32(max_16(top));
        if (VB == 2) top -= fabsf(top) < kLargeScore ? kLift : kLargeLift;  // small weights in fp16's full precision
        const float m_new = fmaxf(m, top);
        const float base = m_new == kNothing ? 0.f : m_new;
        float fade = exp2_of(m - base);
        m = m_new;
        l *= fade;
        float to_unit = 1.f;
        if (VB == 1) {
            const float u = fmaxf(unit, max_32(max_16(top_scale)));
            if (u > unit) fade *= unit * __builtin_amdgcn_rcpf(u);  // a unit that stays leaves o as it is: the product need not be 1
            unit = u;
            to_unit = 16384.f * __builtin_amdgcn_rcpf(u);
        }
        float w[8], block_sum = 0.f;  // a block's first: to a large sum, single small ones may add nothing
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = exp2_of(x[j] - base);
            block_sum += w[j];
            if (VB == 1) w[j] *= vs[j / 4][j % 4] * to_unit;
        }
        // What is rounded off the weights takes part too: the matrix unit idles. (16 sequences of up to 1023 tokens 34.8 ->
        // 35.2 us, long ones and 8 bits nothing; errors against 64 bits 2.2e-4 -> 2.1e-4, of which the result's rounding is
        // most.) fp16 values may be infinite, so it must be neither negative nor nothing: weights are rounded down, and it is
        // 2^-24 at least where there is a weight.
        half8 p, rest;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            half2a high = {(_Float16)w[j], (_Float16)w[j + 1]};
            if (VB == 2) high = __builtin_bit_cast(half2a, __builtin_amdgcn_cvt_pkrtz(w[j], w[j + 1]));
            half2a low = {(_Float16)(w[j] - (float)high[0]), (_Float16)(w[j + 1] - (float)high[1])};
            if (VB == 2) low = __builtin_elementwise_max(low, __builtin_elementwise_min(high, half2a{(_Float16)0x1p-24f, (_Float16)0x1p-24f}));
            p[j] = high[0], p[j + 1] = high[1];
            rest[j] = low[0], rest[j + 1] = low[1];
        }
        l += block_sum;
#pragma unroll
        for (int d = 0; d < 2 * DS; ++d) {
            o[d] *= fade;
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[d], p, o[d], 0, 0, 0);
            o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[d], rest, o[d], 0, 0, 0);
        }
    }

    // The wavefronts' results together, in their order.
    l = sum_32(sum_16(l));
    if (g == 0) {
        sm[wave][r] = m;
        sl[wave][r] = l;
    }
    if (r < columns) {
        const float back = VB == 1 ? unit * (1.f / 16384.f) : 1.f;
#pragma unroll
        for (int d = 0; d < 2 * DS; ++d)
            *reinterpret_cast<floatx4 *>(&so[(wave * 16 + r) * kStride + 16 * d + 4 * g]) = o[d] * back;
    }
    __syncthreads();
    float *slots = a.partials;
    const int slot_floats = partial_floats(min(16, a.group), W);
    for (int e = threadIdx.x; e < columns * (W / 4); e += kRowWaves * kLanes) {
        const int col = e / (W / 4), d = 4 * (e % (W / 4));
        float top = sm[0][col];
#pragma unroll
        for (int w = 1; w < kRowWaves; ++w) top = fmaxf(top, sm[w][col]);
        const float base = top == kNothing ? 0.f : top;
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
            const float f = exp2_of(sm[w][col] - base);
            total += sl[w][col] * f;
            sum += *reinterpret_cast<const floatx4 *>(&so[(w * 16 + col) * kStride + d]) * f;
        }
        if (pieces == 1) {
            if (d < a.c.head_dim) store_out4(a, it.t, head0 + col, d, total == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : sum * (1.f / total));
        } else {
            float *slot = slots + ((int64_t)(it.slot + it.piece) * a.c.kv_heads + h) * slot_floats;
            const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(slot, (short)0, slot_floats * 4, kBufferRsrcWord3);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u32, sum), to, (32 + col * W + d) * 4, 0, kCachePolicyDevice);
            if (d == 0) {
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, top), to, col * 4, 0, kCachePolicyDevice);
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, total), to, (16 + col) * 4, 0, kCachePolicyDevice);
            }
        }
    }
    if (pieces == 1) return;

    // The last piece to arrive joins them, in their order.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part lies in memory
    __syncthreads();
    uint32_t *counter = a.counters + (int64_t)it.counter * a.c.kv_heads + h;
    if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (arrived != (uint32_t)pieces - 1) return;
    const int64_t step = (int64_t)a.c.kv_heads * slot_floats;  // from a piece's slot to the next
    float *first = slots + ((int64_t)it.slot * a.c.kv_heads + h) * slot_floats;
    for (int e = threadIdx.x; e < pieces * 32; e += kRowWaves * kLanes) {
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(first, (short)0, -1, kBufferRsrcWord3);
        so[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, (int)((e / 32 * step + e % 32) * 4), 0, kCachePolicyDevice));
    }
    __syncthreads();
    for (int e = threadIdx.x; e < columns * (W / 4); e += kRowWaves * kLanes) {
        const int col = e / (W / 4), d = 4 * (e % (W / 4));
        float top = kNothing;
        for (int i = 0; i < pieces; ++i) top = fmaxf(top, so[i * 32 + col]);
        const float base = top == kNothing ? 0.f : top;
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(first, (short)0, -1, kBufferRsrcWord3);
        floatx4 sum = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
        constexpr int kBatch = 32;  // loads of a turn, all under way at once
        for (int i0 = 0; i0 < pieces; i0 += kBatch) {
            v4u32 v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i0 + i < pieces)
                    v[i] = __builtin_amdgcn_raw_buffer_load_b128(from, (int)(((i0 + i) * step + 32 + col * W + d) * 4), 0, kCachePolicyDevice);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i0 + i < pieces) {
                    const float f = exp2_of(so[(i0 + i) * 32 + col] - base);
                    total += so[(i0 + i) * 32 + 16 + col] * f;
                    sum += __builtin_bit_cast(floatx4, v[i]) * f;
                }
        }
        if (d < a.c.head_dim) store_out4(a, it.t, head0 + col, d, total == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : sum * (1.f / total));
    }
    if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

typedef void (*AttendFn)(AttendArgs);

template <int VB, bool MOD>
AttendFn rows_kernel_of(int width) {
    switch (width) {
        case 32: return attend_rows_kernel<1, VB, MOD>;
        case 64: return attend_rows_kernel<2, VB, MOD>;
        case 96: return attend_rows_kernel<3, VB, MOD>;
        case 128: return attend_rows_kernel<4, VB, MOD>;
        case 192: return attend_rows_kernel<6, VB, MOD>;
        default: return attend_rows_kernel<8, VB, MOD>;
    }
}

struct AttendPlan {
    bool rows;             // the rows kernel; else the tiles kernel
    bool split;
    int tiles, pieces_bits, min_blocks;
    int pieces;            // of a tile at most (tiles kernel)
    int64_t limit, slots;  // items and partial results of a head
    size_t partial_bytes;
};

// Pieces that the rows kernel aims at, and blocks of a piece at least. Two workgroups of it fit a CU, 512 the chip. Few
// tiles, so long ones or an idle chip: one round of pieces, down to two blocks for each wavefront (8 tiles of 4096
// blocks of 16 KB: 92 us; 1024 pieces 105). Many tiles differ in length and are cut finer, so that the last to end are
// short (64 sequences of 1024 to 8192 tokens, 8 tiles each, 8 bits: 129 us; 143 with 512), but not where a piece's start
// and join would take as long as it (640 tiles of up to 32 blocks: 34.4 us whole, 43 in 1024 pieces).
constexpr int kFewTiles = 128, kFewBits = 9, kFewMinBlocks = 8, kManyBits = 10, kManyMinBlocks = 32;
// Workgroups of the tiles kernel that run at once, by the bytes of a value: three on a CU, two that convert 8 bits (512
// rows over 16512 tokens, 256 tiles: 426 us in two pieces each; a step before this one 438, and 493 in three). Counted at
// widths of up to 128; at 192 and 256 one workgroup fits a CU, and fewer pieces were not tried there.
constexpr int64_t kTilePlaces[] = {0, 512, 768};
constexpr int64_t kMostTilePieces = 16;
// The largest cap whose scores may be off by 2^-22 of it: 2^-14, a quarter of a weight's rounding to fp16.
constexpr float kPlainCap = 256.f;

AttendPlan plan_attention(const CacheView &c, const RowsView &r, int heads) {
    const int64_t group = heads / c.kv_heads;
    AttendPlan p = {};
    // The rows kernel reads the cache for each row, the tiles kernel for 128 columns, with fewer workgroups where there are
    // few sequences. 16 sequences of 4096 tokens, 8 heads for each of 8: 1 row each 46 against 67 us, 2 rows 66 / 66, 4
    // rows 97 / 65; one sequence of 65536: 54 / 122, 74 / 125, 96 / 126, 6 rows 198 / 129; with a head for each of 40 there:
    // 257 / 263, 2 rows 455 / 262.
    const int64_t S = r.sequences, T = r.rows;
    p.rows = T <= S || (T <= 4 * S && group >= 4 && S * c.kv_heads <= 64);
    if (!p.rows) {
        const int64_t columns = tile_columns(c.width);
        p.limit = ((int64_t)r.rows * group + columns - 1) / columns + r.sequences - 1;
        p.pieces = (int)std::max<int64_t>(1, std::min<int64_t>(kMostTilePieces, kTilePlaces[c.value_bytes] / (p.limit * c.kv_heads)));
        if (p.pieces > 1) p.partial_bytes = (size_t)(p.limit * c.kv_heads * p.pieces * tile_slot_floats(c.width)) * sizeof(float);
        return p;
    }
    p.tiles = (int)((group + 15) / 16);
    const int64_t all = (int64_t)r.rows * p.tiles;
    const bool few = all * c.kv_heads <= kFewTiles;
    p.pieces_bits = few ? kFewBits : kManyBits;
    p.min_blocks = few ? kFewMinBlocks : kManyMinBlocks;
    const int64_t pieces = ((int64_t)1 << p.pieces_bits) / c.kv_heads;
    // Cut where there are few tiles, and their counters and the lanes' sequences fit.
    p.split = all * c.kv_heads <= 16384 && r.sequences <= 4096 && (all + pieces) * c.kv_heads <= kMaxCounters &&
              r.capacity > p.min_blocks * kBlockTokens;
    p.limit = p.split ? all + pieces : all;
    if (p.split) {
        // Tiles of more than one piece have at most twice their even share.
        p.slots = std::min(p.limit, 2 * pieces + 2);
        p.partial_bytes = (size_t)(p.slots * c.kv_heads) * partial_floats((int)std::min<int64_t>(16, group), c.width) * sizeof(float);
    }
    return p;
}

}  // namespace

size_t attention_workspace_bytes(const CacheView &c, const RowsView &r, int heads) {
    const AttendPlan p = plan_attention(c, r, heads);
    return p.partial_bytes ? kCounterRegionBytes + p.partial_bytes : 0;
}

std::string describe_attention(const CacheView &c, const RowsView &r, int heads) {
    const AttendPlan p = plan_attention(c, r, heads);
    return std::string(p.rows ? "rows" : "tiles") + " W=" + std::to_string(c.width) +
           (p.rows ? p.split ? " pieces=" + std::to_string(1 << p.pieces_bits) : "" : " pieces=" + std::to_string(p.pieces)) +
           " grid=" + std::to_string(p.limit * c.kv_heads * (p.rows ? 1 : p.pieces));
}

bool attention_fits(const CacheView &c, const RowsView &r, int heads) {
    const AttendPlan p = plan_attention(c, r, heads);
    return p.limit * c.kv_heads * (p.rows ? 1 : p.pieces) <= kMostWorkgroups;
}

int launch_attention(const CacheView &c, const RowsView &r, const usp_attention_args &p, void *workspace, void *stream) {
    const AttendPlan plan = plan_attention(c, r, p.heads);
    AttendArgs a = {};
    a.c = c;
    a.r = r;
    a.first = p.first;
    a.last = p.last;
    a.q = reinterpret_cast<const uint16_t *>(p.q);
    a.out = reinterpret_cast<uint16_t *>(p.out);
    a.slopes = p.slopes;
    a.ld_q = p.ld_q;
    a.head_q = p.head_q;
    a.ld_out = p.ld_out;
    a.head_out = p.head_out;
    a.cap = std::min(p.cap, 1e38f) * kLog2e;  // twice it is finite
    a.cap_inv = p.cap > kPlainCap ? 1.f / a.cap : 0.f;
    a.scale = p.cap > 0.f && !a.cap_inv ? 2.f * kLog2e * p.scale / p.cap : p.scale * kLog2e;
    a.heads = p.heads;
    a.group = p.heads / c.kv_heads;
    a.window = p.window < r.capacity ? (int)p.window : 0;  // a longer one hides nothing
    a.tiles = plan.tiles;
    a.q_vec = (reinterpret_cast<uintptr_t>(p.q) & 15) == 0 && p.ld_q % 8 == 0 && p.head_q % 8 == 0;
    a.out_vec = (reinterpret_cast<uintptr_t>(p.out) & 7) == 0 && p.ld_out % 4 == 0 && p.head_out % 4 == 0;
    a.split = plan.split;
    a.pieces = plan.pieces;
    a.pieces_bits = plan.pieces_bits;
    a.min_blocks = plan.min_blocks;
    a.limit = (int)plan.limit;
    a.slot_limit = (int)plan.slots;
    a.counters = reinterpret_cast<uint32_t *>(workspace);
    a.partials = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + kCounterRegionBytes);
    const int64_t grid = plan.limit * c.kv_heads * (plan.rows ? 1 : plan.pieces);
    // (The tiles kernel multiplies plain scores by the product of their scale and the key's: up to 2^10, a finite one.)
    const bool modified = a.cap > 0.f || a.slopes || !(a.scale > 0.f) || (c.value_bytes == 1 && a.scale > 0x1p64f);
    if (!plan.rows) return launch_tiles(&a, c.width, c.value_bytes, modified, grid, stream);
    const AttendFn fn = c.value_bytes == 2 ? modified ? rows_kernel_of<2, true>(c.width) : rows_kernel_of<2, false>(c.width)
                                           : modified ? rows_kernel_of<1, true>(c.width) : rows_kernel_of<1, false>(c.width);
    hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(kRowWaves * kLanes), 0, reinterpret_cast<hipStream_t>(stream), a);
    return (int)hipGetLastError();
}

}  // namespace usp
