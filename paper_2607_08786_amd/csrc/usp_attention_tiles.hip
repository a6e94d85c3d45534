// usp_attention_tiles.hip -- attention of many rows of each sequence (prompts and pieces of
// prompts): tiles of columns of consecutive rows and the heads that a cache's head serves.
//
// A workgroup of four wavefronts has 128 columns, 32 each; a block of keys and values goes through
// LDS once for all of them, double buffered, by transfers straight into LDS (fp16), where its
// units already lie in operand order. Products are v_mfma_f32_32x32x16_f16.
//
// What bounds it: one prompt of 4096 tokens, 64 heads on 8 of 128 channels, takes 317 us, 869 TFLOP/s;
// an 8192^3 library product reaches 1157 on the same card, a 16384^3 one 1310. A wavefront's step over a
// block is 16 products (512 cycles of the matrix unit) and 157 vector instructions, all else counted in, 16 of them
// exponentials, of which half overlap at best: a matrix and eight vector instructions took 19.6 ns a step where the one
// alone takes 14.6 and the others 11.3. About 40 of the 157 are o and l faded: 66 in each step where one of 32 columns
// finds a larger maximum, which for scores in random order is 1 - (1 - 1 / b)^32 at block b, 61% of this prompt's steps. That
// part need not be: a maximum that grows little could stay. And the clock falls under this load, from 2.5 (a long cache's
// single token) to 1.8-1.9 GHz. Steps on the way: a plain loop 779 us; blocks requested ahead and operands read together
// 348; straight into LDS, operands four products ahead, three wavefronts a SIMD 312; weights lifted into fp16's range, sums
// by blocks, large scores 317. Without gain: priorities of wavefronts, 2 or 6 products ahead. Slower: two blocks under way
// (339, registers spilled), softmax of a block between the products of its neighbours (369, two wavefronts a SIMD), two
// tiles of columns a wavefront (556, one). At 192 and 256 channels one wavefront a SIMD is left: the same prompt takes 838
// and 993 us, 493 and 554 TFLOP/s.
//
// 8 bits: 512 rows over 16512 tokens, the same heads, 428 us, 638 TFLOP/s (at 256 channels 1323, 412): codes go raw into
// LDS and are converted there once for the four wavefronts, two wavefronts a SIMD for want of registers. Scales of values
// taken apart, for exact products with the codes, cost 50 us of it (374 without, at an error against 64 bits of 3.1e-4
// instead of 2.4e-4).
#include "usp_attention.h"

#include <utility>

namespace usp {
namespace {

constexpr int kAhead = 4;           // products that operands are read ahead
constexpr int kMinTileBlocks = 6;   // blocks of a piece at least

// The first tile of sequence s: those before it have at most so many.
template <int COLUMNS>
__device__ inline int first_tile(const AttendArgs &a, int s) {
    return (int)((int64_t)offset_of(a.r, s) * a.group / COLUMNS) + s;
}

// A scale of values is taken apart into one of 4 bits, whose products with codes fp16 holds exactly (from 2^-21 on; those of
// smaller ones are rounded to multiples of 2^-24, as the result is), and a factor near 1 that the weight of its key takes,
// in its exponent (so that the largest weight is a power of two all the same, which has no rounding): rounded products would
// add to the result's error as much as its own rounding.
__device__ inline float short_scale(float s) { return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, s) + 0x80000u) & 0xFFF00000u); }

// Eight codes of keys j .. j + 7 of a channel times their short scales, as fp16 values.
__device__ inline half8 values_of(v2u32 codes, floatx4 s0, floatx4 s1) {
    half8 out;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int8_t c = (int8_t)(codes[i / 4] >> (8 * (i % 4)));
        out[i] = (_Float16)((float)c * (i < 4 ? s0[i % 4] : s1[i % 4]));
    }
    return out;
}

// A wavefront has 32 of the tile's columns. MOD: scores are capped, biased or not scaled by a positive number.
template <int DS, int VB, bool MOD>
__global__ __launch_bounds__(kTileWaves *kLanes, DS > 4 ? 1 : VB == 1 ? 2 : 3) void attend_tiles_kernel(AttendArgs a) {
    constexpr int W = 32 * DS, kBlockBytes = (int)cache_block_bytes(W, VB);
    constexpr int kColumns = 32 * kTileWaves;
    constexpr int kKeyUnits = W / 8 * kBlockTokens;  // units of 8 keys' channels, and as many of values'
    constexpr int kThreads = kTileWaves * kLanes;
    __shared__ half8 staged[2][2 * kKeyUnits];  // blocks of keys, then of values, as in the cache
    // 8 bits: blocks as they lie in the cache, and of the keys of four blocks their scales (times that of the scores), the
    // short scales of their values, and the factors f of their weights as logarithms and as 1 / f - 1 (near 0 both: in
    // fp16 they are off by less than 2^-15).
    __shared__ v2u32 raw[3][VB == 1 ? kBlockBytes / 8 : 1];
    __shared__ floatx4 key_scales[4][VB == 1 ? kBlockTokens / 4 : 1], value_scales[4][VB == 1 ? kBlockTokens / 4 : 1];
    __shared__ half8 factors[4][2][VB == 1 ? kBlockTokens / 8 : 1];
    __shared__ int ends[4][kTileWaves];
    __shared__ int odd[kTileWaves];  // whether a wavefront's part of a block's values holds any that is not finite
    __shared__ uint32_t arrived;

    const int h = blockIdx.x % a.c.kv_heads, piece = (int)(blockIdx.x / a.c.kv_heads) % a.pieces;
    const int tile = a.limit - 1 - (int)(blockIdx.x / a.c.kv_heads) / a.pieces;  // a prompt's last rows see most: they begin
    int s = 0;
    {
        int below = a.r.sequences;  // first_tile(s) <= tile < first_tile(below)
        while (below - s > 1) {
            const int mid = (s + below) / 2;
            if (first_tile<kColumns>(a, mid) <= tile)
                s = mid;
            else
                below = mid;
        }
    }
    const int off = offset_of(a.r, s), n = offset_of(a.r, s + 1) - off, len = length_of(a.r, s);
    const int64_t column0 = (int64_t)(tile - first_tile<kColumns>(a, s)) * kColumns;
    if (column0 < 0 || column0 >= (int64_t)n * a.group) return;

    const int lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes, c = lane & 31, half = lane >> 5;
    const int64_t column = column0 + 32 * wave + c;
    const int row = (int)(column / a.group), head = h * a.group + (int)(column - (int64_t)row * a.group);
    const bool there = row < n;
    const int p = len - n + row;
    // The keys that this column sees, that the wavefront's see any of, and that all of them see.
    int lo = 0, hi = 0, any_lo = 0x7FFFFFFF, any_hi = 0, all_lo = 0, all_hi = 0x7FFFFFFF;
    if (there) {
        span_of(a, off + row, p, len, lo, hi);
        if (hi > lo) {
            any_lo = min(any_lo, lo);
            any_hi = max(any_hi, hi);
        }
        all_lo = lo;
        all_hi = hi;
    }
    const float slope = MOD && a.slopes && there ? a.slopes[head] * kLog2e : 0.f;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        any_lo = min(any_lo, __shfl_xor(any_lo, d, kLanes));
        any_hi = max(any_hi, __shfl_xor(any_hi, d, kLanes));
        all_lo = max(all_lo, __shfl_xor(all_lo, d, kLanes));
        all_hi = min(all_hi, __shfl_xor(all_hi, d, kLanes));
    }
    any_lo = __builtin_amdgcn_readfirstlane(any_lo);
    any_hi = __builtin_amdgcn_readfirstlane(any_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    if (lane == 0) {
        ends[0][wave] = any_lo;
        ends[1][wave] = any_hi;
        ends[2][wave] = all_lo;
        ends[3][wave] = all_hi;
    }
    __syncthreads();
    int tile_lo = ends[0][0], tile_hi = ends[1][0], tile_all_lo = ends[2][0], tile_all_hi = ends[3][0];
#pragma unroll
    for (int w = 1; w < kTileWaves; ++w) {
        tile_lo = min(tile_lo, ends[0][w]);
        tile_hi = max(tile_hi, ends[1][w]);
        tile_all_lo = max(tile_all_lo, ends[2][w]);
        tile_all_hi = min(tile_all_hi, ends[3][w]);
    }
    tile_lo = __builtin_amdgcn_readfirstlane(tile_lo);
    tile_hi = __builtin_amdgcn_readfirstlane(tile_hi);
    tile_all_lo = __builtin_amdgcn_readfirstlane(tile_all_lo);
    tile_all_hi = __builtin_amdgcn_readfirstlane(tile_all_hi);
    int b1 = (tile_hi + kBlockTokens - 1) / kBlockTokens;
    int b0 = tile_hi > tile_lo ? tile_lo / kBlockTokens : b1;
    int pieces = 1;
    if (a.pieces > 1) {
        const int want = min(a.pieces, max(1, (b1 - b0) / kMinTileBlocks));
        const int each = max(1, (b1 - b0 + want - 1) / want);
        pieces = max(1, (b1 - b0 + each - 1) / each);
        if (piece >= pieces) return;
        b0 += piece * each;
        b1 = min(b1, b0 + each);
    }

    half8 q[2 * DS];
#pragma unroll
    for (int i = 0; i < 2 * DS; ++i) q[i] = load_q8(a, off + row, head, 16 * i + 8 * half, there);

    floatx16 o[DS];
#pragma unroll
    for (int d = 0; d < DS; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = kNothing, l = 0.f;
    // Weights are taken relative to m, a column's largest scaled score less `lift`, so that fp16 holds the largest one as some
    // 2^lift and small ones to its full precision down to 2^(-14 - lift) of it. Plain scores are scaled in the exponent's one
    // sum, which holds their product exactly, so all weights of a column are off by m's rounding: by 2 in the exponent below
    // kLargeScore, and by anything beyond. Where q and the biases do not rule that out (|q . K| is at most 65504 sum |q|),
    // scores are scaled and rounded first, as the other kernels' are, on the way past the masks, and lifted less. (Branches in
    // the loop that look at m took 1.4 to 10% of a prompt; this takes nothing at 64 and 128 channels and 1% at 256, and
    // `late` in a vector register spilled 16 others.)
    constexpr bool kPlain = !MOD && VB == 2;
    float bound = a.cap;
    if (!MOD || a.cap == 0.f) {
        float sum = W * 0x1p-14f;  // covers subnormal channels, whether or not the sum takes them as zeros
#pragma unroll
        for (int i = 0; i < 2 * DS; ++i) {
            const v4u32 bits = __builtin_bit_cast(v4u32, q[i]) & 0x7FFF7FFFu;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2a, bits[j]), half2a{(_Float16)1.f, (_Float16)1.f}, sum, false);
        }
        sum = sum_32(sum);
        bound = sum < __builtin_inff() ? sum * 65504.f * fabsf(a.scale) : 0.f;  // a row of NaN: no cause to round others otherwise
    }
    if (MOD) bound += fabsf(slope) * (float)len;
    const bool large = __any(!(bound < kLargeScore)), scale_first = kPlain && large;
    const float lift = uniform(large ? kLargeLift : kLift);
    const float late = kPlain ? uniform(large ? 1.f : a.scale) : 1.f;  // what is left to multiply scores by in the exponent

    const int32_t *table = a.r.table + (int64_t)s * a.r.ld_table;
    const uint8_t *head_base = a.c.base + (int64_t)h * a.c.page_blocks * kBlockBytes;
    int listed = b0 - kLanes, pages = 0, places = 0;  // lane i: page, and block in it, of block listed + i
    // The first block from b on whose page is one of the cache's, or b1; its address.
    auto next = [&](int b, const uint8_t *&block) {
        for (; b < b1; ++b) {
            if (b - listed >= kLanes) {
                listed = b;
                const int mine = b + lane;
                if (mine < b1) {
                    const int in = mine / a.c.page_blocks;
                    pages = table[in];
                    places = mine - in * a.c.page_blocks;
                }
            }
            const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages, b - listed);
            if (page < a.c.pages) {
                block = head_base + (int64_t)page * a.c.page_bytes + (int64_t)__builtin_amdgcn_readlane(places, b - listed) * kBlockBytes;
                break;
            }
        }
        return b;
    };
    // A block on its way into LDS, 16 bytes a lane: the compiler neither sees these transfers nor waits for them.
    auto request = [&](const uint8_t *block, int buffer) {
        const uint64_t from = reinterpret_cast<uint64_t>(block);
        const v4i32 rsrc = {(int)(uint32_t)from, (int)((uint32_t)(from >> 32) & 0xFFFFu), kBlockBytes, kBufferRsrcWord3};
        const void *base = VB == 2 ? (const void *)staged[buffer] : (const void *)raw[VB == 1 ? buffer : 0];
        const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)as_lds(base) + wave * kLanes * 16);
#pragma unroll
        for (int i = 0; i * kThreads * 16 < kBlockBytes; ++i)
            if ((i + 1) * kThreads * 16 <= kBlockBytes || (i * kThreads + (int)threadIdx.x) * 16 < kBlockBytes)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                             :
                             : "s"(to + 16u * kThreads * i), "v"(16 * (kThreads * i + (int)threadIdx.x)), "s"(rsrc)
                             : "memory", "m0");
    };
    // 8 bits: codes as fp16, those of values times their short scales.
    auto convert = [&](int from, int slot, int buffer) {
        const v2u32 *codes = raw[VB == 1 ? from : 0];
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            const int u = i * kThreads + (int)threadIdx.x;
            if ((i + 1) * kThreads <= kKeyUnits || u < kKeyUnits) {
                staged[buffer][u] = halves_of(codes[u]);
            } else {
                const floatx4 *scales = &value_scales[slot][VB == 1 ? 2 * ((u - kKeyUnits) / W) : 0];
                staged[buffer][u] = values_of(codes[u], scales[0], scales[1]);
            }
        }
    };
    // What the scales of a block's 32 keys and values come to, one of each a lane.
    auto put_scales = [&](int from, int slot) {
        if (lane >= kBlockTokens) return;
        const float *scales = reinterpret_cast<const float *>(raw[VB == 1 ? from : 0] + 2 * kKeyUnits) + lane;
        const float value = scales[kBlockTokens], brief = short_scale(value), f = value * __builtin_amdgcn_rcpf(brief);
        const _Float16 log = (_Float16)(fabsf(f - 1.f) < 0.5f ? __builtin_amdgcn_logf(f) : 0.f);  // of 0 and NaN: none
        reinterpret_cast<float *>(key_scales[slot])[lane] = scales[0] * (MOD ? 1.f : a.scale);
        reinterpret_cast<float *>(value_scales[slot])[lane] = brief;
        reinterpret_cast<_Float16 *>(factors[slot][0])[lane] = log;
        reinterpret_cast<_Float16 *>(factors[slot][1])[lane] = (_Float16)(exp2_of(-(float)log) - 1.f);
    };
    // Nothing times infinity is not nothing: in a block that some column does not see the whole of, values that are not
    // finite are left out of the product, and added to the columns that see them (below).
    auto clean = [&](int buffer) {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < DS; ++i) {
            const int u = i * kThreads + (int)threadIdx.x;
            if ((i + 1) * kThreads <= kKeyUnits || u < kKeyUnits) continue;
            v4u32 bits = __builtin_bit_cast(v4u32, staged[buffer][u]);
            uint32_t any = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t inf = ((bits[j] & 0x7C007C00u) + 0x04000400u) >> 15 & 0x00010001u;
                any |= inf;
                bits[j] &= ~(inf * 0xFFFFu);
            }
            if (any) staged[buffer][u] = __builtin_bit_cast(half8, bits);
            bad |= any;
        }
        const int any = __any(bad != 0);
        if (lane == 0) odd[wave] = any;
        lds_barrier();
    };
    auto all_see = [&](int b) { return tile_all_lo <= b * kBlockTokens && (b + 1) * kBlockTokens <= tile_all_hi; };

    // Blocks under way: the one at work, and those after it, b1 where there is none. fp16: the next is requested while one is
    // at work. 8 bits: of the three after it the first is converted, the second's scales are taken apart, the third requested.
    constexpr int kUnderWay = VB == 1 ? 3 : 1;
    int blocks[4];
    const uint8_t *at[4] = {nullptr, nullptr, nullptr, nullptr};
    blocks[0] = next(b0, at[0]);
    if (blocks[0] < b1) request(at[0], 0);
#pragma unroll
    for (int i = 1; i < kUnderWay; ++i) {
        at[i] = at[i - 1];
        blocks[i] = next(blocks[i - 1] + 1, at[i]);
        if (blocks[i] < b1) request(at[i], i);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_only(0));  // of q too: else the loop waits for what it requests ahead
    __syncthreads();
    if (VB == 1) {
        if (wave < 2 && blocks[wave] < b1) put_scales(wave, wave);
        lds_barrier();
        if (blocks[0] < b1) convert(0, 0, 0);
        lds_barrier();
    }
    int ring = 0;  // the first block's place among the raw ones
    for (int step = 0; blocks[0] < b1; ++step) {
        const int buffer = step & 1, slot = step & 3, b = blocks[0];
        const uint8_t *here = at[0];
        at[kUnderWay] = at[kUnderWay - 1];
        blocks[kUnderWay] = next(blocks[kUnderWay - 1] + 1, at[kUnderWay]);
        if (blocks[kUnderWay] < b1) request(at[kUnderWay], VB == 1 ? ring : buffer ^ 1);
        const int second = ring == 2 ? 0 : ring + 1, third = second == 2 ? 0 : second + 1;
        if (VB == 1 && blocks[1] < b1) convert(second, (slot + 1) & 3, buffer ^ 1);
        const int block_lo = b * kBlockTokens, block_hi = block_lo + kBlockTokens;
        if (!all_see(b)) clean(buffer);
        if (VB == 1 && blocks[VB == 1 ? 2 : 0] < b1 && wave == slot) put_scales(third, (slot + 2) & 3);  // in turn
        if (block_hi > any_lo && block_lo < any_hi) {  // else this wavefront sees nothing of it
            const half8 *keys = staged[buffer], *values = staged[buffer] + kKeyUnits;
            const bool whole = all_lo <= block_lo && block_hi <= all_hi;
            constexpr int kProducts = 2 * DS;  // with the keys, and as many with the values
            constexpr int ahead = kAhead < kProducts ? kAhead : kProducts;
            half8 k[kProducts], v[kProducts];
#pragma unroll
            for (int i = 0; i < ahead; ++i) k[i] = keys[(2 * i + half) * kBlockTokens + c];
            floatx16 st;
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = 0.f;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                if (i + ahead < kProducts)
                    k[i + ahead] = keys[(2 * (i + ahead) + half) * kBlockTokens + c];
                else {
                    const int j = i + ahead - kProducts;
                    v[j] = values[(2 * (j % 2) + half) * W + 32 * (j / 2) + c];
                }
                st = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[i], q[i], st, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            half8 w[2];
            // Register 8 u + j holds the score of key block_lo + 16 u + 8 half + j.
            half8 log_factor[2], less_one[2];
            if (VB == 1) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    log_factor[u] = factors[slot][0][VB == 1 ? 2 * u + half : 0];
                    less_one[u] = factors[slot][1][VB == 1 ? 2 * u + half : 0];
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float by = key_scales[slot][VB == 1 ? 4 * (i / 8) + 2 * half + i % 8 / 4 : 0][i % 4];
                    st[i] = fmaf(st[i], by, MOD ? 0.f : (float)log_factor[i / 8][i % 8]);
                }
            }
            if (MOD) modify_scores(a, st, 16, slope, p, block_lo + 8 * half, [](int i) { return 16 * (i / 8) + i % 8; });
            if (MOD && VB == 1) {
#pragma unroll
                for (int i = 0; i < 16; ++i) st[i] += (float)log_factor[i / 8][i % 8];
            }
            if (!whole || scale_first) {
                if (scale_first) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) st[i] *= a.scale;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = block_lo + 16 * (i / 8) + 8 * half + i % 8;
                    st[i] = key >= lo && key < hi ? st[i] : kNothing;
                }
            }
            float top = st[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, st[i]);
            top = fmaxf(m, fmaf(max_32(top), late, -lift));
            if (__any(top > m)) {
                const float fade = exp2_of(m - (top == kNothing ? 0.f : top));
                m = top;
                l *= fade;
#pragma unroll
                for (int d = 0; d < DS; ++d) o[d] *= fade;
            }
            const float base = m == kNothing ? 0.f : -m;
            // The sum takes the weights as the product does. (A block's first: to a large weight, two small ones may add nothing.)
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i / 8][i % 8] = (_Float16)exp2_of(fmaf(st[i], late, base));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const half2a pair = {w[i / 4][2 * (i % 4)], w[i / 4][2 * (i % 4) + 1]};
                sum = __builtin_amdgcn_fdot2(pair, half2a{(_Float16)1.f, (_Float16)1.f}, sum, false);
                if (VB == 1) sum = __builtin_amdgcn_fdot2(pair, half2a{less_one[i / 4][2 * (i % 4)], less_one[i / 4][2 * (i % 4) + 1]}, sum, false);
            }
            l += sum;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                const int j = i + ahead;
                if (j < kProducts) v[j] = values[(2 * (j % 2) + half) * W + 32 * (j / 2) + c];
                o[i / 2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[i], w[i % 2], o[i / 2], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (!all_see(b) && (odd[0] | odd[1] | odd[2] | odd[3])) {
                // Rare, so straight from the cache.
#pragma unroll 1
                for (int j = 0; j < kBlockTokens; ++j) {
                    const bool sees = block_lo + j >= lo && block_lo + j < hi;
#pragma unroll
                    for (int d = 0; d < DS; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int at = kKeyUnits * 8 + ((j / 8) * W + 32 * d + 8 * (i / 4) + 4 * half + i % 4) * 8 + j % 8;
                            float x;
                            if (VB == 2)
                                x = (float)reinterpret_cast<const _Float16 *>(here)[at];
                            else
                                x = reinterpret_cast<const float *>(here + 2 * kBlockTokens * W)[kBlockTokens + j];
                            if (sees && !(fabsf(x) < __builtin_inff())) o[d][i] += x;
                        }
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what was requested lies in LDS
        lds_barrier();
#pragma unroll
        for (int i = 0; i < kUnderWay; ++i) {
            blocks[i] = blocks[i + 1];
            at[i] = at[i + 1];
        }
        ring = second;
    }

    l = sum_32(l);
    if (pieces > 1) {
        // A piece's result lies as the lanes hold it. The last piece to arrive joins them, in their order.
        constexpr int kParts = DS * 4 + 1;  // of 16 bytes a lane
        constexpr int64_t kSlotFloats = (int64_t)kParts * 4 * kThreads;
        float *slot = a.partials + ((int64_t)tile * a.pieces * a.c.kv_heads + h) * kSlotFloats;
        const int64_t step = a.c.kv_heads * kSlotFloats;
        const int at = (int)threadIdx.x * 16;
        {
            const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(slot + piece * step, (short)0, (int)(kSlotFloats * 4), kBufferRsrcWord3);
#pragma unroll
            for (int i = 0; i < DS * 4; ++i) {
                const floatx4 x = {o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u32, x), to, i * kThreads * 16 + at, 0, kCachePolicyDevice);
            }
            const floatx4 x = {m, l, 0.f, 0.f};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u32, x), to, DS * 4 * kThreads * 16 + at, 0, kCachePolicyDevice);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's part lies in memory
        __syncthreads();
        uint32_t *counter = a.counters + (int64_t)tile * a.c.kv_heads + h;
        if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != (uint32_t)pieces - 1) return;
        float top = kNothing;
        for (int i = 0; i < pieces; ++i) {
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(slot + i * step, (short)0, (int)(kSlotFloats * 4), kBufferRsrcWord3);
            top = fmaxf(top, __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from, DS * 4 * kThreads * 16 + at, 0, kCachePolicyDevice)));
        }
        const float base = top == kNothing ? 0.f : top;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < DS; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        for (int i = 0; i < pieces; ++i) {
            const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(slot + i * step, (short)0, (int)(kSlotFloats * 4), kBufferRsrcWord3);
            v4u32 x[DS * 4 + 1];
#pragma unroll
            for (int j = 0; j < DS * 4 + 1; ++j)
                x[j] = __builtin_amdgcn_raw_buffer_load_b128(from, j * kThreads * 16 + at, 0, kCachePolicyDevice);
            const floatx4 ml = __builtin_bit_cast(floatx4, x[DS * 4]);
            const float f = exp2_of(ml[0] - base);
            l = fmaf(ml[1], f, l);
#pragma unroll
            for (int j = 0; j < DS * 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j / 4][4 * (j % 4) + e] = fmaf(__builtin_bit_cast(floatx4, x[j])[e], f, o[j / 4][4 * (j % 4) + e]);
        }
        if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (!there) return;
#pragma unroll
    for (int d = 0; d < DS; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int channel = 32 * d + 8 * i + 4 * half;
            floatx4 v = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
            v = l == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : v * inv;
            if (channel < a.c.head_dim) store_out4(a, off + row, head, channel, v);
        }
}

template <int VB, bool MOD>
void (*tiles_kernel_of(int width))(AttendArgs) {
    switch (width) {
        case 32: return attend_tiles_kernel<1, VB, MOD>;
        case 64: return attend_tiles_kernel<2, VB, MOD>;
        case 96: return attend_tiles_kernel<3, VB, MOD>;
        case 128: return attend_tiles_kernel<4, VB, MOD>;
        case 192: return attend_tiles_kernel<6, VB, MOD>;
        default: return attend_tiles_kernel<8, VB, MOD>;
    }
}

}  // namespace

int tile_columns(int) { return 32 * kTileWaves; }

int64_t tile_slot_floats(int width) { return (int64_t)(width / 8 + 1) * 4 * kTileWaves * kLanes; }

int launch_tiles(const void *args, int width, int value_bytes, bool modified, int64_t grid, void *stream) {
    const AttendArgs &a = *reinterpret_cast<const AttendArgs *>(args);
    const auto fn = value_bytes == 2 ? modified ? tiles_kernel_of<2, true>(width) : tiles_kernel_of<2, false>(width)
                                     : modified ? tiles_kernel_of<1, true>(width) : tiles_kernel_of<1, false>(width);
    hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(kTileWaves * kLanes), 0, reinterpret_cast<hipStream_t>(stream), a);
    return (int)hipGetLastError();
}

}  // namespace usp
