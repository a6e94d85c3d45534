// usp_product.h -- what the kernels of 8-bit products and of products grouped by
// expert share: arguments, the two value formats, and the search for a workgroup's
// part of a ragged batch.
#pragma once
#include <algorithm>

#include "usp_device.h"
#include "usp_internal.h"

namespace usp {

struct ProductArgs {
    ExpertRef one;             // the matrix, when there is no group
    const ExpertRef *experts;  // the group's matrices, or null
    const int32_t *offsets;    // [E + 1]
    int E;
    int64_t M;
    int K, RB, KT;             // K: columns of X in memory
    int sets;                  // row sets of a workgroup's R row blocks
    int job0;                  // the launch's first job
    const uint8_t *X;
    int64_t ldx;               // bytes
    const uint8_t *xp;         // X packed (pack_kernel)
    int64_t x_rows;
    const int32_t *rows;       // row of X for each row of Y, or null
    const float *xs;           // scales of 8-bit rows, or null
    const int32_t *xs_rows;    // the scale's index for each row of Y, or null
    int64_t xs_count;
    const float *weight;       // factor of each row of Y, or null
    uint16_t *Y;
    int64_t ldy;
    int N;                     // rows of Y
    int y_vec, y_wide;         // rows 4 (8) a multiple of 4 (8) apart may be stored as one 8-byte (16-byte) vector
    const uint16_t *bias, *res;
    int64_t ldb, ldr;
    int act, e_flags;
};

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));

// ---- Records of 8-bit values (usp_format.h)
//
// Four prefix scans over pairs of 16-bit fields give every lane the start of its
// values in all 8 blocks, the blocks' own starts coming with the record. Per mask
// byte (8 positions): three LDS dwords hold its up to 8 values whatever their
// alignment, two funnel shifts align them, and two byte permutes place them (or
// zeros) by the selectors of a table of all 256 masks. About 110 VALU and 34 LDS
// instructions per record; with nibble blocks as in fp16 records (twice the
// offsets, a selector of 16 entries per nibble, block sums in scalar code) it was
// 175, 49 and 97 scalar ones, and what bounds a decode is its instructions: 70B
// FFN at 16 tokens 32.4 us.

// Selectors of mask byte n: output byte j takes the value of its rank when bit j is
// set and zero (0x0c) otherwise.
__device__ inline uint2 byte_selectors(uint32_t n) {
    uint32_t sel[2] = {0x0c0c0c0cu, 0x0c0c0c0cu}, r = 0;
    for (int j = 0; j < 8; ++j)
        if (n & (1u << j)) sel[j / 4] = (sel[j / 4] & ~(0xFFu << (8 * (j % 4)))) | (r++ << (8 * (j % 4)));
    return make_uint2(sel[0], sel[1]);
}

struct RecStateQ {
    uint32_t at[4];  // LDS byte offsets of the lane's values: blocks (0, 2), (1, 3), (4, 6), (5, 7) in 16-bit halves
    uint2 msk;
};

// start: LDS byte offset of the record from the region that read_step_q is given,
// below 2^16 - 8192.
__device__ inline RecStateQ rec_state_q(uint2 msk, v4u32 starts, uint32_t start) {
    RecStateQ o;
    o.msk = msk;
    const uint32_t m[2] = {msk.x, msk.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t n = nibble_popcounts(m[i]);
        const uint32_t b = (n + (n >> 4)) & 0x0F0F0F0Fu;
        const uint32_t w[2] = {b & 0x00FF00FFu, (b >> 8) & 0x00FF00FFu};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t inc = wave_inclusive_scan(w[h]);
            asm("" : "+v"(inc));  // keeps the scan's last add a DPP add
            o.at[2 * i + h] = inc + starts[2 * i + h] + (start * 0x00010001u - w[h]);
        }
    }
    return o;
}

struct StepWordsQ {
    uint32_t e[6];
    uint2 sel[2];
    uint32_t hb[2];
};

// Issues the LDS reads of step s of the staged record.
__device__ inline StepWordsQ read_step_q(lds_u32 *region, const uint8_t *lut, const RecStateQ &rs, int s) {
    typedef const __attribute__((address_space(3))) uint8_t lds_u8;
    typedef volatile const __attribute__((address_space(3))) uint32_t lds_vu32;
    StepWordsQ w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int y = 2 * s + h;
        const uint32_t at = rs.at[2 * (y / 4) + y % 2], m = y < 4 ? rs.msk.x : rs.msk.y;
        w.hb[h] = (y & 2) ? at >> 16 : at;  // the low half's other bits are not looked at
        lds_vu32 *d = (lds_vu32 *)((lds_u8 *)region + (w.hb[h] & 0xFFFCu));
        w.e[3 * h] = d[0];
        w.e[3 * h + 1] = d[1];
        w.e[3 * h + 2] = d[2];
        w.sel[h] = *reinterpret_cast<const uint2 *>(lut + 8 * ((m >> (8 * (y % 4))) & 0xFFu));
    }
    return w;
}

// The A operand (16 bytes) of a step from its LDS words.
__device__ inline v4u32 finish_step_q(const StepWordsQ &w) {
    v4u32 a;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t x0 = __builtin_amdgcn_alignbyte(w.e[3 * h + 1], w.e[3 * h], w.hb[h]);  // uses hb & 3
        const uint32_t x1 = __builtin_amdgcn_alignbyte(w.e[3 * h + 2], w.e[3 * h + 1], w.hb[h]);
        a[2 * h] = __builtin_amdgcn_perm(x1, x0, w.sel[h].x);
        a[2 * h + 1] = __builtin_amdgcn_perm(x1, x0, w.sel[h].y);
    }
    return a;
}

// fp16 values: products of 16 rows x 32 columns with fp32 sums.
struct ValuesF16 {
    static constexpr int kBytes = 2, kStepsPerTile = kSteps, kLutEntries = 16;
    typedef StepWords Words;
    typedef RecState State;
    typedef floatx4 Acc;
    __device__ static uint2 selectors(int i) { return nibble_selectors((uint32_t)i); }
    // The record at `slot`, `start` bytes into the region.
    __device__ static State state(const uint8_t *slot, int lane, uint32_t start) {
        return rec_state(slot_mask(slot, lane), start + kMaskBytes);
    }
    __device__ static Words read(lds_u32 *region, const uint8_t *lut, const State &rs, int s) {
        return read_step(region, lut, rs, s);
    }
    __device__ static v4u32 finish(const Words &w) { return __builtin_bit_cast(v4u32, finish_step(w)); }
    __device__ static Acc multiply(v4u32 a, v4u32 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
    }
    __device__ static floatx4 sum(Acc v) { return v; }
};

// 8-bit values: 16 rows x 64 columns with exact 32-bit integer sums.
struct ValuesQ {
    static constexpr int kBytes = 1, kStepsPerTile = kStepsQ, kLutEntries = 256;
    typedef StepWordsQ Words;
    typedef RecStateQ State;
    typedef intx4 Acc;
    __device__ static uint2 selectors(int i) { return byte_selectors((uint32_t)i); }
    __device__ static State state(const uint8_t *slot, int lane, uint32_t start) {
        typedef const __attribute__((address_space(3))) v4u32 lds_v4;
        const v4u32 starts = *(lds_v4 *)(const __attribute__((address_space(3))) void *)(slot + kMaskBytes);
        return rec_state_q(slot_mask(slot, lane), starts, start);
    }
    __device__ static Words read(lds_u32 *region, const uint8_t *lut, const State &rs, int s) {
        return read_step_q(region, lut, rs, s);
    }
    __device__ static v4u32 finish(const Words &w) { return finish_step_q(w); }
    __device__ static Acc multiply(v4u32 a, v4u32 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, a), __builtin_bit_cast(intx4, b), c, 0, 0, 0);
    }
    __device__ static floatx4 sum(Acc v) { return floatx4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}; }
};

// Waits until at most n loads are outstanding (they complete in order). Stated where a
// record's transfer must have ended: the compiler's own waits for transfers into LDS
// go by what it knows of each read, and it has left one out.
template <int N>
__device__ inline void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N < 63 ? N : 63) : "memory");
}

// Fills the selector table with `threads` threads.
template <class V>
__device__ inline void fill_lut(uint8_t *lut, int thread, int threads) {
    for (int i = thread; i < V::kLutEntries; i += threads) reinterpret_cast<uint2 *>(lut)[i] = V::selectors(i);
}

// A workgroup's part: row set `set` of expert e for rows [row0, row0 + n), whose X
// packed in blocks of 16 rows (pack_kernel) starts at block tb.
struct Job {
    int e, set, row0, n, tb;
};
constexpr int kBlock = 16;  // tokens of an MFMA operand

// Inclusive scans over the wavefront's lanes.
__device__ inline int scan_max(int v, int lane) {
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) {
        const int u = __shfl_up(v, o, kLanes);
        if (lane >= o) v = v > u ? v : u;
    }
    return v;
}
__device__ inline int scan_sum(int v, int lane) {
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) {
        const int u = __shfl_up(v, o, kLanes);
        if (lane >= o) v += u;
    }
    return v;
}

// Rows of expert c0 + lane (empty past the last one); run: the end of the rows
// before c0, replaced by the end of these. Offsets are taken into [0, N] and made
// non-decreasing, so every row has at most one expert whatever they hold.
__device__ inline void expert_rows(const ProductArgs &a, int c0, int lane, int &run, int &lo, int &hi) {
    const int e = c0 + lane;
    int v = e < a.E ? a.offsets[e + 1] : 0;
    v = v < 0 ? 0 : v > a.N ? a.N : v;
    v = scan_max(v, lane);
    hi = v > run ? v : run;
    lo = __shfl_up(hi, 1, kLanes);
    if (lane == 0) lo = run;
    run = __builtin_amdgcn_readlane(hi, kLanes - 1);
}

__device__ inline int first_row(const ProductArgs &a) {
    const int v = __builtin_amdgcn_readfirstlane(a.offsets[0]);
    return v < 0 ? 0 : v > a.N ? a.N : v;
}

// Job `b` of the grid, in wavefront-uniform registers; false past the last one.
// An expert with n rows has ceil(n / TB) groups of at most TB rows, and sets x
// groups jobs, the groups of a row set next to each other.
template <int TB>
__device__ inline bool find_job(const ProductArgs &a, int b, int sets, int lane, Job &j) {
    if (!a.experts) {
        const int groups = (a.N + TB - 1) / TB;
        j.e = 0;
        j.set = b / groups;
        j.row0 = b % groups * TB;
        j.n = a.N - j.row0 < TB ? a.N - j.row0 : TB;
        j.tb = j.row0 / kBlock;
        return j.set < sets;
    }
    int run = first_row(a), blocks = 0;
    for (int c0 = 0; c0 < a.E; c0 += kLanes) {
        int lo, hi;
        expert_rows(a, c0, lane, run, lo, hi);
        const int jobs = (hi - lo + TB - 1) / TB * sets, mine = (hi - lo + kBlock - 1) / kBlock;
        const int end = scan_sum(jobs, lane), tb = scan_sum(mine, lane);
        const uint64_t past = __ballot(b < end);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int r0 = __builtin_amdgcn_readlane(lo, l), r1 = __builtin_amdgcn_readlane(hi, l);
            const int at = b - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(jobs, l));
            const int groups = (r1 - r0 + TB - 1) / TB;
            j.e = c0 + l;
            j.set = at / groups;
            const int first = at % groups * TB;
            j.row0 = r0 + first;
            j.n = r1 - j.row0 < TB ? r1 - j.row0 : TB;
            j.tb = blocks + __builtin_amdgcn_readlane(tb, l) - __builtin_amdgcn_readlane(mine, l) + first / kBlock;
            return true;
        }
        b -= __builtin_amdgcn_readlane(end, kLanes - 1);
        blocks += __builtin_amdgcn_readlane(tb, kLanes - 1);
    }
    return false;
}

// The job's matrix, in scalar registers: buffer resources are made of its pointers,
// and a resource that is not known to be uniform costs a loop at every load.
__device__ inline ExpertRef job_matrix(const ProductArgs &a, const Job &j) {
    if (!a.experts) return a.one;
    const uint32_t *p = reinterpret_cast<const uint32_t *>(a.experts + j.e);
    auto word = [&](int i) -> uint64_t { return (uint32_t)__builtin_amdgcn_readfirstlane((int)p[i]); };
    ExpertRef r;
    r.stream = reinterpret_cast<const uint8_t *>(word(0) | word(1) << 32);
    r.off = reinterpret_cast<const uint32_t *>(word(2) | word(3) << 32);
    r.scale = reinterpret_cast<const float *>(word(4) | word(5) << 32);
    return r;
}

// Scale of the 8-bit row of X that row n of Y multiplies; 0 for a row of zeros.
__device__ inline float token_scale(const ProductArgs &a, int n) {
    const int64_t x = a.xs_rows ? a.xs_rows[n] : n;
    return x >= 0 && x < a.xs_count ? a.xs[x] : 0.f;
}

// bias, activation, residual. The activations by the exponential and reciprocal
// instructions: gelu(v) = v / (1 + exp(-2 u)), the tanh form's 0.5 (1 + tanh(u)), and
// silu(v) = v / (1 + exp(-v)). An exponent's rounding moves the result by at most
// 2^-23 |v| (x exp(-x) < 0.37). With the library's tanhf the activations of 13B FFN up
// at 1024 tokens took 7.6 us more (93.2 against 85.6): all workgroups of a round come to them at once.
__device__ inline floatx4 product_epilogue(const ProductArgs &a, floatx4 v, uint2 bias, uint2 res) {
    if (a.bias) v = add_quad(v, bias);
    if (a.act == USP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_elementwise_maximum(v[i], 0.f);  // a NaN stays
    } else if (a.act != USP_ACT_NONE) {
        constexpr float kLog2e = 1.4426950408889634f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float e = a.act == USP_ACT_SILU ? v[i] : 1.5957691216057308f * (v[i] + 0.044715f * v[i] * v[i] * v[i]);
            v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * e));
        }
    }
    if (a.res) v = add_quad(v, res);
    return v;
}

// Four outputs from their sums, rounded to fp16: scales, the fused epilogue and the
// row's factor, the operands at hand.
template <class V>
__device__ inline uint2 finished_quad(const ProductArgs &a, typename V::Acc acc, floatx4 ws, float xs, uint2 bias,
                                      uint2 res, float weight) {
    typedef _Float16 half4 __attribute__((ext_vector_type(4)));
    floatx4 v = V::sum(acc);
    if (V::kBytes == 1) {
        // The product of finite scales, held within fp32: a sum of zero times an overflow would be no
        // zero (any other sum's is fp16's too). An infinite scale stays one, and gives NaN with a sum of
        // zero; a token's NaN, which the holding loses, comes back with the addition.
        // (A select for each sum of zero took 1.1 us of the 83 of 13B FFN up at 1024 tokens with GELU, this 0.5.)
        constexpr float kMost = 3.40282347e38f;
        const float most = fabsf(xs) <= kMost ? kMost : __builtin_inff(), nan = xs == xs ? 0.f : xs;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(v[i], __builtin_amdgcn_fmed3f(xs * ws[i], -most, most), nan);
    }
    if (a.e_flags & kEpiAny) v = product_epilogue(a, v, bias, res);
    if (a.weight) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= weight;
    }
    return __builtin_bit_cast(uint2, half4{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]});
}

// Stores rows m .. m + 3 of row n of Y, those < M.
__device__ inline void store_quad(const ProductArgs &a, int n, int64_t m, uint2 q) {
    uint16_t *const dst = a.Y + (int64_t)n * a.ldy + m;
    if (a.y_vec && m + 4 <= a.M) {
        *reinterpret_cast<uint2 *>(dst) = q;
    } else {
        if (m < a.M) dst[0] = (uint16_t)q.x;
        if (m + 1 < a.M) dst[1] = (uint16_t)(q.x >> 16);
        if (m + 2 < a.M) dst[2] = (uint16_t)q.y;
        if (m + 3 < a.M) dst[3] = (uint16_t)(q.y >> 16);
    }
}

// Rows m .. m + 3 of row n of Y from their sums (w_scale: the expert's scales, of
// whole row blocks).
template <class V>
__device__ inline void finish_quad(const ProductArgs &a, const float *w_scale, int e, int n, int64_t m,
                                   typename V::Acc acc) {
    const floatx4 ws = V::kBytes == 1 ? *reinterpret_cast<const floatx4 *>(w_scale + m) : floatx4{};
    const float xs = V::kBytes == 1 ? token_scale(a, n) : 0.f, weight = a.weight ? a.weight[n] : 1.f;
    const uint2 bias = load_quad(a.bias ? a.bias + e * a.ldb : nullptr, m, a.M, a.e_flags & kEpiBiasVec);
    store_quad(a, n, m, finished_quad<V>(a, acc, ws, xs, bias, residual_quad(a, n, m), weight));
}

}  // namespace

typedef void (*ProductKernelFn)(ProductArgs);

// The wide kernel (usp_product_wide.hip): column tiles whose records are in LDS; whether
// it is built for records of L KB, R row blocks and NB token blocks per wavefront (of
// 2 and 4; what fits 160 KB of LDS and 256 registers); and the kernel.
constexpr int wide_ring(int L) { return L <= 3 ? 3 : 2; }
constexpr bool wide_serves_rows(int value_bytes, int L, int R, int NB) {
    return 2048 + 8192 * R + wide_ring(L) * (1024 * L * R + 16) <= 160 * 1024 && (R == 4 || NB == 2 || value_bytes == 1);
}
ProductKernelFn wide_product_kernel_of(int value_bytes, int loads, int rows, int nb);

}  // namespace usp
