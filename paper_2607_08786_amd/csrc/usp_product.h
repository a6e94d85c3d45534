// usp_product.h -- what the kernels of 8-bit products and of products grouped by
// expert share: arguments, the two value formats, and the search for a workgroup's
// part of a ragged batch.
#pragma once
#include "usp_device.h"
#include "usp_internal.h"

namespace usp {
namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));

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
    int64_t x_rows;
    const int32_t *rows;       // row of X for each row of Y, or null
    const float *xs;           // scales of 8-bit rows, or null
    const int32_t *xs_rows;    // the scale's index for each row of Y, or null
    int64_t xs_count;
    const float *weight;       // factor of each row of Y, or null
    uint16_t *Y;
    int64_t ldy;
    int N;                     // rows of Y
    int y_vec;
    const uint16_t *bias, *res;
    int64_t ldb, ldr;
    int act, e_flags;
};

// fp16 values: products of 16 rows x 32 columns with fp32 sums.
struct ValuesF16 {
    static constexpr int kBytes = 2, kStepsPerTile = kSteps, kLutBytes = 16 * 8;
    typedef StepWords Words;
    typedef floatx4 Acc;
    __device__ static void fill_lut(uint8_t *lut, int i) {
        reinterpret_cast<uint2 *>(lut)[i] = nibble_selectors((uint32_t)i);
    }
    __device__ static Words read(lds_u32 *region, const uint8_t *lut, const RecState &rs, int s) {
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
    static constexpr int kBytes = 1, kStepsPerTile = kStepsQ, kLutBytes = 16 * 4;
    typedef StepWordsQ Words;
    typedef intx4 Acc;
    __device__ static void fill_lut(uint8_t *lut, int i) {
        reinterpret_cast<uint32_t *>(lut)[i] = nibble_selector_q((uint32_t)i);
    }
    __device__ static Words read(lds_u32 *region, const uint8_t *lut, const RecState &rs, int s) {
        return read_step_q(region, lut, rs, s);
    }
    __device__ static v4u32 finish(const Words &w) { return finish_step_q(w); }
    __device__ static Acc multiply(v4u32 a, v4u32 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, a), __builtin_bit_cast(intx4, b), c, 0, 0, 0);
    }
    __device__ static floatx4 sum(Acc v) { return floatx4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}; }
};

// A workgroup's part: row set `set` of expert e for rows [row0, row0 + n).
struct Job {
    int e, set, row0, n;
};

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
__device__ inline bool find_job(const ProductArgs &a, int b, int lane, Job &j) {
    if (!a.experts) {
        const int groups = (a.N + TB - 1) / TB;
        j.e = 0;
        j.set = b / groups;
        j.row0 = b % groups * TB;
        j.n = a.N - j.row0 < TB ? a.N - j.row0 : TB;
        return j.set < a.sets;
    }
    int run = first_row(a);
    for (int c0 = 0; c0 < a.E; c0 += kLanes) {
        int lo, hi;
        expert_rows(a, c0, lane, run, lo, hi);
        const int jobs = (hi - lo + TB - 1) / TB * a.sets;
        const int end = scan_sum(jobs, lane);
        const uint64_t past = __ballot(b < end);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int r0 = __builtin_amdgcn_readlane(lo, l), r1 = __builtin_amdgcn_readlane(hi, l);
            const int at = b - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(jobs, l));
            const int groups = (r1 - r0 + TB - 1) / TB;
            j.e = c0 + l;
            j.set = at / groups;
            j.row0 = r0 + at % groups * TB;
            j.n = r1 - j.row0 < TB ? r1 - j.row0 : TB;
            return true;
        }
        b -= __builtin_amdgcn_readlane(end, kLanes - 1);
    }
    return false;
}

// The fused epilogue and store of rows m .. m + 3 of row n of Y from their sums.
// e: the expert (its scales w_scale, its bias).
template <class V>
__device__ inline void finish_quad(const ProductArgs &a, const float *w_scale, int e, int n, int64_t m,
                                   typename V::Acc acc) {
    floatx4 v = V::sum(acc);
    if (V::kBytes == 1) {  // w_scale holds whole row blocks
        const int64_t x = a.xs_rows ? a.xs_rows[n] : n;
        const float xs = x >= 0 && x < a.xs_count ? a.xs[x] : 0.f;  // a row of zeros
        const floatx4 ws = *reinterpret_cast<const floatx4 *>(w_scale + m);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= xs * ws[i];
    }
    if (a.e_flags & kEpiAny) {
        const uint2 bq = load_quad(a.bias ? a.bias + e * a.ldb : nullptr, m, a.M, a.e_flags & kEpiBiasVec);
        v = epilogue(a, v, bq, residual_quad(a, n, m));
    }
    if (a.weight) {
        const float w = a.weight[n];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= w;
    }
    store_rounded4(a, n, m, v);
}

}  // namespace
}  // namespace usp
