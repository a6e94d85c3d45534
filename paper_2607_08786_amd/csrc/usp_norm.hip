// usp_norm.hip -- the norms around a block, fused with its gate, residual and
// residual scale, and tokens in 8 bits (include/usp.h, usp_norm and usp_quantize).
//
// Per token, in fp32:   r = residual + scale * act(gate) * post(y),   h = pre(r),
// and for 8-bit tokens  q = rint(h16 * (127 / a)),  a = max |h16|,  h16 = fp16(h).
//
// Every input is read once and every output written once, so the call is bound by HBM
// at many tokens and by its launch and one round trip to memory at few. The vector
// units come close behind HBM (a wavefront's fp32 instruction takes 4 cycles: 20 for a
// channel of 10 bytes are 5 us of 2048 x 5120 tokens), so what a channel costs is kept
// low: selects for a vector, conversions in the products (v_fma_mix). In graphs over
// buffers of 1 GB together, so that all comes from HBM: 2048 x 5120, 105 MB, layer norms
// and a gate 28.2 us (3.7 TB/s), RMS norms and a gate 26.3, a gate alone 22.0 (4.8 TB/s, where
// a copy of as many bytes takes 20.5); RMS before and no gate, 84 MB, 20.3 (4.1). Over one set
// of buffers, much of which the 256 MB cache keeps: 22.5, 20.7, 16.8 and 16.1. There selects
// for each channel cost 5.5 us more. 1 x 8192, RMS: 3.5 us.
//
// One workgroup per token keeps the token in registers (C chunks of 8 channels per
// thread) between the reductions: the mean and then the centred sum of squares (a
// one-pass variance would cancel where the mean is large), the maximum. Tokens of more
// channels than the registers hold are read again for every reduction instead.
#include "usp_codes.h"
#include "usp_device.h"
#include "usp_internal.h"

#include <algorithm>

namespace usp {
namespace {

struct NormArgs {
    usp_norm_args p;
    int K;
};

constexpr int kMaxWaves = 16;  // wavefronts of a workgroup
constexpr int kVec = 8;  // channels of a chunk: one 16-byte load of fp16

struct Sum {
    __device__ static float apply(float a, float b) { return a + b; }
};
struct Max {
    __device__ static uint32_t apply(uint32_t a, uint32_t b) { return a > b ? a : b; }
};

// One step of a wavefront's reduction: v with what the lanes that DPP control CTRL
// names hold (0, the identity of both operations, where it names none).
template <class Op, int CTRL, int ROWS, class T>
__device__ inline T dpp_step(T v) {
    const uint32_t u = __builtin_amdgcn_update_dpp(0u, __builtin_bit_cast(uint32_t, v), CTRL, ROWS, 0xF, ROWS == 0xF);
    return Op::apply(v, __builtin_bit_cast(T, u));
}

// The reduction of v over the workgroup's threads, in every thread (the
// same bits whatever the wavefronts' timing: fixed pairing, then wavefront order).
// Within a wavefront by DPP row shifts and broadcasts, whose last lane holds the
// result. `part` holds one value per wavefront and is not in use on entry.
template <class Op, class T>
__device__ inline T reduce(T v, T *part) {
    v = dpp_step<Op, 0x111, 0xF>(v);  // row_shr:1
    v = dpp_step<Op, 0x112, 0xF>(v);  // row_shr:2
    v = dpp_step<Op, 0x114, 0xF>(v);  // row_shr:4
    v = dpp_step<Op, 0x118, 0xF>(v);  // row_shr:8
    v = dpp_step<Op, 0x142, 0xA>(v);  // row_bcast:15
    v = dpp_step<Op, 0x143, 0xC>(v);  // row_bcast:31
    v = __builtin_bit_cast(T, (uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, v), kLanes - 1));
    if ((threadIdx.x & (kLanes - 1)) == 0) part[threadIdx.x / kLanes] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < (int)blockDim.x / kLanes; ++w) v = Op::apply(v, part[w]);
    return v;
}

typedef _Float16 half8v __attribute__((ext_vector_type(8)));

// A row of K elements of ES bytes as a buffer resource, empty where there is none:
// loads past its end give zeros and stores there do nothing, so neither needs a
// branch. (Behind branches the compiler waited for each of a norm's vectors before
// it requested the next: 28.9 us for 2048 x 5120 with RMS norms and a gate.)
// A resource's base is a multiple of 4 bytes; `sh` is how far the row starts behind it.
// READ: its size is too, so that the dword of the last element is read.
struct Row {
    __amdgpu_buffer_rsrc_t rsrc;
    int sh, n;
};
template <int ES, bool READ = false>
__device__ inline Row row_of(const void *base, int64_t offset, int K, bool there = true) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(base) + offset * ES;
    Row r;
    r.sh = (int)(at & 3);
    r.n = K;
    const int bytes = K * ES + r.sh;
    r.rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(at - r.sh), (short)0,
                                               base && there ? READ ? (bytes + 3) & ~3 : bytes : 0, kBufferRsrcWord3);
    return r;
}

// Channels k .. k + 7 of a row of fp16 (zeros past its end). VEC: 16-byte aligned
// and K a multiple of 8; else five dwords hold them, shifted into place, what follows
// the row in its last dword cleared (a load for each channel took 5.0 us for 21 tokens
// of 4093 channels in 8 bits against 2.8 for aligned ones).
template <bool VEC>
__device__ inline half8v load8h(Row row, int k) {
    v4u32 d = __builtin_bit_cast(v4u32, __builtin_amdgcn_raw_buffer_load_b128(row.rsrc, 2 * k, 0, 0));
    if (!VEC) {
        const uint32_t e = __builtin_amdgcn_raw_buffer_load_b32(row.rsrc, 2 * k + 16, 0, 0);
        const int left = row.n - k;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = __builtin_amdgcn_alignbyte(i < 3 ? d[i < 3 ? i + 1 : 3] : e, d[i], row.sh);
            d[i] = left >= 2 * i + 2 ? w : left == 2 * i + 1 ? w & 0xFFFFu : 0u;
        }
    }
    return __builtin_bit_cast(half8v, d);
}

// Whole chunks of dword-aligned rows in one piece also where K is no multiple of 8.
template <bool VEC>
__device__ inline void store8(Row row, int k, const half8v &h) {
    if (VEC || (row.sh == 0 && k + kVec <= row.n)) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u32, h), row.rsrc, 2 * k, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (_Float16)h[i]), row.rsrc, row.sh + 2 * (k + i), 0, 0);
    }
}

// 8-bit codes of 8 channels; inv is 0 for tokens whose codes are all 0.
template <bool VEC>
__device__ inline void store_codes(Row row, int k, const half8v &h, float inv) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    u32x2 w = {0, 0};
#pragma unroll
    for (int i = 0; i < kVec; ++i) w[i / 4] |= code_bits(h[i], inv) << (8 * (i % 4));
    if (VEC || (row.sh == 0 && k + kVec <= row.n)) {
        __builtin_amdgcn_raw_buffer_store_b64(w, row.rsrc, k, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            __builtin_amdgcn_raw_buffer_store_b8((uint8_t)(w[i / 4] >> (8 * (i % 4))), row.rsrc, row.sh + k + i, 0, 0);
    }
}

// v <- (v - shift) * inv * w + b.
__device__ inline void scale8(float (&v)[kVec], float shift, float inv, half8v w, half8v b) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = fmaf((v[i] - shift) * inv, (float)w[i], (float)b[i]);
}

// A weight or a gate that is not there is 1 (a bias that is not there reads as 0): a
// select for a vector instead of a branch for a channel.
__device__ inline half8v or_ones(bool there, half8v w) {
    const v4u32 one = {0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u};
    return there ? w : __builtin_bit_cast(half8v, one);
}

// act(gate) of 8 channels. One branch for all of them.
// The reciprocal instruction's error is one unit in the last place.
__device__ inline void gate8(float (&g)[kVec], int act) {
    if (act == USP_GATE_NONE) return;
    if (act == USP_GATE_TANH) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) g[i] = tanhf(g[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float s = __builtin_amdgcn_rcpf(1.f + expf(-g[i]));
        g[i] = act == USP_GATE_SILU ? g[i] * s : s;
    }
}

__device__ inline void to_float(half8v h, float (&v)[kVec]) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = (float)h[i];
}

// r += scale * act(gate) * y for the channels < K (past the token's end r stays 0,
// which y after a norm's bias would change).
template <bool VEC>
__device__ inline void update8(const NormArgs &a, int k, const float (&y)[kVec], half8v gate, float (&r)[kVec]) {
    float g[kVec];
    to_float(or_ones(a.p.gate, gate), g);
    gate8(g, a.p.gate ? a.p.gate_activation : USP_GATE_NONE);
    if (VEC && k >= a.K) return;
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (VEC || k + i < a.K) r[i] = fmaf(a.p.scale, y[i] * g[i], r[i]);
}

// The rows of a token.
struct Rows {
    Row y, residual, gate, post_weight, post_bias, pre_weight, pre_bias;
    __device__ Rows(const NormArgs &a, int64_t n)
        : y(row_of<2, true>(a.p.y, n * a.p.ld_y, a.K)),
          residual(row_of<2, true>(a.p.residual, n * a.p.ld_residual, a.K)),
          gate(row_of<2, true>(a.p.gate, n * a.p.ld_gate, a.K)),
          post_weight(row_of<2, true>(a.p.post_weight, 0, a.K, a.p.post_kind)),
          post_bias(row_of<2, true>(a.p.post_bias, 0, a.K, a.p.post_kind)),
          pre_weight(row_of<2, true>(a.p.pre_weight, 0, a.K, a.p.pre_kind)),
          pre_bias(row_of<2, true>(a.p.pre_bias, 0, a.K, a.p.pre_kind)) {}
};

// Mean (layer norm) and 1 / sqrt(mean square of v - mean + eps) of the token whose
// channels thread t holds in v[c] (from channel (c threads + t) 8); part: 2 areas.
template <int C, bool VEC>
__device__ inline void moments(const float (&v)[C][kVec], int kind, float eps, int K, float *part, float &shift,
                               float &inv) {
    shift = 0.f;
    if (kind == USP_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) s += v[c][i];
        shift = reduce<Sum>(s, part) / (float)K;
    }
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = (c * (int)blockDim.x + (int)threadIdx.x) * kVec;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = v[c][i] - shift;
            if (VEC || k + i < K) q = fmaf(d, d, q);  // channels past the token's end are 0, not the mean
        }
        s += !VEC || k < K ? q : 0.f;
    }
    inv = 1.f / sqrtf(reduce<Sum>(s, part + kMaxWaves) / (float)K + eps);
}

template <int MOST, int C, bool VEC>
__global__ __launch_bounds__(MOST) void norm_kernel(NormArgs a) {
    // Every reduction has its own values: no barrier between the end of one and the
    // start of the next.
    __shared__ float part[4][kMaxWaves];
    __shared__ uint32_t top_part[kMaxWaves];
    const int64_t n = blockIdx.x;
    const int K = a.K, t = threadIdx.x, threads = blockDim.x;
    auto at = [&](int c) -> int { return (c * threads + t) * kVec; };
    // Everything that comes from HBM is requested first, the vectors of a norm before
    // its reductions: one round trip to memory instead of one behind each reduction.
    const Rows rows(a, n);
    half8v yh[C], rh[C], gh[C], pw[C], pb[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        yh[c] = load8h<VEC>(rows.y, at(c));
        rh[c] = load8h<VEC>(rows.residual, at(c));
        gh[c] = load8h<VEC>(rows.gate, at(c));
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        pw[c] = load8h<VEC>(rows.post_weight, at(c));
        pb[c] = load8h<VEC>(rows.post_bias, at(c));
    }
    float r[C][kVec];
    if (a.p.y) {
        float y[C][kVec];
#pragma unroll
        for (int c = 0; c < C; ++c) to_float(yh[c], y[c]);
        if (a.p.post_kind) {
            float shift, inv;
            moments<C, VEC>(y, a.p.post_kind, a.p.eps, K, part[0], shift, inv);
#pragma unroll
            for (int c = 0; c < C; ++c) scale8(y[c], shift, inv, or_ones(a.p.post_weight, pw[c]), pb[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            to_float(rh[c], r[c]);
            update8<VEC>(a, at(c), y[c], gh[c], r[c]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) to_float(rh[c], r[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        pw[c] = load8h<VEC>(rows.pre_weight, at(c));
        pb[c] = load8h<VEC>(rows.pre_bias, at(c));
    }
    if (a.p.residual_out) {
        const Row row = row_of<2>(a.p.residual_out, n * a.p.ld_residual_out, K);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            half8v h;
#pragma unroll
            for (int i = 0; i < kVec; ++i) h[i] = (_Float16)r[c][i];
            store8<VEC>(row, at(c), h);
        }
    }
    if (!a.p.out && !a.p.out_q) return;
    if (a.p.pre_kind) {
        float shift, inv;
        moments<C, VEC>(r, a.p.pre_kind, a.p.eps, K, part[2], shift, inv);
#pragma unroll
        for (int c = 0; c < C; ++c) scale8(r[c], shift, inv, or_ones(a.p.pre_weight, pw[c]), pb[c]);
    }
    half8v h[C];
    const Row out = row_of<2>(a.p.out, n * a.p.ld_out, K);
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) h[c][i] = (_Float16)r[c][i];
        store8<VEC>(out, at(c), h[c]);
    }
    if (!a.p.out_q) return;
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (VEC || at(c) + i < K) m = Max::apply(m, magnitude_bits(h[c][i]));
        top = Max::apply(top, !VEC || at(c) < K ? m : 0);
    }
    top = reduce<Max>(top, top_part);
    float scale, inv;
    code_scale(top, scale, inv);
    if (t == 0) a.p.out_scale[n] = scale;
    const Row codes = row_of<1>(a.p.out_q, n * a.p.ld_out_q, K);
#pragma unroll
    for (int c = 0; c < C; ++c) store_codes<VEC>(codes, at(c), h[c], inv);
}

// Tokens that do not fit the registers: every reduction reads its inputs again and
// computes r again (the same operations, so the same bits); what may lie over an
// input is written last, each channel by the thread that reads it.
constexpr int kLoopThreads = 1024;

__global__ __launch_bounds__(kLoopThreads) void norm_loop_kernel(NormArgs a) {
    __shared__ float part[4][kMaxWaves];
    __shared__ uint32_t top_part[kMaxWaves];
    const int64_t n = blockIdx.x;
    const int K = a.K, k0 = threadIdx.x * kVec, step = kLoopThreads * kVec;
    float ys = 0.f, yi = 1.f, rs = 0.f, ri = 1.f;  // shift and factor of y and of r
    const Rows rows(a, n);
    auto load_y = [&](int k, float(&y)[kVec]) { to_float(load8h<false>(rows.y, k), y); };
    auto load_r = [&](int k, float(&r)[kVec]) {
        to_float(load8h<false>(rows.residual, k), r);
        if (!a.p.y) return;
        float y[kVec];
        load_y(k, y);
        if (a.p.post_kind)
            scale8(y, ys, yi, or_ones(a.p.post_weight, load8h<false>(rows.post_weight, k)), load8h<false>(rows.post_bias, k));
        update8<false>(a, k, y, load8h<false>(rows.gate, k), r);
    };
    auto loop_moments = [&](auto load, int kind, float *area, float &shift, float &inv) {
        float m = 0.f;
        if (kind == USP_NORM_LAYER) {
            float s = 0.f;
            for (int k = k0; k < K; k += step) {
                float v[kVec] = {};
                load(k, v);
                for (int i = 0; i < kVec; ++i) s += k + i < K ? v[i] : 0.f;
            }
            m = reduce<Sum>(s, area) / (float)K;
        }
        float s = 0.f;
        for (int k = k0; k < K; k += step) {
            float v[kVec] = {};
            load(k, v);
            for (int i = 0; i < kVec; ++i) s += k + i < K ? (v[i] - m) * (v[i] - m) : 0.f;
        }
        inv = 1.f / sqrtf(reduce<Sum>(s, area + kMaxWaves) / (float)K + a.p.eps);
        shift = m;
    };
    if (a.p.y && a.p.post_kind) loop_moments(load_y, a.p.post_kind, part[0], ys, yi);
    const bool normed = a.p.out || a.p.out_q;
    if (normed && a.p.pre_kind) loop_moments(load_r, a.p.pre_kind, part[2], rs, ri);
    auto load_h = [&](int k, float(&r)[kVec], half8v &h) {  // h from r
        float v[kVec];
        for (int i = 0; i < kVec; ++i) v[i] = r[i];
        if (a.p.pre_kind)
            scale8(v, rs, ri, or_ones(a.p.pre_weight, load8h<false>(rows.pre_weight, k)), load8h<false>(rows.pre_bias, k));
        for (int i = 0; i < kVec; ++i) h[i] = (_Float16)v[i];
    };
    float scale = 0.f, inv = 0.f;
    if (a.p.out_q) {
        uint32_t top = 0;
        for (int k = k0; k < K; k += step) {
            float r[kVec];
            half8v h;
            load_r(k, r);
            load_h(k, r, h);
            for (int i = 0; i < kVec; ++i) top = k + i < K ? Max::apply(top, magnitude_bits(h[i])) : top;
        }
        code_scale(reduce<Max>(top, top_part), scale, inv);
        if (threadIdx.x == 0) a.p.out_scale[n] = scale;
    }
    for (int k = k0; k < K; k += step) {
        float r[kVec];
        half8v h, r16;
        load_r(k, r);
        for (int i = 0; i < kVec; ++i) r16[i] = (_Float16)r[i];
        if (normed) load_h(k, r, h);
        store8<false>(row_of<2>(a.p.residual_out, n * a.p.ld_residual_out, K), k, r16);
        if (a.p.out) store8<false>(row_of<2>(a.p.out, n * a.p.ld_out, K), k, h);
        if (a.p.out_q) store_codes<false>(row_of<1>(a.p.out_q, n * a.p.ld_out_q, K), k, h, inv);
    }
}

typedef void (*NormKernelFn)(NormArgs);

template <int MOST, bool VEC>
NormKernelFn norm_kernel_of(int chunks) {
    return chunks <= 1 ? norm_kernel<MOST, 1, VEC>
         : chunks == 2 ? norm_kernel<MOST, 2, VEC>
         : chunks == 3 ? norm_kernel<MOST, 3, VEC>
                       : norm_kernel<MOST, 4, VEC>;
}

constexpr int kMaxChunks = 4;

}  // namespace

int launch_norm(const usp_norm_args &p, int64_t N, int64_t K, void *stream) {
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    NormArgs a = {p, (int)K};
    auto aligned = [](const void *q, int64_t ld, int64_t bytes) {
        return !q || ((reinterpret_cast<uintptr_t>(q) & (8 * bytes - 1)) == 0 && ld % 8 == 0);
    };
    const bool vec = K % 8 == 0 && aligned(p.residual, p.ld_residual, 2) && aligned(p.y, p.ld_y, 2) &&
                     aligned(p.gate, p.ld_gate, 2) && aligned(p.residual_out, p.ld_residual_out, 2) &&
                     aligned(p.out, p.ld_out, 2) && aligned(p.out_q, p.ld_out_q, 1) && aligned(p.post_weight, 0, 2) &&
                     aligned(p.post_bias, 0, 2) && aligned(p.pre_weight, 0, 2) && aligned(p.pre_bias, 0, 2);
    const int64_t chunks = ceil_div(K, kVec);
    // Chunks per thread, then as many whole wavefronts as they need. Many tokens: about
    // five wavefronts each (2048 x 5120, layer norms and a gate: 27.1 us; one chunk per
    // thread 30.0, three wavefronts 26.5, and 36.9 against 35.7 at 4096 x 4096); few
    // leave CUs idle, so one chunk per thread.
    constexpr int kMost = 512;
    NormKernelFn fn = norm_loop_kernel;
    int64_t threads = kLoopThreads;
    if (chunks <= (int64_t)kLoopThreads * kMaxChunks) {
        const int64_t c = std::max(ceil_div(chunks, (int64_t)kLoopThreads),
                                   N > 512 ? std::min<int64_t>(kMaxChunks, ceil_div(chunks, (int64_t)320)) : 1);
        threads = ceil_div(ceil_div(chunks, c), (int64_t)kLanes) * kLanes;
        fn = threads <= kMost ? vec ? norm_kernel_of<kMost, true>((int)c) : norm_kernel_of<kMost, false>((int)c)
             : vec            ? norm_kernel_of<kLoopThreads, true>((int)c)
                              : norm_kernel_of<kLoopThreads, false>((int)c);
    }
    hipLaunchKernelGGL(fn, dim3((unsigned)N), dim3((unsigned)threads), 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace usp
