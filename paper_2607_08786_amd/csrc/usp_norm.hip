// usp_norm.hip -- the norms around a block, fused with its gate, residual and
// residual scale, and tokens in 8 bits (include/usp.h, usp_norm and usp_quantize).
//
// Per token, in fp32:   r = residual + scale * act(gate) * post(y),   h = pre(r),
// and for 8-bit tokens  q = rint(h16 * (127 / a)),  a = max |h16|,  h16 = fp16(h).
//
// Every input is read once and every output written once; a few operations per
// byte, so the call is bound by HBM at many tokens and by its launch and one round
// trip to memory at few. One workgroup per token keeps the token in registers
// (C chunks of 8 channels per thread) between the reductions: the mean and then
// the centred sum of squares (a one-pass variance would cancel where the mean is
// large), the maximum. Tokens of more channels than the registers hold are read
// again for every reduction instead.
#include "usp_device.h"
#include "usp_internal.h"

#include <algorithm>

namespace usp {
namespace {

struct NormArgs {
    usp_norm_args p;
    int K;
};

constexpr int kVec = 8;  // channels of a chunk: one 16-byte load of fp16

struct Sum {
    __device__ static float apply(float a, float b) { return a + b; }
};
struct Max {
    __device__ static uint32_t apply(uint32_t a, uint32_t b) { return a > b ? a : b; }
};

// The reduction of v over the workgroup's THREADS threads, in every thread (the
// same bits whatever the wavefronts' timing: fixed pairing, then wavefront order).
// `part` holds one value per wavefront and is not in use on entry.
template <class Op, int THREADS, class T>
__device__ inline T reduce(T v, T *part) {
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) v = Op::apply(v, __shfl_xor(v, o, kLanes));
    if (THREADS == kLanes) return v;
    if ((threadIdx.x & (kLanes - 1)) == 0) part[threadIdx.x / kLanes] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / kLanes; ++w) v = Op::apply(v, part[w]);
    return v;
}

__device__ inline float gate_act(float g, int act) {
    switch (act) {  // uniform
        case USP_GATE_SIGMOID: return 1.f / (1.f + expf(-g));
        case USP_GATE_TANH: return tanhf(g);
        case USP_GATE_SILU: return g / (1.f + expf(-g));
        default: return g;
    }
}

typedef _Float16 half8v __attribute__((ext_vector_type(8)));

// Channels k .. k + 7 of a row of fp16, those < K (the others 0). VEC: 16-byte
// aligned and K a multiple of 8.
template <bool VEC>
__device__ inline half8v load8h(const void *row, int k, int K) {
    const _Float16 *p = reinterpret_cast<const _Float16 *>(row);
    half8v h = {};
    if (VEC) {
        if (k < K) h = *reinterpret_cast<const half8v *>(p + k);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k + i < K) h[i] = p[k + i];
    }
    return h;
}

template <bool VEC>
__device__ inline void load8(const void *row, int k, int K, float (&v)[kVec]) {
    const half8v h = load8h<VEC>(row, k, K);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = (float)h[i];
}

template <bool VEC>
__device__ inline void store8(void *row, int k, int K, const half8v &h) {
    _Float16 *p = reinterpret_cast<_Float16 *>(row);
    if (VEC) {
        if (k < K) *reinterpret_cast<half8v *>(p + k) = h;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k + i < K) p[k + i] = h[i];
    }
}

__device__ inline uint32_t abs_bits(_Float16 h) { return __builtin_bit_cast(uint16_t, h) & 0x7FFFu; }

// 8-bit codes of 8 channels; inv is 0 for tokens whose codes are all 0.
template <bool VEC>
__device__ inline void store_codes(void *row, int k, int K, const half8v &h, float inv) {
    int8_t *p = reinterpret_cast<int8_t *>(row);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        // inv 0 may meet a NaN or an infinity, whose product must not be converted.
        const int c = inv == 0.f ? 0 : (int)rintf((float)h[i] * inv);
        w[i / 4] |= (uint32_t)(uint8_t)c << (8 * (i % 4));
    }
    if (VEC) {
        if (k < K) *reinterpret_cast<uint2 *>(p + k) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (k + i < K) p[k + i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

// Scale and reciprocal of a token's codes from the bits of its largest magnitude.
// fp16 magnitudes order as their bits do, NaN above infinity above all others.
__device__ inline void code_scale(uint32_t top, float &scale, float &inv) {
    const float a = (float)__builtin_bit_cast(_Float16, (uint16_t)top);
    const bool finite = top < 0x7C00u;
    scale = finite ? a / 127.f : __builtin_nanf("");
    inv = finite && top ? 127.f / a : 0.f;
}

// v <- (v - shift) * inv * weight + bias
template <bool VEC>
__device__ inline void scale8(float (&v)[kVec], float shift, float inv, const void *weight, const void *bias, int k,
                              int K) {
    float w[kVec], b[kVec];
    if (weight) load8<VEC>(weight, k, K, w);
    if (bias) load8<VEC>(bias, k, K, b);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        float x = (v[i] - shift) * inv;
        if (weight) x *= w[i];
        if (bias) x += b[i];
        v[i] = x;
    }
}

// r of 8 channels from y's (normed already if a norm is asked for).
template <bool VEC>
__device__ inline void update8(const NormArgs &a, int64_t n, int k, const float (&y)[kVec], float (&r)[kVec]) {
    load8<VEC>(reinterpret_cast<const _Float16 *>(a.p.residual) + n * a.p.ld_residual, k, a.K, r);
    if (!a.p.y) return;
    float g[kVec];
    if (a.p.gate) load8<VEC>(reinterpret_cast<const _Float16 *>(a.p.gate) + n * a.p.ld_gate, k, a.K, g);
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        float v = y[i];
        if (a.p.gate) v *= gate_act(g[i], a.p.gate_activation);
        r[i] += a.p.scale * v;
    }
}

// Mean (layer norm) and 1 / sqrt(mean square of v - mean + eps) of the token whose
// channels thread t holds in v[c] (from channel (c THREADS + t) 8); part: 2 areas.
template <int THREADS, int C>
__device__ inline void moments(const float (&v)[C][kVec], int kind, float eps, int K, float *part, float &shift,
                               float &inv) {
    shift = 0.f;
    if (kind == USP_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) s += v[c][i];
        shift = reduce<Sum, THREADS>(s, part) / (float)K;
    }
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = (c * THREADS + (int)threadIdx.x) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const float d = v[c][i] - shift;
            if (k + i < K) s += d * d;  // channels past the token's end are 0, not the mean
        }
    }
    inv = 1.f / sqrtf(reduce<Sum, THREADS>(s, part + THREADS / kLanes) / (float)K + eps);
}

// v <- (v - shift) * inv * w + b, with w and b at hand where there are any.
__device__ inline void scale8h(float (&v)[kVec], float shift, float inv, bool weight, half8v w, bool bias, half8v b) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        float x = (v[i] - shift) * inv;
        if (weight) x *= (float)w[i];
        if (bias) x += (float)b[i];
        v[i] = x;
    }
}

template <int THREADS, int C, bool VEC>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a) {
    // Every reduction has its own values: no barrier between the end of one and the
    // start of the next.
    __shared__ float part[4][THREADS / kLanes];
    __shared__ uint32_t top_part[THREADS / kLanes];
    const int64_t n = blockIdx.x;
    const int K = a.K, t = threadIdx.x;
    auto at = [&](int c) -> int { return (c * THREADS + t) * kVec; };
    // Everything that comes from HBM is requested first, the vectors of a norm before
    // its reductions: one round trip to memory instead of one behind each reduction
    // (2048 tokens of 5120 channels, layer norms on both sides, a gate: 35.0 us before).
    half8v yh[C], rh[C], gh[C], pw[C], pb[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (a.p.y) yh[c] = load8h<VEC>(reinterpret_cast<const _Float16 *>(a.p.y) + n * a.p.ld_y, at(c), K);
        rh[c] = load8h<VEC>(reinterpret_cast<const _Float16 *>(a.p.residual) + n * a.p.ld_residual, at(c), K);
        if (a.p.gate) gh[c] = load8h<VEC>(reinterpret_cast<const _Float16 *>(a.p.gate) + n * a.p.ld_gate, at(c), K);
        if (a.p.post_kind && a.p.post_weight) pw[c] = load8h<VEC>(a.p.post_weight, at(c), K);
        if (a.p.post_kind && a.p.post_bias) pb[c] = load8h<VEC>(a.p.post_bias, at(c), K);
    }
    float r[C][kVec];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < kVec; ++i) r[c][i] = (float)rh[c][i];
    if (a.p.y) {
        float y[C][kVec];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) y[c][i] = (float)yh[c][i];
        if (a.p.post_kind) {
            float shift, inv;
            moments<THREADS, C>(y, a.p.post_kind, a.p.eps, K, part[0], shift, inv);
#pragma unroll
            for (int c = 0; c < C; ++c) scale8h(y[c], shift, inv, a.p.post_weight, pw[c], a.p.post_bias, pb[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                // Channels past the token's end stay 0 (a bias would make them otherwise).
                float v = at(c) + i < K ? y[c][i] : 0.f;
                if (a.p.gate) v *= gate_act((float)gh[c][i], a.p.gate_activation);
                r[c][i] += a.p.scale * v;
            }
    }
    if (a.p.pre_kind) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (a.p.pre_weight) pw[c] = load8h<VEC>(a.p.pre_weight, at(c), K);
            if (a.p.pre_bias) pb[c] = load8h<VEC>(a.p.pre_bias, at(c), K);
        }
    }
    if (a.p.residual_out) {
        _Float16 *row = reinterpret_cast<_Float16 *>(a.p.residual_out) + n * a.p.ld_residual_out;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            half8v h;
#pragma unroll
            for (int i = 0; i < kVec; ++i) h[i] = (_Float16)r[c][i];
            store8<VEC>(row, (c * THREADS + t) * kVec, K, h);
        }
    }
    if (!a.p.out && !a.p.out_q) return;
    if (a.p.pre_kind) {
        float shift, inv;
        moments<THREADS, C>(r, a.p.pre_kind, a.p.eps, K, part[2], shift, inv);
#pragma unroll
        for (int c = 0; c < C; ++c) scale8h(r[c], shift, inv, a.p.pre_weight, pw[c], a.p.pre_bias, pb[c]);
    }
    half8v h[C];
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int k = (c * THREADS + t) * kVec;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            h[c][i] = (_Float16)r[c][i];
            if (k + i < K) top = Max::apply(top, abs_bits(h[c][i]));
        }
        if (a.p.out) store8<VEC>(reinterpret_cast<_Float16 *>(a.p.out) + n * a.p.ld_out, k, K, h[c]);
    }
    if (!a.p.out_q) return;
    top = reduce<Max, THREADS>(top, top_part);
    float scale, inv;
    code_scale(top, scale, inv);
    if (t == 0) a.p.out_scale[n] = scale;
#pragma unroll
    for (int c = 0; c < C; ++c)
        store_codes<VEC>(reinterpret_cast<int8_t *>(a.p.out_q) + n * a.p.ld_out_q, (c * THREADS + t) * kVec, K, h[c], inv);
}

// Tokens that do not fit the registers: every reduction reads its inputs again and
// computes r again (the same operations, so the same bits); what may lie over an
// input is written last, each channel by the thread that reads it.
constexpr int kLoopThreads = 1024;

__global__ __launch_bounds__(kLoopThreads) void norm_loop_kernel(NormArgs a) {
    __shared__ float part[4][kLoopThreads / kLanes];
    __shared__ uint32_t top_part[kLoopThreads / kLanes];
    const int64_t n = blockIdx.x;
    const int K = a.K, k0 = threadIdx.x * kVec, step = kLoopThreads * kVec;
    float ys = 0.f, yi = 1.f, rs = 0.f, ri = 1.f;  // shift and factor of y and of r
    auto load_y = [&](int k, float(&y)[kVec]) {
        if (a.p.y) load8<false>(reinterpret_cast<const _Float16 *>(a.p.y) + n * a.p.ld_y, k, K, y);
    };
    auto load_r = [&](int k, float(&r)[kVec]) {
        float y[kVec] = {};
        load_y(k, y);
        if (a.p.y && a.p.post_kind) scale8<false>(y, ys, yi, a.p.post_weight, a.p.post_bias, k, K);
        update8<false>(a, n, k, y, r);
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
            m = reduce<Sum, kLoopThreads>(s, area) / (float)K;
        }
        float s = 0.f;
        for (int k = k0; k < K; k += step) {
            float v[kVec] = {};
            load(k, v);
            for (int i = 0; i < kVec; ++i) s += k + i < K ? (v[i] - m) * (v[i] - m) : 0.f;
        }
        inv = 1.f / sqrtf(reduce<Sum, kLoopThreads>(s, area + kLoopThreads / kLanes) / (float)K + a.p.eps);
        shift = m;
    };
    if (a.p.y && a.p.post_kind) loop_moments(load_y, a.p.post_kind, part[0], ys, yi);
    const bool normed = a.p.out || a.p.out_q;
    if (normed && a.p.pre_kind) loop_moments(load_r, a.p.pre_kind, part[2], rs, ri);
    auto load_h = [&](int k, float(&r)[kVec], half8v &h) {  // h from r
        float v[kVec];
        for (int i = 0; i < kVec; ++i) v[i] = r[i];
        if (a.p.pre_kind) scale8<false>(v, rs, ri, a.p.pre_weight, a.p.pre_bias, k, K);
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
            for (int i = 0; i < kVec; ++i) top = k + i < K ? Max::apply(top, abs_bits(h[i])) : top;
        }
        code_scale(reduce<Max, kLoopThreads>(top, top_part), scale, inv);
        if (threadIdx.x == 0) a.p.out_scale[n] = scale;
    }
    for (int k = k0; k < K; k += step) {
        float r[kVec];
        half8v h, r16;
        load_r(k, r);
        for (int i = 0; i < kVec; ++i) r16[i] = (_Float16)r[i];
        if (normed) load_h(k, r, h);
        if (a.p.residual_out)
            store8<false>(reinterpret_cast<_Float16 *>(a.p.residual_out) + n * a.p.ld_residual_out, k, K, r16);
        if (a.p.out) store8<false>(reinterpret_cast<_Float16 *>(a.p.out) + n * a.p.ld_out, k, K, h);
        if (a.p.out_q) store_codes<false>(reinterpret_cast<int8_t *>(a.p.out_q) + n * a.p.ld_out_q, k, K, h, inv);
    }
}

typedef void (*NormKernelFn)(NormArgs);

template <int THREADS, bool VEC>
NormKernelFn norm_kernel_of(int chunks) {
    return chunks <= 1 ? norm_kernel<THREADS, 1, VEC>
         : chunks == 2 ? norm_kernel<THREADS, 2, VEC>
         : chunks == 3 ? norm_kernel<THREADS, 3, VEC>
                       : norm_kernel<THREADS, 4, VEC>;
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
    NormKernelFn fn;
    int threads;
    // Few tokens leave CUs idle: more threads with fewer chunks each then.
    if (chunks <= 256 * (N <= 512 ? 1 : kMaxChunks)) {
        threads = 256;
        const int c = (int)ceil_div(chunks, threads);
        fn = vec ? norm_kernel_of<256, true>(c) : norm_kernel_of<256, false>(c);
    } else if (chunks <= 1024 * kMaxChunks) {
        threads = 1024;
        const int c = (int)ceil_div(chunks, threads);
        fn = vec ? norm_kernel_of<1024, true>(c) : norm_kernel_of<1024, false>(c);
    } else {
        threads = kLoopThreads;
        fn = norm_loop_kernel;
    }
    hipLaunchKernelGGL(fn, dim3((unsigned)N), dim3(threads), 0, st, a);
    return (int)hipGetLastError();
}

}  // namespace usp
