// usp_product_wide.hip -- products on 8-bit values and products grouped by expert
// over many tokens (X packed first).
#include "usp_product.h"

namespace usp {
namespace {

constexpr int kGroup = 4;  // steps that one of the two operand buffers holds

// ---------------------------------------------------------------------------
// A workgroup of R wavefronts takes R row blocks and R NB blocks of 16 tokens.
// Wavefront j decodes row block j of every column tile into LDS, once for all the
// workgroup's tokens, and multiplies all rows by its own NB blocks of tokens, X read
// from the packed copy a group of steps ahead.
//
// What bounds it is neither HBM nor the matrix rate but how a SIMD's two wavefronts
// share it: a record's decode takes a wavefront 2050-2200 cycles (LDS round trips and
// about 150 VALU instructions), the products of a tile of 8-bit values with 64 tokens
// and 128 rows 2700 (128 MFMAs of 16 cycles, and the waits for A operands in LDS). They
// are not interleaved within a wavefront (no gain: a wavefront issues in order) but
// between the two of a SIMD: with 8 row blocks wavefronts j and j + 4 do their two
// parts in opposite order, with 4 two workgroups share a CU. 13B FFN up, 8-bit, us:
//
//   tokens   R=4 NB=2   R=4 NB=4   R=8 NB=2   R=8 NB=4
//   256        39.3       39.0       47.2       70.3
//   512        71.0       51.3       53.3       72.9
//   1024      124.5       96.1       93.9       75.3
//
// Four wavefronts that only decode and four that only multiply: 61 at 256 tokens and
// 118 at 1024 (a decoding wavefront has two records then); eight and eight: 46 and 95.
// ---------------------------------------------------------------------------
template <class V, int L, int R, int NB>
__global__ __launch_bounds__(R *kLanes, 2) void wide_product_kernel(ProductArgs a) {
    constexpr int S = V::kStepsPerTile, G = S / kGroup, TB = kBlock * NB * R;
    constexpr int kStepBytes = R * kLanes * 16;
    constexpr int kSlot = 1024 * L, kRing = wide_ring(L), kBuf = kGroup * kStepBytes;
    constexpr int kLut = V::kLutEntries * 8 > 1024 ? V::kLutEntries * 8 : 1024;  // the selector table, at the start of LDS
    // A wavefront's sums of a block of tokens on their way to Y: 128 rows each, 16 bytes
    // between the tokens' rows against bank conflicts.
    constexpr int kSumRow = 4 * R * kTileRows + 16, kSumBytes = kBlock * kSumRow;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[kLut + 2 * kBuf > R * kSumBytes ? kLut + 2 * kBuf : R * kSumBytes];
    __shared__ __attribute__((aligned(16))) uint8_t slot0[R * kSlot + 16], slot1[R * kSlot + 16],
        slot2[kRing > 2 ? R * kSlot + 16 : 16];
    uint8_t *const lut = smem, *const abuf = smem + kLut;
    uint8_t *const slots[3] = {slot0, slot1, slot2};
    const int lane = threadIdx.x & (kLanes - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    Job job;
    if (!find_job<TB>(a, a.job0 + (int)blockIdx.x, a.sets, lane, job)) return;  // the whole workgroup
    const ExpertRef ref = job_matrix(a, job);
    fill_lut<V>(lut, threadIdx.x, R * kLanes);

    const int rb = job.set * R + wave;
    const __amdgpu_buffer_rsrc_t offr = __builtin_amdgcn_make_buffer_rsrc(
        (void *)ref.off, (short)0, (a.RB * a.KT + 1) * 4, kBufferRsrcWord3);
    uint32_t off = 0;  // lane l: the offset of tile 63 c + l of the row block
    auto request = [&](int kt, uint8_t *slot) __attribute__((always_inline)) {
        if (kt % 63 == 0)
            off = __builtin_amdgcn_raw_buffer_load_b32(
                offr, rb < a.RB && kt + lane <= a.KT ? (rb * a.KT + kt + lane) * 4 : 0x7FFFFFF0, 0, 0);
        const bool real = kt < a.KT;
        const uint32_t o0 = real ? __builtin_amdgcn_readlane(off, kt % 63) : 0;
        const uint32_t o1 = real ? __builtin_amdgcn_readlane(off, kt % 63 + 1) : 0;
        const __amdgpu_buffer_rsrc_t rec = __builtin_amdgcn_make_buffer_rsrc(
            (void *)(ref.stream + (uint64_t)o0 * 16), (short)0, (int)((o1 - o0) * 16), kBufferRsrcWord3);
#pragma unroll
        for (int l = 0; l < L; ++l)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rec, (__attribute__((address_space(3))) void *)(slot + wave * kSlot + 1024 * l), 16, 1024 * l + lane * 16, 0,
                0, 0);
    };
    const int steps = a.KT * S;
    const int64_t block = (int64_t)steps << 10;
    const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(a.xp + (job.tb + wave * NB) * block), (short)0, (int)(NB * block), kBufferRsrcWord3);
    auto load_x = [&](int step, v4u32(&x)[NB]) __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            x[nb] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)(nb * block) + 16 * lane, step << 10, 0);
    };

    const int mine = wave * NB * kBlock + lane;
    const bool token = lane < NB * kBlock && mine < job.n;
    const float xs = V::kBytes == 1 && token ? token_scale(a, job.row0 + mine) : 0.f;
    const float weight = a.weight && token ? a.weight[job.row0 + mine] : 1.f;
    typename V::Acc acc[R][NB] = {};
    v4u32 xb[kGroup][NB];
    typename V::State rs;
    // Steps g kGroup .. of tile kt, whose record is in `slot`, into operand buffer `buf`;
    // with the tile's last steps its slot is free for tile kt + kRing.
    auto decode = [&](int kt, int g, uint8_t *slot, int buf) __attribute__((always_inline)) {
        if (g == 0) {
            // Since this record at least the other slots' records and a group's X have been
            // requested, on every path.
            wait_loads<(kRing - 1) * L + kGroup * NB>();
            rs = V::state(slot + wave * kSlot, lane, (uint32_t)(wave * kSlot));
        }
        typename V::Words w = V::read(as_lds(slot), lut, rs, g * kGroup);
#pragma unroll
        for (int s = 0; s < kGroup; ++s) {
            typename V::Words wn;
            if (s + 1 < kGroup) wn = V::read(as_lds(slot), lut, rs, g * kGroup + s + 1);
            *reinterpret_cast<v4u32 *>(abuf + buf * kBuf + s * kStepBytes + wave * 1024 + lane * 16) = V::finish(w);
            if (s + 1 < kGroup) w = wn;
        }
        if (g == G - 1) request(kt + kRing, slot);
    };
    // Products of the kGroup steps from `step` on, their operands in buffer `buf`: four
    // row blocks' operands are read half a step ahead.
    auto products = [&](int step, int buf) __attribute__((always_inline)) {
        constexpr int H = R / 2;
        const uint8_t *const from = abuf + buf * kBuf + lane * 16;
        v4u32 av[2][H];
        auto read_a = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < H; ++r)
                av[i % 2][r] = *reinterpret_cast<const v4u32 *>(from + i / 2 * kStepBytes + (i % 2 * H + r) * 1024);
        };
        read_a(0);
        static_for(
            [&](auto ic) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value, s = i / 2;
                __builtin_amdgcn_sched_barrier(0);
                if (i + 1 < 2 * kGroup) read_a(i + 1);
#pragma unroll
                for (int r = 0; r < H; ++r)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        acc[i % 2 * H + r][nb] = V::multiply(av[i % 2][r], xb[s][nb], acc[i % 2 * H + r][nb]);
                if (i % 2 == 1) load_x(step + kGroup + s, xb[s]);
            },
            std::make_integer_sequence<int, 2 * kGroup>{});
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int i = 0; i < kRing; ++i) request(i, slots[i]);
    asm volatile("" ::: "memory");  // X after the records, as decode()'s wait counts them
#pragma unroll
    for (int s = 0; s < kGroup; ++s) load_x(s, xb[s]);
    lds_barrier();  // the selector table
    decode(0, 0, slot0, 0);
    lds_barrier();  // the first group's operands
    // A SIMD's two wavefronts (j and j + 4) do a group's two parts in opposite order:
    // one decodes the next group while the other multiplies this one.
    const bool early = wave < R / 2;
    int buf = 0;
    for (int kt0 = 0; kt0 < a.KT; kt0 += kRing) {
#pragma unroll
        for (int u = 0; u < kRing; ++u) {
            const int kt = kt0 + u;
            if (u && kt >= a.KT) break;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int last = g == G - 1;
                if (early) decode(kt + last, (g + 1) % G, slots[(u + last) % kRing], buf ^ 1);
                products(kt * S + g * kGroup, buf);
                if (!early) decode(kt + last, (g + 1) % G, slots[(u + last) % kRing], buf ^ 1);
                lds_barrier();
                buf ^= 1;
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(0);  // the transfers past the end
    // A block of tokens at a time the sums pass through LDS, after which 16 lanes hold
    // the 128 rows of a token, 8 each: stores of 256 contiguous bytes, scales and biases
    // read once. One copy of the code for all blocks: unrolled, its instructions (the
    // activations' among them) came from memory once each, 12.5 us at 512 tokens.
    // Scales and factors of the tokens are read at the start, lane l the wavefront's
    // token l: a load between the stores would wait for those too.
    lds_barrier();  // everyone is done with the operand buffers
    uint8_t *const sums = smem + wave * kSumBytes;
    constexpr int kRowLanes = 2 * R, kAtOnce = kLanes / kRowLanes, kRounds = kBlock / kAtOnce;  // lanes of a token; tokens at once
    const int64_t m = (int64_t)job.set * R * kTileRows + 8 * (lane % kRowLanes);
    floatx4 ws[2] = {};
    uint2 bias[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (V::kBytes == 1 && m + 4 * h < (int64_t)a.RB * kTileRows)
            ws[h] = *reinterpret_cast<const floatx4 *>(ref.scale + m + 4 * h);
        bias[h] = load_quad(a.bias ? a.bias + job.e * a.ldb : nullptr, m + 4 * h, a.M, a.e_flags & kEpiBiasVec);
    }
    const bool wide_store = a.y_wide && m + 8 <= a.M;
#pragma unroll 1
    for (int nb = 0; nb < NB && (wave * NB + nb) * kBlock < job.n; ++nb) {
        static_for(
            [&](auto c) __attribute__((always_inline)) {
                if (nb == c.value) {
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        *reinterpret_cast<typename V::Acc *>(sums + (lane & 15) * kSumRow + r * 64 + 16 * (lane >> 4)) =
                            acc[r][c.value];
                }
            },
            std::make_integer_sequence<int, NB>{});
        const int t0 = (wave * NB + nb) * kBlock + lane / kRowLanes;
        uint2 res[kRounds][2];
        if (a.res) {
#pragma unroll
            for (int i = 0; i < kRounds; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    res[i][h] = t0 + kAtOnce * i < job.n ? residual_quad(a, job.row0 + t0 + kAtOnce * i, m + 4 * h) : make_uint2(0, 0);
        }
        uint2 out[kRounds][2];
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int from = nb * kBlock + kAtOnce * i + lane / kRowLanes;  // the lane that holds the token's factors
            const float x = __shfl(xs, from, kLanes), f = __shfl(weight, from, kLanes);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                out[i][h] = finished_quad<V>(
                    a,
                    *reinterpret_cast<const typename V::Acc *>(sums + (kAtOnce * i + lane / kRowLanes) * kSumRow + 32 * (lane % kRowLanes) + 16 * h),
                    ws[h], x, bias[h], res[i][h], f);
        }
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const int t = t0 + kAtOnce * i;
            if (t >= job.n || m >= a.M) continue;
            if (wide_store) {
                *reinterpret_cast<uint4 *>(a.Y + (int64_t)(job.row0 + t) * a.ldy + m) =
                    make_uint4(out[i][0].x, out[i][0].y, out[i][1].x, out[i][1].y);
            } else {
                store_quad(a, job.row0 + t, m, out[i][0]);
                store_quad(a, job.row0 + t, m + 4, out[i][1]);
            }
        }
    }
}

}  // namespace

namespace {

template <class V, int L>
ProductKernelFn wide_kernel_for(int rows, int nb) {
    if (rows == 4) return nb == 2 ? wide_product_kernel<V, L, 4, 2> : wide_product_kernel<V, L, 4, 4>;
    // With eight row blocks what fits LDS and, at four token blocks, the registers.
    if constexpr (wide_serves_rows(V::kBytes, L, 8, 2)) {
        if constexpr (wide_serves_rows(V::kBytes, L, 8, 4)) {
            if (nb == 4) return wide_product_kernel<V, L, 8, 4>;
        }
        return wide_product_kernel<V, L, 8, 2>;
    }
    return nullptr;
}

}  // namespace

ProductKernelFn wide_product_kernel_of(int value_bytes, int loads, int rows, int nb) {
    if (value_bytes == 1) return loads == 3 ? wide_kernel_for<ValuesQ, 3>(rows, nb) : wide_kernel_for<ValuesQ, 5>(rows, nb);
    return loads == 5 ? wide_kernel_for<ValuesF16, 5>(rows, nb) : wide_kernel_for<ValuesF16, 9>(rows, nb);
}

}  // namespace usp
