// usp_product.hip -- products on 8-bit values, and products grouped by expert on
// fp16 and 8-bit values (include/usp.h, usp_spmm_q and usp_spmm_grouped).
#include "usp_product.h"

#include "usp_codes.h"

#include <algorithm>
#include <cmath>

namespace usp {
namespace {

// 16 bytes of a row from p, of which `left` >= 1 bytes remain; zeros past those. Five
// dwords hold them whatever p's alignment (four, ALIGNED: p a multiple of 4); only those
// that hold some of the row are read, and the bytes past it cleared.
template <bool ALIGNED>
__device__ inline v4u32 load_chunk(const uint8_t *p, int left) {
    typedef v4u32 __attribute__((aligned(4))) v4u32_a4;
    const uint32_t sh = ALIGNED ? 0 : (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const uint32_t *const q = reinterpret_cast<const uint32_t *>(p - sh);
    v4u32 v;
    if (left >= 16) {
        const v4u32 d = *reinterpret_cast<const v4u32_a4 *>(q);
        if (ALIGNED) return d;
        const uint32_t e = q[sh ? 4 : 3];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(i < 3 ? d[i < 3 ? i + 1 : 3] : e, d[i], sh);
    } else {
        uint32_t d[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) d[i] = 4 * i < left + (int)sh ? q[i] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = __builtin_amdgcn_alignbyte(d[i + 1], d[i], sh);
            const int bytes = left - 4 * i;
            v[i] = bytes >= 4 ? x : bytes > 0 ? x & ((1u << (8 * bytes)) - 1) : 0;
        }
    }
    return v;
}

// ---------------------------------------------------------------------------
// X packed in the order of the products' B operands: block (tb KT + kt) S + s of
// 1 KB, lane 16 g + n, holds bytes 64 s + 16 g .. + 15 of column tile kt of row
// 16 tb + n (of an expert's rows, gathered; zeros past them and past K). A load of
// X in place touches 16 rows' segments of 64 bytes, which the memory pipeline takes
// several times as long for as for 1 KB in one piece, and each column tile is
// loaded once per row set. One wavefront per block of rows and column tile. ALIGNED: rows
// at multiples of 4 bytes, without the fifth dword of every chunk (traced, 4096 gathered rows
// of 2048 fp16 channels: 16.2 against 18.1 us; 32 x 5120 in 8 bits: 3.6 against 3.8). What
// remains is a chain of latencies: offsets, row indices, X, the store.
// ---------------------------------------------------------------------------
template <class V, bool ALIGNED>
__global__ __launch_bounds__(kLanes) void pack_kernel(ProductArgs a, uint8_t *__restrict__ xp) {
    constexpr int S = V::kStepsPerTile;
    const int lane = threadIdx.x;
    const int kt = blockIdx.x % a.KT;
    Job j;
    if (!find_job<kBlock>(a, a.job0 + (int)(blockIdx.x / a.KT), 1, lane, j)) return;
    const int n = lane & 15;
    int64_t x = j.row0 + n;
    if (a.rows && n < j.n) x = a.rows[j.row0 + n];
    const bool real = n < j.n && x >= 0 && x < a.x_rows;
    const uint8_t *const row = a.X + (real ? x * a.ldx : 0);
    v4u32 v[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int k = kt * kTileK + (64 * s + 16 * (lane >> 4)) / V::kBytes;
        v[s] = v4u32{0u, 0u, 0u, 0u};
        if (!real || k >= a.K) continue;
        v[s] = load_chunk<ALIGNED>(row + (int64_t)k * V::kBytes, (a.K - k) * V::kBytes);
    }
    v4u32 *const out = reinterpret_cast<v4u32 *>(xp + (((int64_t)j.tb * a.KT + kt) * S << 10));
#pragma unroll
    for (int s = 0; s < S; ++s) out[s * kLanes + lane] = v[s];
}

// ---------------------------------------------------------------------------
// fp16 tokens in 8 bits, packed as pack_kernel<ValuesQ> packs usp_quantize's codes and
// with the same bits, in one launch instead of two and without the codes in between.
// A workgroup takes 4 tokens, a quarter of a block of 16, lane by lane, so that a
// wavefront reads 512 bytes of each row and writes pieces of 64 bytes; whole blocks, a
// wavefront to a token, left three quarters of the chip idle at 1024 tokens. Threads keep
// the values of their first kKept chunks of 16 channels between the maximum and the
// codes and read what follows again. VEC: rows of whole 16-byte vectors; others by
// load_chunk (21 tokens of 4093 channels: 4.8 us, 6.2 channel by channel).
// ---------------------------------------------------------------------------
constexpr int kPackTokens = 4, kPackThreads = 1024, kKept = 2;

template <bool VEC>
__global__ __launch_bounds__(kPackThreads) void quantize_pack_kernel(const _Float16 *__restrict__ X, int64_t ldx, int N,
                                                                     int K, int chunks, uint8_t *__restrict__ xp,
                                                                     float *__restrict__ scales) {
    constexpr int kStride = kPackThreads / kPackTokens, kWaves = kPackThreads / kLanes;
    __shared__ uint32_t tops[kWaves][kPackTokens];
    const int t = threadIdx.x % kPackTokens, first = threadIdx.x / kPackTokens;
    const int64_t n = (int64_t)blockIdx.x * kPackTokens + t;
    const _Float16 *const row = X + (n < N ? n : 0) * ldx;
    const int cols = n < N ? K : 0;
    // Channels 16 c .. 16 c + 15, zeros past the row.
    auto load = [&](int c, half8 (&h)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = 16 * c + 8 * i;
            h[i] = half8{};
            if (k >= cols) continue;
            if (VEC)
                h[i] = *reinterpret_cast<const half8 *>(row + k);
            else
                h[i] = __builtin_bit_cast(half8, load_chunk<false>(reinterpret_cast<const uint8_t *>(row + k), 2 * (cols - k)));
        }
    };
    half8 kept[kKept][2];
    uint32_t top = 0;
    auto larger = [&](const half8 (&h)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, magnitude_bits(h[i / 8][i % 8]));
    };
#pragma unroll
    for (int i = 0; i < kKept; ++i) load(first + i * kStride, kept[i]);
#pragma unroll
    for (int i = 0; i < kKept; ++i) larger(kept[i]);
    for (int c = first + kKept * kStride; c < chunks; c += kStride) {
        half8 h[2];
        load(c, h);
        larger(h);
    }
#pragma unroll
    for (int o = kPackTokens; o < kLanes; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, kLanes));
    if (threadIdx.x % kLanes < kPackTokens) tops[threadIdx.x / kLanes][t] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = max(top, tops[w][t]);
    float scale, inv;
    code_scale(top, scale, inv);
    if (threadIdx.x < kPackTokens && n < N) scales[n] = scale;
    // Chunk c of a block's token: step c / 4, lane 16 (c % 4) + the token.
    v4u32 *const out = reinterpret_cast<v4u32 *>(xp) + n / kBlock * kBlock * chunks + n % kBlock;
    auto store = [&](int c, const half8 (&h)[2]) __attribute__((always_inline)) {
        v4u32 v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i / 4] |= code_bits(h[i / 8][i % 8], inv) << (8 * (i % 4));
        out[(int64_t)c * kBlock] = v;
    };
#pragma unroll
    for (int i = 0; i < kKept; ++i)
        if (first + i * kStride < chunks) store(first + i * kStride, kept[i]);
    for (int c = first + kKept * kStride; c < chunks; c += kStride) {
        half8 h[2];
        load(c, h);
        store(c, h);
    }
}

// ---------------------------------------------------------------------------
// Product kernel: a workgroup of W wavefronts takes R row blocks and NB blocks of
// 16 tokens; its wavefronts split the column tiles and sum their parts in LDS.
//
//   Y[n, m] = act(sx[n] sw[m] sum_k q[m, k] x[n, k] + bias[m]) + residual[n, m]
//   (fp16 values: no scales), times the row's weight in a group.
//
// At few tokens it is bound by reading the records from HBM: 70B FFN (28672 x 8192, 50%,
// 8-bit, 148 MB), 16 tokens, R = 4, W = 4: 30.5 us, 4.85 TB/s, where a copy of 2 GB runs
// at 4.94. Every record is read once and decoded in registers, each lane's mask bits into
// the A operand of its products; the next record of a wavefront is in flight into LDS
// meanwhile. Three or four slots a wavefront gain nothing over two there (a record takes 2-3 us
// to come, and 16 wavefronts of a CU keep 32 in flight), and cost wavefronts; on layers of one
// workgroup a CU, with 8 records in flight, they were not measured. More row
// blocks share a load of X; more wavefronts shorten the chain of records where there are
// few row blocks. At 32 and more tokens what bounds it is the decode, 2050-2200 cycles a
// record of a wavefront, so that a decoded operand serves NB blocks of tokens: 70B FFN at
// 64 tokens 51.2 us with NB = 4. X comes straight from memory at NB = 1 and packed above,
// where the packing's launch (3.5 us) is worth it.
// ---------------------------------------------------------------------------

// Requests the whole record at 16-byte units [o0, o1) into an LDS slot: L transfers
// of 16 bytes per lane; past the record's end they read nothing and write zeros.
template <int L>
__device__ inline void request_record(const uint8_t *stream, uint32_t o0, uint32_t o1, int lane, uint8_t *slot) {
    const __amdgpu_buffer_rsrc_t rec = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(stream + (uint64_t)o0 * 16), (short)0, (int)((o1 - o0) * 16), kBufferRsrcWord3);
#pragma unroll
    for (int i = 0; i < L; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rec, (__attribute__((address_space(3))) void *)(slot + 1024 * i), 16,
                                                 1024 * i + lane * 16, 0, 0, kCachePolicyStream);
}

template <class V, int L, int R, int W, int NB, bool PACKED>
__global__ __launch_bounds__(W *kLanes) void product_kernel(ProductArgs a) {
    constexpr int S = V::kStepsPerTile, TB = 16 * NB;
    constexpr int kSlots = 2;  // records of a wavefront in LDS: one being decoded, one in flight
    constexpr int U = 2;       // column tiles per round of the loop, buffers of X
    constexpr int XD = 1;      // how many tiles ahead X is requested
    constexpr int kSlot = 1024 * L;
    // One array per slot (the compiler then waits for the transfers into the one that
    // a decode reads, and no others), each with a part for every wavefront.
    __shared__ __attribute__((aligned(16))) uint8_t slot0[W * kSlot + 16], slot1[W * kSlot + 16];
    __shared__ __attribute__((aligned(16))) uint8_t lut[V::kLutEntries * 8];
    const int lane = threadIdx.x & (kLanes - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    uint8_t *const slots[kSlots] = {slot0 + wave * kSlot, slot1 + wave * kSlot};
    Job job;
    if (!find_job<TB>(a, a.job0 + (int)blockIdx.x, a.sets, lane, job)) return;  // the whole workgroup
    const ExpertRef ref = job_matrix(a, job);
    fill_lut<V>(lut, threadIdx.x, W * kLanes);

    const int kt0 = wave * a.KT / W, kt1 = (wave + 1) * a.KT / W;
    // Lane l: the offset of tile kt0 + l of each row block (0, an empty record, past
    // the matrix and past the next wavefront's first).
    const __amdgpu_buffer_rsrc_t offr = __builtin_amdgcn_make_buffer_rsrc(
        (void *)ref.off, (short)0, (a.RB * a.KT + 1) * 4, kBufferRsrcWord3);
    uint32_t off[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int rb = job.set * R + r;
        const bool ok = rb < a.RB && lane <= kt1 - kt0;
        off[r] = __builtin_amdgcn_raw_buffer_load_b32(offr, ok ? (rb * a.KT + kt0 + lane) * 4 : 0x7FFFFFF0, 0, 0);
    }
    // X: the packed blocks of the job's rows; or in place, from a resource over the
    // job's rows (over all of X where rows are gathered), which lanes of tokens past
    // the job's end read past the end of (zeros).
    __amdgpu_buffer_rsrc_t xr;
    uint32_t x_bytes, xoff[NB];
    if (PACKED) {
        const int64_t block = (int64_t)a.KT * S << 10;
        x_bytes = (uint32_t)(NB * block);
        xr = __builtin_amdgcn_make_buffer_rsrc((void *)(a.xp + job.tb * block), (short)0, (int)x_bytes, kBufferRsrcWord3);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) xoff[nb] = (uint32_t)(nb * block) + 16 * lane;
    } else {
        const int64_t x0 = a.rows ? 0 : (int64_t)job.row0 * a.ldx;
        const int64_t x_rows = a.rows ? a.x_rows : job.n;
        x_bytes = (uint32_t)(((x_rows - 1) * a.ldx + (int64_t)a.K * V::kBytes + 3) & ~(int64_t)3);
        xr = __builtin_amdgcn_make_buffer_rsrc((void *)(a.X + x0), (short)0, (int)x_bytes, kBufferRsrcWord3);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int t = kBlock * nb + (lane & 15);
            int64_t x = t;
            if (a.rows && t < job.n) x = a.rows[job.row0 + t];
            xoff[nb] = t < job.n && x >= 0 && x < x_rows ? (uint32_t)(x * a.ldx) + 16 * (lane >> 4) : x_bytes;
        }
    }
    auto request_x = [&](int kt, v4u32(&xb)[NB][S]) __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                uint32_t at = xoff[nb];
                if (PACKED) {
                    xb[nb][s] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)at, (kt * S + s) << 10, 0);
                } else {
                    at += (uint32_t)(kt * kTileK * V::kBytes + 64 * s);
                    // fp16 past a row's end could be a NaN, which zeros in W do not undo.
                    if (V::kBytes == 2 && kt * kTileK + 32 * s + 8 * (lane >> 4) >= a.K) at = x_bytes;
                    xb[nb][s] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)at, 0, 0);
                }
            }
    };
    // Record `rec` (0 .. U R + 2, a constant) of the round that starts at tile kt.
    auto request = [&](int kt, int rec) __attribute__((always_inline)) {
        const int r = rec % R, u = kt - kt0 + rec / R;
        const bool real = kt0 + u < kt1;
        const uint32_t o0 = real ? __builtin_amdgcn_readlane(off[r], u) : 0;
        const uint32_t o1 = real ? __builtin_amdgcn_readlane(off[r], u + 1) : 0;
        request_record<L>(ref.stream, o0, o1, lane, slots[rec % kSlots]);
    };
    __syncthreads();  // the selector table
    typename V::Acc acc[R][NB] = {};
    v4u32 xb[U][NB][S];
#pragma unroll
    for (int u = 0; u < XD; ++u) request_x(kt0 + u, xb[u]);
#pragma unroll
    for (int i = 0; i < kSlots - 1; ++i) request(kt0, i);
    for (int kt = kt0; kt < kt1; kt += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u && kt + u >= kt1) break;
            request_x(kt + u + XD, xb[(u + XD) % U]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int rec = u * R + r;
                request(kt, rec + kSlots - 1);
                uint8_t *const slot = slots[rec % kSlots];
                // The record is there once at most the loads issued after it are outstanding:
                // the next tile's X, at a tile's first record, and the next record's.
                if (r == 0)
                    wait_loads<L + NB * S>();
                else
                    wait_loads<L>();
                const typename V::State rs = V::state(slot, lane, (uint32_t)(wave * kSlot));
                lds_u32 *const region = as_lds(rec % kSlots == 0 ? slot0 : slot1);
                typename V::Words w = V::read(region, lut, rs, 0);
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    typename V::Words next;
                    if (s + 1 < S) next = V::read(region, lut, rs, s + 1);
                    const v4u32 av = V::finish(w);
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) acc[r][nb] = V::multiply(av, xb[u][nb][s], acc[r][nb]);
                    if (s + 1 < S) w = next;
                }
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(0);  // the transfers past the range's end
    // Item i of the R x NB products is finished by wavefront i % W, parts in wavefront
    // order; they pass through the slots, as many at a time as those hold. One copy of
    // the code that finishes an item: with one for each, its instructions came from
    // memory for every item.
    constexpr int kItems = R * NB, kRound = kSlots * L;
    uint8_t *const area[kSlots] = {slot0, slot1};
    typedef typename V::Acc Acc;
    static_assert(kSlots == 2 && kRound * W * 1024 <= kSlots * W * kSlot, "the slots hold a round's sums");
#pragma unroll
    for (int i0 = 0; i0 < kItems; i0 += kRound) {
        __syncthreads();
#pragma unroll
        for (int i = i0; i < i0 + kRound && i < kItems; ++i)
            reinterpret_cast<Acc *>(area[i % 2])[((i - i0) / 2 * W + wave) * kLanes + lane] = acc[i / NB][i % NB];
        __syncthreads();
#pragma unroll 1
        for (int i = i0 + (wave + W - i0 % W) % W; i < i0 + kRound && i < kItems; i += W) {
            const Acc *const p = reinterpret_cast<const Acc *>(i % 2 ? slot1 : slot0) + (i - i0) / 2 * W * kLanes + lane;
            Acc sum = {};
#pragma unroll
            for (int w = 0; w < W; ++w) sum += p[w * kLanes];
            const int t = kBlock * (i % NB) + (lane & 15);
            const int64_t m = ((int64_t)job.set * R + i / NB) * kTileRows + 4 * (lane >> 4);
            if (t < job.n && m < a.M) finish_quad<V>(a, ref.scale, job.e, job.row0 + t, m, sum);
        }
    }
}

// One wavefront per tile of 8-bit values: every lane-step decoded, times the row's
// scale, rounded to fp16.
__global__ __launch_bounds__(kLanes) void densify_q_kernel(ExpertRef ref, int64_t M, int64_t K, int64_t KT,
                                                           uint16_t *Wd, int64_t ldw) {
    __shared__ __attribute__((aligned(16))) uint8_t region[kMaskBytes + kStartBytesQ + kTileRows * kTileK + 16];
    __shared__ __attribute__((aligned(16))) uint8_t lut[ValuesQ::kLutEntries * 8];
    const int lane = threadIdx.x;
    const int64_t t = blockIdx.x, rb = t / KT, kt = t % KT;
    fill_lut<ValuesQ>(lut, lane, kLanes);
    const uint32_t o0 = ref.off[t], o1 = ref.off[t + 1];
    const uint4 *rec = reinterpret_cast<const uint4 *>(ref.stream + (size_t)o0 * 16);
    for (int c = lane; c < (int)(o1 - o0); c += kLanes) reinterpret_cast<uint4 *>(region)[c] = rec[c];
    __syncthreads();
    const RecStateQ rs = ValuesQ::state(region, lane, 0);
    const int64_t row = rb * kTileRows + (lane & 15);
    if (row >= M) return;
    const float scale = ref.scale[row];
    for (int s = 0; s < kStepsQ; ++s) {
        const v4u32 av = ValuesQ::finish(ValuesQ::read(as_lds(region), lut, rs, s));
        const int64_t col = kt * kTileK + tile_col_q(lane >> 4, 2 * s, 0);
        for (int j = 0; j < 16; ++j) {
            const int q = (int8_t)(av[j / 4] >> (8 * (j % 4)));
            if (col + j < K) Wd[row * ldw + col + j] = __builtin_bit_cast(uint16_t, (_Float16)(scale * (float)q));
        }
    }
}

template <class V, int L, int NB, bool PACKED>
ProductKernelFn product_kernel_of(int rows, int waves) {
    if (rows == 1) return waves == 4 ? product_kernel<V, L, 1, 4, NB, PACKED> : product_kernel<V, L, 1, 8, NB, PACKED>;
    if (rows == 2) return waves == 4 ? product_kernel<V, L, 2, 4, NB, PACKED> : product_kernel<V, L, 2, 8, NB, PACKED>;
    return waves == 4 ? product_kernel<V, L, 4, 4, NB, PACKED> : product_kernel<V, L, 4, 8, NB, PACKED>;
}

typedef void (*PackKernelFn)(ProductArgs, uint8_t *);
template <class V>
PackKernelFn pack_kernel_of(bool aligned) {
    return aligned ? pack_kernel<V, true> : pack_kernel<V, false>;
}

// The smallest built count of 1 KB transfers that covers every record, the decode's
// reads past its values included.
int record_loads(const ProductShape &s) {
    const int64_t kb = ceil_div(16 * (kMaskChunks + s.max_chunks) + 12, (int64_t)1024);
    return s.value_bytes == 1 ? kb <= 3 ? 3 : 5 : kb <= 5 ? 5 : 9;
}

struct ProductPlan {
    bool wide, packed;
    int rows, waves, nb;  // wide: waves = rows
    int64_t sets, grid;
};

// Groups of at most tb tokens that a call has, at most and as expected. A group's counts
// are known on the device alone: at most one group beyond N / tb for every expert with
// rows; expected, half of one for every expert that random rows reach.
int64_t most_groups(const ProductShape &s, int64_t N, int64_t tb) {
    return s.G ? N / tb + std::min(s.G->E, N) : ceil_div(N, tb);
}
double expected_groups(const ProductShape &s, int64_t N, int64_t tb) {
    if (!s.G) return (double)ceil_div(N, tb);
    const double E = (double)s.G->E, active = 0.9 * E * (1.0 - std::exp(-(double)N / E));
    return std::max(1.0, std::max(active, (double)N / (double)tb + 0.5 * active));
}

// Up to so many tokens no wide kernel is considered (the model below took none up to 18 in
// 3 million random shapes), so that few tokens need little behind X packed.
constexpr int64_t kFewTokens = kBlock;

// The kernel that costs least by a model of what was measured (us; 8-bit values at 50%,
// fp16 records scaled; layers of 1024 x 1024 to 28672 x 8192 and groups of 7 to 64
// experts). Product kernel: a launch, a wavefront's start, and the longer of a
// wavefront's chain of records and the records of a CU, whose time has a part for X
// that R row blocks share. At 16 tokens (R W): 13B attention 1 4 10.3, 2 8 9.6, 4 8
// 13.3; 13B FFN up 1 4 18.6, 2 4 13.9, 4 8 14.1; 70B FFN 1 8 43.4, 2 4 34.3, 4 4 30.5;
// at 64: 70B FFN 2 4 57.2, 4 8 51.2. Wide kernel: rounds of workgroups of KT tiles and an
// epilogue; two of 4 row blocks share a CU. It wins from about 128 tokens on large
// layers (70B FFN at 128 63.3 against 99.0) and 256 on small ones (13B attention at 128
// 31.5 against 22.6, at 256 33.0 against 34.0). Packing is a launch more, but not for fp16
// tokens of 8-bit products (`quantize`), which take one either way (4999 x 4096, 21 tokens:
// 12.4 us, 13.9 planned as packed at a cost; 3584 x 8192, 24: 14.5 and 16.1).
ProductPlan plan_product(const ProductShape &s, int64_t N, bool quantize = false) {
    const double cus = s.num_cus > 0 ? s.num_cus : 256;
    const int loads = record_loads(s);
    const double value = s.value_bytes == 1 ? 1.0 : 1.8, size = value * (loads > 5 || (loads > 3 && s.value_bytes == 1) ? 1.5 : 1.0);
    ProductPlan best = {};
    double least = 0;
    auto consider = [&](const ProductPlan &p, double cost) {
        if (best.grid && cost >= least) return;
        best = p;
        least = cost;
    };
    static const struct {
        int rows, waves, nb;
        double record;  // us of a CU
    } kernels[] = {{1, 4, 1, .15}, {1, 8, 1, .15}, {2, 4, 1, .118}, {2, 8, 1, .118}, {4, 4, 1, .107}, {4, 8, 1, .107},
                   {1, 4, 2, .16}, {1, 8, 2, .16}, {2, 4, 2, .13},  {2, 8, 2, .13},  {4, 4, 2, .121}, {4, 8, 2, .121},
                   {1, 4, 4, .27}, {2, 4, 4, .19}, {4, 8, 4, .167}};
    for (const auto &k : kernels) {
        if (k.nb == 4 && s.value_bytes != 1) continue;  // registers
        if (ceil_div(s.KT, (int64_t)k.waves) >= kLanes) continue;  // a lane per tile's offset and one for the end
        const int64_t tb = kBlock * k.nb, sets = ceil_div(s.RB, (int64_t)k.rows);
        const double wgs = std::ceil((double)sets * expected_groups(s, N, tb) / cus);
        const double chain = 0.75 * size * k.rows * (double)ceil_div(s.KT, (int64_t)k.waves);
        const double cost = 2.6 + (k.nb > 1 && !quantize ? 3.5 : 0.0) + 0.24 * std::min(16.0, wgs * k.waves) +
                            std::max(chain, wgs * k.rows * (double)s.KT * k.record * size * (k.nb > 1 && value > 1 ? 1.2 : 1.0));
        consider({false, k.nb > 1, k.rows, k.waves, k.nb, sets, sets * most_groups(s, N, tb)}, cost);
    }
    static const struct {
        int rows, nb;
        double alone[2], shared[2];  // us of a tile of fp16 and 8-bit values, for one workgroup on a CU and for two
    } wides[] = {{4, 2, {1.65, 1.22}, {2.3, 1.7}}, {4, 4, {2.2, 1.5}, {3.3, 2.15}}, {8, 2, {4.2, 2.1}, {0, 0}}, {8, 4, {0, 3.25}, {0, 0}}};
    for (const auto &k : wides) {
        if (N <= kFewTokens) break;
        if (!wide_serves_rows(s.value_bytes, loads, k.rows, k.nb)) continue;
        const int q = s.value_bytes == 1;
        const int64_t tb = (int64_t)kBlock * k.nb * k.rows, sets = ceil_div(s.RB, (int64_t)k.rows);
        const bool two = k.rows == 4 && loads <= 5;
        const double wgs = (double)sets * expected_groups(s, N, tb), slots = two ? 2 * cus : cus;
        const double full = std::floor(wgs / slots), rest = wgs - full * slots;
        const double tile = two ? k.shared[q] : k.alone[q];
        // A group's last round is as full as its counts make it.
        const double tiles = s.G ? std::max(k.alone[q], wgs / slots * tile + 0.5 * k.alone[q])
                                 : full * tile + (rest <= 0 ? 0 : rest > cus ? tile : k.alone[q]);
        const double cost = (quantize ? 4.0 : 7.5) + std::ceil(wgs / slots) * (1.0 + k.nb) + tiles * (double)s.KT;
        consider({true, true, k.rows, k.rows, k.nb, sets, sets * most_groups(s, N, tb)}, cost);
    }
    return best;
}

template <class V, int L>
ProductKernelFn kernel_for(const ProductPlan &p) {
    if (p.nb == 1)
        return p.packed ? product_kernel_of<V, L, 1, true>(p.rows, p.waves) : product_kernel_of<V, L, 1, false>(p.rows, p.waves);
    if constexpr (V::kBytes == 1) {
        if (p.nb == 4)
            return p.rows == 1   ? product_kernel<V, L, 1, 4, 4, true>
                   : p.rows == 4 ? product_kernel<V, L, 4, 8, 4, true>
                                 : product_kernel<V, L, 2, 4, 4, true>;
    }
    return product_kernel_of<V, L, 2, true>(p.rows, p.waves);
}

ProductKernelFn plan_kernel(const ProductShape &s, const ProductPlan &p) {
    const int l = record_loads(s);
    if (p.wide) return wide_product_kernel_of(s.value_bytes, l, p.rows, p.nb);
    if (s.value_bytes == 1) return l == 3 ? kernel_for<ValuesQ, 3>(p) : kernel_for<ValuesQ, 5>(p);
    return l == 5 ? kernel_for<ValuesF16, 5>(p) : kernel_for<ValuesF16, 9>(p);
}

// X in place: dword-aligned rows, whole 16-byte chunks of fp16 (what follows a row
// of 8-bit values meets zeros in W), rows of a resource within 32-bit offsets.
constexpr int64_t kMaxSpan = ((int64_t)1 << 32) - ((int64_t)1 << 20);
// Workgroups of one launch (a grid has fewer than 2^32 threads).
constexpr int64_t kMaxGrid = (int64_t)1 << 21;

// Blocks of 16 rows of X packed, at most, and what a job may read past its last one: a
// job has at least one block of its own and reads as many as its workgroup takes (4 at most
// of the product kernel, 8 x 4 of the wide one), and a column tile past those.
int64_t packed_blocks(const ProductShape &s, int64_t N) { return most_groups(s, N, kBlock); }
constexpr int64_t more_blocks(int64_t N) { return N <= kFewTokens ? 4 : 32; }

size_t packed_bytes(const ProductShape &s, int64_t N) {
    return (size_t)(packed_blocks(s, N) + more_blocks(N)) * s.KT * kTileK * s.value_bytes * kBlock;
}

}  // namespace

// Where in the workspace what lies: X packed, after the region that other products keep
// cleared, or in its place (8-bit matrices) the codes of fp16 tokens, in rows that are read
// in place and are no longer than packed ones; then the scales of those tokens.
struct ProductSpace {
    size_t packed, codes, scales, end;
    int64_t ld_codes;
};
static ProductSpace product_space(const ProductShape &s, int64_t N) {
    ProductSpace w;
    w.ld_codes = ceil_div(s.K, (int64_t)16) * 16;
    w.packed = kCounterRegionBytes;
    w.codes = w.packed;
    w.scales = w.packed + packed_bytes(s, N);
    w.end = w.scales + (s.A && s.value_bytes == 1 ? (size_t)(4 * N) : 0);
    return w;
}

// No kernel's grid is larger than that of one row block and 16 tokens a workgroup, and
// where that is too large Y would take 1 TB.
bool product_fits(const ProductShape &s, int64_t N) { return s.RB * most_groups(s, N, kBlock) < ((int64_t)1 << 31); }

size_t product_workspace_bytes(const ProductShape &s, int64_t N) { return product_space(s, N).end; }

std::string describe_product(const ProductShape &s, int64_t N) {
    const ProductPlan p = plan_product(s, N);
    return std::string(p.wide ? "wide-product" : "product") + " R=" + std::to_string(p.rows) +
           (p.wide ? "" : " W=" + std::to_string(p.waves)) + " nb=" + std::to_string(p.nb) +
           " grid=" + std::to_string(p.grid);
}

int launch_densify_q(const usp_matrix *A, void *Wd, int64_t ldw, void *stream) {
    hipLaunchKernelGGL(densify_q_kernel, dim3((unsigned)(A->RB * A->KT)), dim3(kLanes), 0,
                       reinterpret_cast<hipStream_t>(stream),
                       ExpertRef{reinterpret_cast<const uint8_t *>(A->d_stream), A->d_off, A->d_scale}, A->M, A->K, A->KT,
                       reinterpret_cast<uint16_t *>(Wd), ldw);
    return (int)hipGetLastError();
}

int launch_product(const ProductShape &s, const ProductCall &call, void *workspace, void *stream) {
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const ProductSpace space = product_space(s, call.N);
    uint8_t *const ws = reinterpret_cast<uint8_t *>(workspace);
    ProductCall c = call;
    ProductPlan p = plan_product(s, c.N, c.quantize);
    const bool fused = c.quantize && p.packed;
    if (fused) {
        const bool vec = (reinterpret_cast<uintptr_t>(c.X) & 15) == 0 && c.ldx % 8 == 0 && s.K % 8 == 0;
        c.x_scale = reinterpret_cast<const float *>(ws + space.scales);
        hipLaunchKernelGGL(vec ? quantize_pack_kernel<true> : quantize_pack_kernel<false>,
                           dim3((unsigned)(ceil_div(c.N, (int64_t)kBlock) * (kBlock / kPackTokens))), dim3(kPackThreads), 0, st,
                           reinterpret_cast<const _Float16 *>(c.X), c.ldx, (int)c.N, (int)s.K,
                           (int)(s.KT * kTileK / 16), ws + space.packed, reinterpret_cast<float *>(ws + space.scales));
    } else if (c.quantize) {
        usp_norm_args q = {};
        q.residual = c.X;
        q.ld_residual = c.ldx;
        q.out_q = ws + space.codes;
        q.ld_out_q = space.ld_codes;
        q.out_scale = reinterpret_cast<float *>(ws + space.scales);
        if (const int rc = launch_norm(q, c.N, s.K, stream)) return rc;
        // Read where they are, which is where X would be packed: their rows are aligned, and
        // a job's (64 of at most USP_MAX_K_Q bytes) are within a resource's offsets.
        static_assert(64 * (int64_t)(USP_MAX_K_Q + 16) <= kMaxSpan, "");
        c.X = q.out_q;
        c.ldx = q.ld_out_q;
        c.x_scale = q.out_scale;
    }
    const int vb = s.value_bytes;
    ProductArgs a = {};
    if (s.G) {
        a.experts = reinterpret_cast<const ExpertRef *>(s.G->d_experts);
        a.E = (int)s.G->E;
        a.offsets = c.offsets;
    } else {
        a.one = {reinterpret_cast<const uint8_t *>(s.A->d_stream), s.A->d_off, s.A->d_scale};
    }
    a.M = s.M;
    a.K = (int)s.K;
    a.RB = (int)s.RB;
    a.KT = (int)s.KT;
    a.sets = (int)p.sets;
    a.X = reinterpret_cast<const uint8_t *>(c.X);
    a.ldx = c.ldx * vb;
    a.x_rows = c.x_rows;
    a.xs = c.x_scale;
    a.rows = c.rows;
    a.xs_rows = c.rows;
    a.xs_count = c.x_rows;
    a.weight = c.weight;
    a.Y = reinterpret_cast<uint16_t *>(c.Y);
    a.ldy = c.ldy;
    a.N = (int)c.N;
    a.y_vec = (reinterpret_cast<uintptr_t>(c.Y) & 7) == 0 && c.ldy % 4 == 0;
    a.y_wide = (reinterpret_cast<uintptr_t>(c.Y) & 15) == 0 && c.ldy % 8 == 0;
    a.bias = c.ep.bias;
    a.ldb = c.ldb;
    a.res = c.ep.res;
    a.ldr = c.ep.ldr;
    a.act = c.ep.act;
    a.e_flags = epilogue_flags(c.ep);
    if (c.ldb % 4 != 0) a.e_flags &= ~kEpiBiasVec;
    const int64_t span = c.rows ? c.x_rows : std::min<int64_t>(c.N, kBlock * p.nb);
    const bool aligned = (reinterpret_cast<uintptr_t>(c.X) & 3) == 0 && a.ldx % 4 == 0;
    p.packed = p.packed || !aligned || (vb == 2 && s.K % 8 != 0) ||
               span > kMaxSpan / a.ldx;
    if (p.packed) {
        uint8_t *const xp = ws + space.packed;
        const int64_t blocks = packed_blocks(s, c.N), most = kMaxGrid / s.KT;
        a.xp = xp;
        for (int64_t b0 = 0; !fused && b0 < blocks; b0 += most) {
            a.job0 = (int)b0;
            hipLaunchKernelGGL(vb == 1 ? pack_kernel_of<ValuesQ>(aligned) : pack_kernel_of<ValuesF16>(aligned),
                               dim3((unsigned)(std::min(most, blocks - b0) * s.KT)), dim3(kLanes), 0, st, a, xp);
        }
    }
    const ProductKernelFn fn = plan_kernel(s, p);
    for (int64_t j0 = 0; j0 < p.grid; j0 += kMaxGrid) {
        a.job0 = (int)j0;
        hipLaunchKernelGGL(fn, dim3((unsigned)std::min(kMaxGrid, p.grid - j0)), dim3(p.waves * kLanes), 0, st, a);
    }
    return (int)hipGetLastError();
}

}  // namespace usp
