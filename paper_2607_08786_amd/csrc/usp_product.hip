// usp_product.hip -- products on 8-bit values, and products grouped by expert on
// fp16 and 8-bit values (include/usp.h, usp_spmm_q and usp_spmm_grouped).
#include "usp_product.h"

#include <algorithm>

namespace usp {
namespace {

// ---------------------------------------------------------------------------
// X copied to rows of whole column tiles, zeros past K (and gathered, where it is
// to be): for X whose rows the products cannot load in place. One thread per 16
// bytes of a row; elements of ES bytes at any alignment.
// ---------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(256) void copy_x_kernel(const E *__restrict__ X, int64_t ldx, int64_t x_rows,
                                                     const int32_t *__restrict__ rows, int64_t K, int64_t row_chunks,
                                                     int64_t chunks, E *__restrict__ out) {
    constexpr int V = 16 / sizeof(E);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= chunks) return;
    const int64_t t = i / row_chunks, k = i % row_chunks * V, r = rows ? rows[t] : t;
    const bool real = r >= 0 && r < x_rows;
    E v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = real && k + j < K ? X[r * ldx + k + j] : (E)0;
#pragma unroll
    for (int j = 0; j < V; ++j) out[i * V + j] = v[j];
}

// ---------------------------------------------------------------------------
// Product kernel: a workgroup of W wavefronts takes R row blocks and NB blocks of
// 16 tokens; its wavefronts split the column tiles and sum their parts in LDS.
// ---------------------------------------------------------------------------
template <class V, int L, int R, int W, int NB>
__global__ __launch_bounds__(W *kLanes) void product_kernel(ProductArgs a) {
    constexpr int S = V::kStepsPerTile, TB = 16 * NB;
    constexpr int kSlot = 1024 * L;
    constexpr int kSum = R * NB * 1024;  // a wavefront's sums
    constexpr int kWave = kSlot > kSum ? kSlot : kSum;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[W * kWave + 16];
    __shared__ __attribute__((aligned(16))) uint8_t lut[V::kLutBytes];
    const int lane = threadIdx.x & (kLanes - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
    Job job;
    if (!find_job<TB>(a, a.job0 + (int)blockIdx.x, lane, job)) return;  // the whole workgroup
    const ExpertRef ref = a.experts ? a.experts[job.e] : a.one;
    if (threadIdx.x < 16) V::fill_lut(lut, threadIdx.x);
    __syncthreads();

    // Rows of X: a resource over the job's rows, or over all of X where rows are
    // gathered; lanes of tokens past the job's end read past its end (zeros).
    const int64_t x0 = a.rows ? 0 : (int64_t)job.row0 * a.ldx;
    const int64_t x_rows = a.rows ? a.x_rows : job.n;
    const uint32_t x_bytes = (uint32_t)(((x_rows - 1) * a.ldx + (int64_t)a.K * V::kBytes + 3) & ~(int64_t)3);
    const __amdgpu_buffer_rsrc_t xr =
        __builtin_amdgcn_make_buffer_rsrc((void *)(a.X + x0), (short)0, (int)x_bytes, kBufferRsrcWord3);
    uint32_t xoff[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int t = 16 * nb + (lane & 15);
        int64_t x = t;
        if (a.rows && t < job.n) x = a.rows[job.row0 + t];
        xoff[nb] = t < job.n && x >= 0 && x < x_rows ? (uint32_t)(x * a.ldx) + 16 * (lane >> 4) : x_bytes;
    }
    const __amdgpu_buffer_rsrc_t offr = __builtin_amdgcn_make_buffer_rsrc(
        (void *)ref.off, (short)0, (a.RB * a.KT + 1) * 4, kBufferRsrcWord3);
    const int slot = wave * kWave;
    const uint32_t lds = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)smem) + slot;

    typename V::Acc acc[R][NB] = {};
    const int kt0 = wave * a.KT / W, kt1 = (wave + 1) * a.KT / W;
    for (int kt = kt0; kt < kt1; ++kt) {
        v4u32 xb[NB][S];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < S; ++s) {
                uint32_t at = xoff[nb] + (uint32_t)(kt * kTileK * V::kBytes + 64 * s);
                // fp16 past a row's end could be a NaN, which zeros in W do not undo.
                if (V::kBytes == 2 && kt * kTileK + 32 * s + 8 * (lane >> 4) >= a.K) at = x_bytes;
                xb[nb][s] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)at, 0, 0);
            }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int rb = job.set * R + r;
            const bool ok = rb < a.RB && lane < 2;
            const uint32_t o = __builtin_amdgcn_raw_buffer_load_b32(offr, ok ? (rb * a.KT + kt + lane) * 4 : 0x7FFFFFF0, 0, 0);
            dma_rec_asm<L>(ref.stream, __builtin_amdgcn_readlane(o, 0), __builtin_amdgcn_readlane(o, 1), lane, lds);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const RecState rs = rec_state<V::kBytes>(slot_mask(smem + slot, lane), (uint32_t)(slot + kMaskBytes));
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const v4u32 av = V::finish(V::read(as_lds(smem), lut, rs, s));
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[r][nb] = V::multiply(av, xb[nb][s], acc[r][nb]);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot's reads, before its next record
        }
    }
    __syncthreads();
    typename V::Acc *const part = reinterpret_cast<typename V::Acc *>(smem + slot);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) part[(r * NB + nb) * kLanes + lane] = acc[r][nb];
    __syncthreads();
    for (int i = wave; i < R * NB; i += W) {
        typename V::Acc sum = reinterpret_cast<typename V::Acc *>(smem)[i * kLanes + lane];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += reinterpret_cast<typename V::Acc *>(smem + w * kWave)[i * kLanes + lane];
        const int t = 16 * (i % NB) + (lane & 15);
        const int64_t m = ((int64_t)job.set * R + i / NB) * kTileRows + 4 * (lane >> 4);
        if (t < job.n && m < a.M) finish_quad<V>(a, ref.scale, job.e, job.row0 + t, m, sum);
    }
}

// One wavefront per tile of 8-bit values: every lane-step decoded, times the row's
// scale, rounded to fp16.
__global__ __launch_bounds__(kLanes) void densify_q_kernel(ExpertRef ref, int64_t M, int64_t K, int64_t KT,
                                                           uint16_t *Wd, int64_t ldw) {
    __shared__ __attribute__((aligned(16))) uint8_t region[kTileRows * kTileK + 16];
    __shared__ __attribute__((aligned(16))) uint8_t lut[ValuesQ::kLutBytes];
    const int lane = threadIdx.x;
    const int64_t t = blockIdx.x, rb = t / KT, kt = t % KT;
    if (lane < 16) ValuesQ::fill_lut(lut, lane);
    const uint32_t o0 = ref.off[t], o1 = ref.off[t + 1];
    const uint8_t *rec = ref.stream + (size_t)o0 * 16;
    const uint2 msk = reinterpret_cast<const uint2 *>(rec)[lane];
    const int nch = (int)(o1 - o0) - kMaskChunks;
    const uint4 *vp = reinterpret_cast<const uint4 *>(rec + kMaskBytes);
    for (int c = lane; c < nch; c += kLanes) reinterpret_cast<uint4 *>(region)[c] = vp[c];
    __syncthreads();
    const RecState rs = rec_state<1>(msk);
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

typedef void (*ProductKernelFn)(ProductArgs);

constexpr int kRows = 1, kWaves = 4;

template <class V, int L>
ProductKernelFn product_kernel_of(int nb) {
    return nb == 1 ? product_kernel<V, L, kRows, kWaves, 1> : product_kernel<V, L, kRows, kWaves, 2>;
}

// 1 KB transfers that cover every record.
int record_loads(const ProductShape &s) { return (int)ceil_div(kMaskChunks + s.max_chunks, kLanes); }

struct ProductPlan {
    ProductKernelFn fn;
    int nb, rows, waves;
    int64_t sets, grid;
};

ProductPlan plan_product(const ProductShape &s, int64_t N) {
    ProductPlan p;
    const int64_t E = s.G ? s.G->E : 1;
    p.nb = N > 16 * E ? 2 : 1;
    p.rows = kRows;
    p.waves = kWaves;
    const int l = record_loads(s);
    if (s.value_bytes == 1)
        p.fn = l <= 3 ? product_kernel_of<ValuesQ, 3>(p.nb) : product_kernel_of<ValuesQ, 5>(p.nb);
    else
        p.fn = l <= 5 ? product_kernel_of<ValuesF16, 5>(p.nb) : product_kernel_of<ValuesF16, 9>(p.nb);
    p.sets = ceil_div(s.RB, p.rows);
    // A group's counts are known on the device alone: at most one group of tokens
    // beyond N / TB for every expert with rows.
    const int64_t tb = 16 * p.nb;
    p.grid = p.sets * (s.G ? N / tb + std::min(E, N) : ceil_div(N, tb));
    return p;
}

// Bytes that a resource over rows of X may span: offsets past its end, for rows and
// columns that are to read zeros, stay below 2^32.
constexpr int64_t kMaxSpan = ((int64_t)1 << 32) - ((int64_t)1 << 20);
// Workgroups of one launch (a grid has fewer than 2^32 threads).
constexpr int64_t kMaxGrid = (int64_t)1 << 21;

size_t copied_x_bytes(const ProductShape &s, int64_t N) { return (size_t)N * s.KT * kTileK * s.value_bytes; }

}  // namespace

bool product_fits(const ProductShape &s, int64_t N) { return plan_product(s, N).grid < ((int64_t)1 << 31); }

// The copy of X follows the region that other products keep cleared.
size_t product_workspace_bytes(const ProductShape &s, int64_t N) { return kCounterRegionBytes + copied_x_bytes(s, N); }

std::string describe_product(const ProductShape &s, int64_t N) {
    const ProductPlan p = plan_product(s, N);
    return "product R=" + std::to_string(p.rows) + " W=" + std::to_string(p.waves) + " nb=" + std::to_string(p.nb) +
           " grid=" + std::to_string(p.grid);
}

int launch_densify_q(const usp_matrix *A, void *Wd, int64_t ldw, void *stream) {
    hipLaunchKernelGGL(densify_q_kernel, dim3((unsigned)(A->RB * A->KT)), dim3(kLanes), 0,
                       reinterpret_cast<hipStream_t>(stream),
                       ExpertRef{reinterpret_cast<const uint8_t *>(A->d_stream), A->d_off, A->d_scale}, A->M, A->K, A->KT,
                       reinterpret_cast<uint16_t *>(Wd), ldw);
    return (int)hipGetLastError();
}

int launch_product(const ProductShape &s, const ProductCall &c, void *workspace, void *stream) {
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const ProductPlan p = plan_product(s, c.N);
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
    a.bias = c.ep.bias;
    a.ldb = c.ldb;
    a.res = c.ep.res;
    a.ldr = c.ep.ldr;
    a.act = c.ep.act;
    a.e_flags = epilogue_flags(c.ep);
    if (c.ldb % 4 != 0) a.e_flags &= ~kEpiBiasVec;
    // In place: dword-aligned rows, whole 16-byte chunks of fp16 (what follows a row
    // of 8-bit values meets zeros in W), rows of a resource within 32-bit offsets.
    const int64_t span = c.rows ? c.x_rows : std::min<int64_t>(c.N, 16 * p.nb);
    if ((reinterpret_cast<uintptr_t>(c.X) & 3) || a.ldx % 4 != 0 || (vb == 2 && s.K % 8 != 0) ||
        span > kMaxSpan / a.ldx) {
        uint8_t *const x = reinterpret_cast<uint8_t *>(workspace) + kCounterRegionBytes;
        const int64_t row_chunks = s.KT * kTileK * vb / 16, chunks = row_chunks * c.N;
        const dim3 grid((unsigned)ceil_div(chunks, 256));
        if (vb == 1)
            hipLaunchKernelGGL(copy_x_kernel<uint8_t>, grid, dim3(256), 0, st, reinterpret_cast<const uint8_t *>(c.X),
                               c.ldx, c.x_rows, c.rows, s.K, row_chunks, chunks, x);
        else
            hipLaunchKernelGGL(copy_x_kernel<uint16_t>, grid, dim3(256), 0, st, reinterpret_cast<const uint16_t *>(c.X),
                               c.ldx, c.x_rows, c.rows, s.K, row_chunks, chunks, reinterpret_cast<uint16_t *>(x));
        a.X = x;
        a.K = (int)(s.KT * kTileK);
        a.ldx = a.K * vb;
        a.x_rows = c.N;
        a.rows = nullptr;
    }
    for (int64_t j0 = 0; j0 < p.grid; j0 += kMaxGrid) {
        a.job0 = (int)j0;
        hipLaunchKernelGGL(p.fn, dim3((unsigned)std::min(kMaxGrid, p.grid - j0)), dim3(p.waves * kLanes), 0, st, a);
    }
    return (int)hipGetLastError();
}

}  // namespace usp
