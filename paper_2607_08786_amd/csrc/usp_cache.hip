// usp_cache.hip -- new tokens into a paged cache and back, and copies of its pages
// (include/usp.h, usp_cache_append, usp_cache_read, usp_cache_copy).
//
// All of it moves bytes: 128 pages of 64 tokens of 8 heads of 128 in 4 layers, 268 MB read and written, in 51.8 us (5.2
// TB/s, the rate of a library copy); 2133 rows of 40 heads of 128 into 8 bits and back, 132 MB, in 36 us (3.7 TB/s, two
// launches); 32 single tokens of 8 heads in 3.1 us, a launch and two dependent reads.
#include "usp_cache.h"
#include "usp_codes.h"

#include <algorithm>

namespace usp {
namespace {

typedef _Float16 half8c __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2c __attribute__((ext_vector_type(2)));

constexpr int kLanes64 = 64;
constexpr int kCacheThreads = 256;

struct RowsArgs {
    CacheView c;
    RowsView r;
    HeadRows k, v;
    int vec;  // 16-byte aligned heads
};

// One wavefront takes a head of a row: lanes 0 .. 31 eight channels of its key each, lanes
// 32 .. 63 of its value.
struct Place {
    int t, h, chunk;
    bool value, there;
    uint8_t *block;
    int j;  // the token in its block
};
__device__ inline Place place_of(const RowsArgs &a) {
    Place p;
    const int lane = threadIdx.x & (kLanes64 - 1);
    const int64_t i = (int64_t)blockIdx.x * (kCacheThreads / kLanes64) + threadIdx.x / kLanes64;
    p.t = (int)(i / a.c.kv_heads);
    p.h = (int)(i - (int64_t)p.t * a.c.kv_heads);
    p.value = lane >= 32;
    p.chunk = lane & 31;
    p.block = nullptr;
    p.j = 0;
    if (p.t < a.r.rows) {
        const int s = sequence_of(a.r, p.t);
        if (s < a.r.sequences && offset_of(a.r, s) <= p.t) {
            const int len = length_of(a.r, s), token = len - (offset_of(a.r, s + 1) - p.t);
            if (token >= 0 && token < len) {
                p.block = block_of(a.c, a.r, s, token, p.h);
                p.j = token % kBlockTokens;
            }
        }
    }
    p.there = p.block && p.chunk * 8 < a.c.width;
    return p;
}

__device__ inline uint16_t *channels_of(const HeadRows &r, const Place &p) {
    return reinterpret_cast<uint16_t *>(r.p) + (int64_t)p.t * r.ld + (int64_t)p.h * r.head + p.chunk * 8;
}

// Where the eight channels of a key lie together, and the first of a value's.
__device__ inline int64_t key_at(const CacheView &c, const Place &p) { return ((int64_t)p.chunk * kBlockTokens + key_place(p.j)) * 8; }
__device__ inline int64_t value_at(const CacheView &c, const Place &p) {
    return (int64_t)kBlockTokens * c.width + ((int64_t)(p.j / 8) * c.width + p.chunk * 8) * 8 + p.j % 8;
}

template <int VB>
__global__ __launch_bounds__(kCacheThreads) void append_kernel(RowsArgs a) {
    const Place p = place_of(a);
    half8c x = {};
    if (p.there && p.chunk * 8 < a.c.head_dim) {
        const uint16_t *from = channels_of(p.value ? a.v : a.k, p);
        if (a.vec) {
            x = *reinterpret_cast<const half8c *>(from);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(_Float16, from[i]);
        }
    }
    if (VB == 2) {
        if (!p.there) return;
        uint16_t *to = reinterpret_cast<uint16_t *>(p.block);
        if (!p.value) {
            *reinterpret_cast<half8c *>(to + key_at(a.c, p)) = x;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[value_at(a.c, p) + 8 * i] = __builtin_bit_cast(uint16_t, (_Float16)x[i]);
        }
        return;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = std::max(top, magnitude_bits(x[i]));
#pragma unroll
    for (int d = 16; d >= 1; d /= 2) top = std::max(top, (uint32_t)__shfl_xor((int)top, d, kLanes64));
    float scale, inv;
    code_scale(top, scale, inv);
    if (!p.there) return;
    if (!p.value) {
        u32x2c w = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i / 4] |= code_bits(x[i], inv) << (8 * (i % 4));
        *reinterpret_cast<u32x2c *>(p.block + key_at(a.c, p)) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p.block[value_at(a.c, p) + 8 * i] = (uint8_t)code_bits(x[i], inv);
    }
    if (p.chunk == 0) {
        float *scales = reinterpret_cast<float *>(p.block + (int64_t)2 * kBlockTokens * a.c.width);
        scales[(p.value ? kBlockTokens : 0) + p.j] = scale;
    }
}

template <int VB>
__global__ __launch_bounds__(kCacheThreads) void read_kernel(RowsArgs a) {
    const Place p = place_of(a);
    if (!p.there || p.chunk * 8 >= a.c.head_dim) return;
    half8c x;
    if (VB == 2) {
        const uint16_t *from = reinterpret_cast<const uint16_t *>(p.block);
        if (!p.value) {
            x = *reinterpret_cast<const half8c *>(from + key_at(a.c, p));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(_Float16, from[value_at(a.c, p) + 8 * i]);
        }
    } else {
        const float scale =
            reinterpret_cast<const float *>(p.block + (int64_t)2 * kBlockTokens * a.c.width)[(p.value ? kBlockTokens : 0) + p.j];
        const int8_t *from = reinterpret_cast<const int8_t *>(p.block) + (p.value ? value_at(a.c, p) : key_at(a.c, p));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (_Float16)((float)from[p.value ? 8 * i : i] * scale);
    }
    uint16_t *to = channels_of(p.value ? a.v : a.k, p);
    if (a.vec) {
        *reinterpret_cast<half8c *>(to) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i] = __builtin_bit_cast(uint16_t, (_Float16)x[i]);
    }
}

// ---- Many rows of each sequence: a wavefront takes a head of eight tokens that lie together in their block, and turns
// their values in LDS, so that a unit of a channel's eight tokens is written (read) at once. A value at a time, 2133
// rows of 40 heads of 128 took 67 us into 8 bits and 57 back; both together take 36.

constexpr int kGroup = 8;
constexpr int kWavesOfGroups = kCacheThreads / kLanes64;

// Groups of the sequences before s at most: of n rows there are up to n / 8 + 2.
__device__ inline int first_group(const RowsView &r, int s) { return offset_of(r, s) / kGroup + 2 * s; }

template <int DS, int VB, bool WRITE>
__global__ __launch_bounds__(kCacheThreads) void group_kernel(RowsArgs a) {
    constexpr int W = 32 * DS, kChunks = W / 8, kTurns = (DS + 1) / 2;  // turns of 64 lanes over 8 x kChunks units
    __shared__ __attribute__((aligned(16))) _Float16 turned[kWavesOfGroups][kGroup][W + 8];
    __shared__ uint32_t tops[kWavesOfGroups][2][kGroup];
    const int lane = threadIdx.x & (kLanes64 - 1), wave = threadIdx.x / kLanes64;
    const int64_t index = (int64_t)blockIdx.x * kWavesOfGroups + wave;
    const int group = (int)(index / a.c.kv_heads), h = (int)(index - (int64_t)group * a.c.kv_heads);
    int s = 0, below = a.r.sequences;  // first_group(s) <= group < first_group(below)
    while (below - s > 1) {
        const int mid = (s + below) / 2;
        if (first_group(a.r, mid) <= group)
            s = mid;
        else
            below = mid;
    }
    const int off = offset_of(a.r, s), n = offset_of(a.r, s + 1) - off, len = length_of(a.r, s);
    const int begin = len - n > 0 ? len - n : 0, local = group - first_group(a.r, s);
    const int64_t from = ((int64_t)begin / kGroup + local) * kGroup;  // the group's first token
    uint8_t *block = nullptr;
    if (local >= 0 && n > 0 && from < len) block = block_of(a.c, a.r, s, (int)from, h);
    const int j0 = (int)(from % kBlockTokens);
    auto there = [&](int token) { return block && from + token >= begin && from + token < len; };
    const bool full = there(0) && there(kGroup - 1);
    auto row_of = [&](const HeadRows &r, int token, int chunk) {
        const int64_t t = off + (from + token - (len - n));
        return reinterpret_cast<uint16_t *>(r.p) + t * r.ld + (int64_t)h * r.head + chunk * 8;
    };
    uint8_t *values = block + kBlockTokens * W * VB + (j0 / 8) * W * 8 * VB;  // units of eight tokens, channel after channel
    float *scales = reinterpret_cast<float *>(block + 2 * kBlockTokens * W);
    if (VB == 1 && lane < 2 * kGroup) tops[wave][lane / kGroup][lane % kGroup] = 0;

    half8c k[kTurns], v[kTurns];
    if (WRITE) {
        if (VB == 1) __syncthreads();
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int u = i * kLanes64 + lane, token = u / kChunks, chunk = u % kChunks;
            k[i] = v[i] = half8c{};
            if (token < kGroup && there(token) && chunk * 8 < a.c.head_dim) {
                const uint16_t *pk = row_of(a.k, token, chunk), *pv = row_of(a.v, token, chunk);
                if (a.vec) {
                    k[i] = *reinterpret_cast<const half8c *>(pk);
                    v[i] = *reinterpret_cast<const half8c *>(pv);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        k[i][e] = __builtin_bit_cast(_Float16, pk[e]);
                        v[i][e] = __builtin_bit_cast(_Float16, pv[e]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int u = i * kLanes64 + lane, token = u / kChunks, chunk = u % kChunks;
            if (token >= kGroup) continue;
            *reinterpret_cast<half8c *>(&turned[wave][token][chunk * 8]) = v[i];
            if (VB == 1) {
                uint32_t top_k = 0, top_v = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    top_k = std::max(top_k, magnitude_bits(k[i][e]));
                    top_v = std::max(top_v, magnitude_bits(v[i][e]));
                }
                atomicMax(&tops[wave][0][token], top_k);
                atomicMax(&tops[wave][1][token], top_v);
            }
        }
        __syncthreads();
        float scale, inv;
        if (VB == 1 && lane < 2 * kGroup && there(lane % kGroup)) {
            code_scale(tops[wave][lane / kGroup][lane % kGroup], scale, inv);
            scales[(lane / kGroup) * kBlockTokens + j0 + lane % kGroup] = scale;
        }
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int u = i * kLanes64 + lane, token = u / kChunks, chunk = u % kChunks;
            if (token >= kGroup || !there(token)) continue;
            const int at = (chunk * kBlockTokens + key_place(j0 + token)) * 8;
            if (VB == 2) {
                *reinterpret_cast<half8c *>(reinterpret_cast<uint16_t *>(block) + at) = k[i];
            } else {
                code_scale(tops[wave][0][token], scale, inv);
                u32x2c w = {0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e / 4] |= code_bits(k[i][e], inv) << (8 * (e % 4));
                *reinterpret_cast<u32x2c *>(block + at) = w;
            }
        }
        float inv_v[kGroup];
        if (VB == 1) {
#pragma unroll
            for (int e = 0; e < kGroup; ++e) code_scale(tops[wave][1][e], scale, inv_v[e]);
        }
#pragma unroll
        for (int i = 0; i < (W + kLanes64 - 1) / kLanes64; ++i) {
            const int d = i * kLanes64 + lane;
            if (d >= W || !block) continue;
            half8c x;
#pragma unroll
            for (int e = 0; e < kGroup; ++e) x[e] = turned[wave][e][d];
            if (VB == 2) {
                if (full) {
                    *reinterpret_cast<half8c *>(reinterpret_cast<uint16_t *>(values) + d * 8) = x;
                } else {
#pragma unroll
                    for (int e = 0; e < kGroup; ++e)
                        if (there(e)) reinterpret_cast<uint16_t *>(values)[d * 8 + e] = __builtin_bit_cast(uint16_t, (_Float16)x[e]);
                }
            } else {
                u32x2c w = {0, 0};
#pragma unroll
                for (int e = 0; e < kGroup; ++e) w[e / 4] |= code_bits(x[e], inv_v[e]) << (8 * (e % 4));
                if (full) {
                    *reinterpret_cast<u32x2c *>(values + d * 8) = w;
                } else {
#pragma unroll
                    for (int e = 0; e < kGroup; ++e)
                        if (there(e)) values[d * 8 + e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
                }
            }
        }
        return;
    }

    float scale_v[kGroup];
    if (VB == 1) {
#pragma unroll
        for (int e = 0; e < kGroup; ++e) scale_v[e] = there(e) ? scales[kBlockTokens + j0 + e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int u = i * kLanes64 + lane, token = u / kChunks, chunk = u % kChunks;
        k[i] = half8c{};
        if (token >= kGroup || !there(token)) continue;
        const int at = (chunk * kBlockTokens + key_place(j0 + token)) * 8;
        if (VB == 2) {
            k[i] = *reinterpret_cast<const half8c *>(reinterpret_cast<const uint16_t *>(block) + at);
        } else {
            const u32x2c w = *reinterpret_cast<const u32x2c *>(block + at);
            const float scale = scales[j0 + token];
#pragma unroll
            for (int e = 0; e < 8; ++e) k[i][e] = (_Float16)((float)(int8_t)(w[e / 4] >> (8 * (e % 4))) * scale);
        }
    }
#pragma unroll
    for (int i = 0; i < (W + kLanes64 - 1) / kLanes64; ++i) {
        const int d = i * kLanes64 + lane;
        if (d >= W || !block) continue;
        half8c x;
        if (VB == 2) {
            x = *reinterpret_cast<const half8c *>(reinterpret_cast<const uint16_t *>(values) + d * 8);
        } else {
            const u32x2c w = *reinterpret_cast<const u32x2c *>(values + d * 8);
#pragma unroll
            for (int e = 0; e < kGroup; ++e) x[e] = (_Float16)((float)(int8_t)(w[e / 4] >> (8 * (e % 4))) * scale_v[e]);
        }
#pragma unroll
        for (int e = 0; e < kGroup; ++e) turned[wave][e][d] = x[e];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int u = i * kLanes64 + lane, token = u / kChunks, chunk = u % kChunks;
        if (token >= kGroup || !there(token) || chunk * 8 >= a.c.head_dim) continue;
        const half8c x = *reinterpret_cast<const half8c *>(&turned[wave][token][chunk * 8]);
        uint16_t *pk = row_of(a.k, token, chunk), *pv = row_of(a.v, token, chunk);
        if (a.vec) {
            *reinterpret_cast<half8c *>(pk) = k[i];
            *reinterpret_cast<half8c *>(pv) = x;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pk[e] = __builtin_bit_cast(uint16_t, (_Float16)k[i][e]);
                pv[e] = __builtin_bit_cast(uint16_t, (_Float16)x[e]);
            }
        }
    }
}

typedef void (*RowsFn)(RowsArgs);

template <int VB, bool WRITE>
RowsFn group_kernel_of(int width) {
    switch (width) {
        case 32: return group_kernel<1, VB, WRITE>;
        case 64: return group_kernel<2, VB, WRITE>;
        case 96: return group_kernel<3, VB, WRITE>;
        case 128: return group_kernel<4, VB, WRITE>;
        case 192: return group_kernel<6, VB, WRITE>;
        default: return group_kernel<8, VB, WRITE>;
    }
}

bool vector_heads(const HeadRows &r) {
    return (reinterpret_cast<uintptr_t>(r.p) & 15) == 0 && r.ld % 8 == 0 && r.head % 8 == 0;
}

// Groups where sequences have four rows or more on average: at fewer, most of a group's lanes have nothing to do.
bool in_groups(const RowsView &r) { return r.offsets && r.rows >= 4 * (int64_t)r.sequences; }

int64_t rows_grid(const CacheView &c, const RowsView &r) {
    const int64_t waves = (in_groups(r) ? (int64_t)r.rows / kGroup + 2 * (int64_t)r.sequences : (int64_t)r.rows) * c.kv_heads;
    return (waves + kWavesOfGroups - 1) / kWavesOfGroups;
}

template <bool WRITE>
int launch_rows(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream) {
    const RowsArgs a = {c, r, K, V, vector_heads(K) && vector_heads(V)};
    const bool groups = in_groups(r);
    RowsFn fn;
    if (groups)
        fn = c.value_bytes == 2 ? group_kernel_of<2, WRITE>(c.width) : group_kernel_of<1, WRITE>(c.width);
    else
        fn = WRITE ? c.value_bytes == 2 ? append_kernel<2> : append_kernel<1> : c.value_bytes == 2 ? read_kernel<2> : read_kernel<1>;
    hipLaunchKernelGGL(fn, dim3((unsigned)rows_grid(c, r)), dim3(kCacheThreads), 0, reinterpret_cast<hipStream_t>(stream), a);
    return (int)hipGetLastError();
}

// Pairs of pages by value: a launch's arguments hold so many.
constexpr int kPairs = 448;
constexpr int kCopyBytes = 16384;  // of a workgroup
struct CopyArgs {
    uint8_t *base;
    int64_t page_bytes, layer_bytes;
    int pairs, parts;  // parts of a page
    int32_t src[kPairs], dst[kPairs];
};

__global__ __launch_bounds__(kCacheThreads) void copy_kernel(CopyArgs a) {
    const int part = blockIdx.x % a.parts, pair = blockIdx.x / a.parts % a.pairs, layer = blockIdx.x / a.parts / a.pairs;
    uint8_t *layer_base = a.base + (int64_t)layer * a.layer_bytes;
    const uint8_t *from = layer_base + (int64_t)a.src[pair] * a.page_bytes;
    uint8_t *to = layer_base + (int64_t)a.dst[pair] * a.page_bytes;
    half8c x[kCopyBytes / 16 / kCacheThreads];
#pragma unroll
    for (int i = 0; i < kCopyBytes / 16 / kCacheThreads; ++i) {
        const int64_t at = (int64_t)part * kCopyBytes + (i * kCacheThreads + (int)threadIdx.x) * 16;
        if (at < a.page_bytes) x[i] = *reinterpret_cast<const half8c *>(from + at);
    }
#pragma unroll
    for (int i = 0; i < kCopyBytes / 16 / kCacheThreads; ++i) {
        const int64_t at = (int64_t)part * kCopyBytes + (i * kCacheThreads + (int)threadIdx.x) * 16;
        if (at < a.page_bytes) *reinterpret_cast<half8c *>(to + at) = x[i];
    }
}

}  // namespace

bool cache_rows_fit(const CacheView &c, const RowsView &r) { return rows_grid(c, r) <= kMostWorkgroups; }

int launch_cache_append(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream) {
    return launch_rows<true>(c, r, K, V, stream);
}

int launch_cache_read(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream) {
    return launch_rows<false>(c, r, K, V, stream);
}

int launch_cache_copy(const CacheView &c, int64_t layers, const int32_t *src, const int32_t *dst, int64_t n, void *stream) {
    CopyArgs a = {};
    a.base = c.base;
    a.page_bytes = c.page_bytes;
    a.layer_bytes = (int64_t)c.pages * c.page_bytes;
    a.parts = (int)((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
    const int64_t most = std::max<int64_t>(1, kMostWorkgroups / a.parts / kPairs);  // layers of a launch
    for (int64_t i = 0; i < n; i += kPairs) {
        a.pairs = (int)std::min<int64_t>(kPairs, n - i);
        std::copy(src + i, src + i + a.pairs, a.src);
        std::copy(dst + i, dst + i + a.pairs, a.dst);
        for (int64_t l = 0; l < layers; l += most) {
            CopyArgs b = a;
            b.base = a.base + l * a.layer_bytes;
            const int64_t grid = std::min(most, layers - l) * a.pairs * a.parts;
            hipLaunchKernelGGL(copy_kernel, dim3((unsigned)grid), dim3(kCacheThreads), 0,
                               reinterpret_cast<hipStream_t>(stream), b);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return (int)e;
        }
    }
    return 0;
}

}  // namespace usp
