// usp_cache.hip -- new tokens into a paged cache and back, and copies of its pages
// (include/usp.h, usp_cache_append, usp_cache_read, usp_cache_copy).
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

bool vector_heads(const HeadRows &r) {
    return (reinterpret_cast<uintptr_t>(r.p) & 15) == 0 && r.ld % 8 == 0 && r.head % 8 == 0;
}

int launch_rows(void (*fn)(RowsArgs), const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream) {
    const RowsArgs a = {c, r, K, V, vector_heads(K) && vector_heads(V)};
    const int64_t grid = ((int64_t)r.rows * c.kv_heads + 3) / (kCacheThreads / kLanes64);
    hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(kCacheThreads), 0, reinterpret_cast<hipStream_t>(stream), a);
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

int launch_cache_append(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream) {
    return launch_rows(c.value_bytes == 2 ? append_kernel<2> : append_kernel<1>, c, r, K, V, stream);
}

int launch_cache_read(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream) {
    return launch_rows(c.value_bytes == 2 ? read_kernel<2> : read_kernel<1>, c, r, K, V, stream);
}

int launch_cache_copy(const CacheView &c, int64_t layers, const int32_t *src, const int32_t *dst, int64_t n, void *stream) {
    CopyArgs a = {};
    a.base = c.base;
    a.page_bytes = c.page_bytes;
    a.layer_bytes = (int64_t)c.pages * c.page_bytes;
    a.parts = (int)((c.page_bytes + kCopyBytes - 1) / kCopyBytes);
    const int64_t most = std::max<int64_t>(1, (((int64_t)1 << 30) / a.parts) / kPairs);  // layers of a launch
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
