// usp_cache.h -- a paged cache as the kernels see it: the geometry of include/usp.h's
// usp_cache and usp_cache_rows, for the host and the device.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "usp_internal.h"

namespace usp {

constexpr int kBlockTokens = 32;  // tokens of a block: the contraction of one MFMA over keys

// Channels of a head in the cache: head_dim rounded up to what a kernel is built for.
inline int cache_width(int head_dim) {
    for (int w : {32, 64, 96, 128, 192})
        if (head_dim <= w) return w;
    return 256;
}

constexpr int64_t cache_block_bytes(int width, int value_bytes) {
    return (int64_t)2 * kBlockTokens * width * value_bytes + (value_bytes == 1 ? 2 * kBlockTokens * 4 : 0);
}

struct CacheView {
    uint8_t *base;         // page 0 of the layer
    int64_t page_bytes;
    uint32_t pages;
    int kv_heads, head_dim, width;
    int page_tokens, page_blocks;
    int value_bytes;
};
inline CacheView cache_view(const usp_cache &c, int64_t layer) {
    CacheView v;
    v.kv_heads = c.kv_heads;
    v.head_dim = c.head_dim;
    v.width = cache_width(c.head_dim);
    v.page_tokens = c.page_tokens;
    v.page_blocks = c.page_tokens / kBlockTokens;
    v.value_bytes = c.value_bytes;
    v.page_bytes = cache_block_bytes(v.width, c.value_bytes) * v.page_blocks * c.kv_heads;
    v.pages = (uint32_t)c.pages;
    v.base = reinterpret_cast<uint8_t *>(c.data) + layer * c.pages * v.page_bytes;
    return v;
}

struct RowsView {
    const int32_t *table, *lengths, *offsets;
    int64_t ld_table;
    int sequences, rows;
    int capacity;          // tokens that a sequence's row of the table has room for
};
inline RowsView rows_view(const usp_cache_rows &r, const usp_cache &c) {
    return {r.table, r.lengths, r.offsets, r.ld_table, (int)r.sequences, (int)r.rows, (int)(r.table_pages * c.page_tokens)};
}

// A token's place in its block of keys: bits 2 and 3 exchanged, so that the rows of S = K Q^T
// that a lane gets are the 8 consecutive keys which it hands over for O = V^T P.
__host__ __device__ inline int key_place(int j) { return (j & ~12) | (j & 4) << 1 | (j & 8) >> 1; }

__device__ inline int clamped(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Tokens of sequence s in the cache, and the rows that it has in the step.
__device__ inline int length_of(const RowsView &r, int s) { return clamped(r.lengths[s], 0, r.capacity); }
__device__ inline int offset_of(const RowsView &r, int s) { return r.offsets ? clamped(r.offsets[s], 0, r.rows) : s; }

// The sequence that row t belongs to: the first whose rows end behind t, or `sequences`.
__device__ inline int sequence_of(const RowsView &r, int t) {
    if (!r.offsets) return t;
    int lo = 0, hi = r.sequences;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (offset_of(r, mid + 1) > t)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

// The block of head h that holds token `token` (within capacity) of sequence s; null where its page is none of the cache's.
__device__ inline uint8_t *block_of(const CacheView &c, const RowsView &r, int s, int token, int h) {
    const int in = token / c.page_tokens, rest = token - in * c.page_tokens;
    const uint32_t page = (uint32_t)r.table[(int64_t)s * r.ld_table + in];
    if (page >= c.pages) return nullptr;
    return c.base + (int64_t)page * c.page_bytes +
           ((int64_t)h * c.page_blocks + rest / kBlockTokens) * cache_block_bytes(c.width, c.value_bytes);
}

constexpr int64_t kMostWorkgroups = ((int64_t)1 << 24) - 1;  // of a launch of 256 threads each: they are counted in 32 bits

// Launchers (usp_cache.hip, usp_attention.hip): hipSuccess or the launch's error.
struct HeadRows {          // rows of heads of fp16
    void *p;
    int64_t ld, head;      // strides of rows and heads in elements
};
bool cache_rows_fit(const CacheView &c, const RowsView &r);  // one launch takes them
int launch_cache_append(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream);
int launch_cache_read(const CacheView &c, const RowsView &r, HeadRows K, HeadRows V, void *stream);
int launch_cache_copy(const CacheView &c, int64_t layers, const int32_t *src, const int32_t *dst, int64_t n, void *stream);
size_t attention_workspace_bytes(const CacheView &c, const RowsView &r, int heads);
std::string describe_attention(const CacheView &c, const RowsView &r, int heads);
bool attention_fits(const CacheView &c, const RowsView &r, int heads);  // one launch takes it
int launch_attention(const CacheView &c, const RowsView &r, const usp_attention_args &p, void *workspace, void *stream);

}  // namespace usp
