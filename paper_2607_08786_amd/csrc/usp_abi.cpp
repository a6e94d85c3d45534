// usp_abi.cpp -- the extern "C" entry points declared in include/usp.h:
// argument checking, handle lifetime, host<->device transfers, error strings.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <mutex>
#include <new>
#include <string>
#include <unordered_set>

#include "usp_cache.h"
#include "usp_internal.h"

namespace {

thread_local std::string g_last_error;

// Makes `dev` current for the scope and restores the caller's device after.
struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = (prev == dev) || hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

// Every handle usp_encode returned and usp_free has not released. A handle is
// checked against this set before it is dereferenced, so a freed (or never
// issued) pointer is reported instead of read.
std::mutex g_live_mu;
std::unordered_set<const usp_matrix *> g_live;
std::unordered_set<const usp_group *> g_live_groups;

bool alive(const usp_matrix *A) {
    if (!A) return false;
    std::lock_guard<std::mutex> lk(g_live_mu);
    return g_live.count(A) != 0;
}

bool alive(const usp_group *G) {
    if (!G) return false;
    std::lock_guard<std::mutex> lk(g_live_mu);
    return g_live_groups.count(G) != 0;
}

// Releases a handle's device memory and the handle itself (registered or not).
void release(usp_matrix *A) {
    {
        DeviceGuard g(A->device);
        if (A->d_stream) (void)hipFree(A->d_stream);
        if (A->d_off) (void)hipFree(A->d_off);
        if (A->d_scale) (void)hipFree(A->d_scale);
    }
    delete A;
}

usp_status hip_fail(hipError_t e, const char *what) {
    return usp::fail(USP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

}  // namespace

namespace usp {
usp_status fail(usp_status st, const std::string &msg) {
    g_last_error = msg;
    return st;
}
}  // namespace usp

// What usp_spmm_q and usp_spmm_grouped check and do alike.
static usp_status product_common(const std::string &f, const usp::ProductShape &s, int device,
                                 const usp::ProductCall &c, void *workspace, size_t ws_bytes, void *stream) {
    if (!c.X || !c.Y) return usp::fail(USP_ERR_INVALID_ARG, f + ": null X or Y");
    if (c.N > (int64_t)1 << 20 || !usp::product_fits(s, c.N)) return usp::fail(USP_ERR_UNSUPPORTED, f + ": too many tokens");
    if (c.ldx < s.K) return usp::fail(USP_ERR_INVALID_ARG, f + ": ldx must be >= K");
    if (c.ldy < s.M) return usp::fail(USP_ERR_INVALID_ARG, f + ": ldy must be >= M");
    if ((reinterpret_cast<uintptr_t>(c.X) & (c.quantize ? 1 : s.value_bytes - 1)) || (reinterpret_cast<uintptr_t>(c.Y) & 1))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": X and Y must be aligned to their elements");
    if (reinterpret_cast<uintptr_t>(c.x_scale) & 3)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": x_scale must be 4-byte aligned");
    if (c.ep.act < USP_ACT_NONE || c.ep.act > USP_ACT_SILU)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": unknown activation");
    if (reinterpret_cast<uintptr_t>(c.ep.bias) & 1)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": bias must be 2-byte aligned");
    const size_t need = usp::product_workspace_bytes(s, c.N);
    if (need && (!workspace || ws_bytes < need))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": workspace too small");
    if (need && (reinterpret_cast<uintptr_t>(workspace) & 15))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": workspace must be 16-byte aligned");
    DeviceGuard g(device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, f + ": cannot select device");
    const int rc = usp::launch_product(s, c, workspace, stream);
    if (rc != 0) return hip_fail((hipError_t)rc, (f + ": launch").c_str());
    return USP_OK;
}

// What usp_norm and usp_quantize check and do alike.
static usp_status norm_common(const char *fn, const usp_norm_args &p, int64_t N, int64_t K, int device, void *stream) {
    const std::string f(fn);
    if (N < 1 || K < 1) return usp::fail(USP_ERR_INVALID_ARG, f + ": N and K must be >= 1");
    if (N > (int64_t)1 << 20 || K > (int64_t)1 << 28)
        return usp::fail(USP_ERR_UNSUPPORTED, f + ": N above 2^20 or K above 2^28");
    if (!p.residual) return usp::fail(USP_ERR_INVALID_ARG, f + ": null input");
    if (!p.residual_out && !p.out && !p.out_q) return usp::fail(USP_ERR_INVALID_ARG, f + ": no output");
    if (p.out_q && !p.out_scale) return usp::fail(USP_ERR_INVALID_ARG, f + ": out_q needs out_scale");
    if (p.post_kind < USP_NORM_NONE || p.post_kind > USP_NORM_LAYER || p.pre_kind < USP_NORM_NONE ||
        p.pre_kind > USP_NORM_LAYER)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": unknown norm");
    if (p.gate_activation < USP_GATE_NONE || p.gate_activation > USP_GATE_SILU)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": unknown gate activation");
    if (!p.y && (p.post_kind || p.gate)) return usp::fail(USP_ERR_INVALID_ARG, f + ": a norm after the block and a gate need y");
    if (!(p.eps >= 0.f)) return usp::fail(USP_ERR_INVALID_ARG, f + ": eps must be >= 0");
    const struct {
        const void *p;
        int64_t ld;
        uintptr_t align;
    } operands[] = {{p.residual, p.ld_residual, 1},   {p.y, p.ld_y, 1},
                    {p.gate, p.ld_gate ? p.ld_gate : K, 1}, {p.residual_out, p.ld_residual_out, 1},
                    {p.out, p.ld_out, 1},             {p.out_q, p.ld_out_q, 0},
                    {p.out_scale, K, 3},              {p.post_weight, K, 1},
                    {p.post_bias, K, 1},              {p.pre_weight, K, 1},
                    {p.pre_bias, K, 1}};
    for (const auto &o : operands) {
        if (!o.p) continue;
        if (o.ld < K) return usp::fail(USP_ERR_INVALID_ARG, f + ": strides must be >= K");
        if (reinterpret_cast<uintptr_t>(o.p) & o.align)
            return usp::fail(USP_ERR_INVALID_ARG, f + ": operands must be aligned to their elements");
    }
    int ndev = 0;
    if (device < 0 || hipGetDeviceCount(&ndev) != hipSuccess || device >= ndev)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": no such device");
    DeviceGuard g(device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, f + ": cannot select device");
    const int rc = usp::launch_norm(p, N, K, stream);
    if (rc != 0) return hip_fail((hipError_t)rc, (f + ": launch").c_str());
    return USP_OK;
}

// Why a cache's description is none; null where it is one. `memory`: its pool too.
static const char *wrong_cache(const usp_cache *c, bool memory) {
    if (!c) return ": null cache";
    if (c->kv_heads < 1 || c->kv_heads > 4096) return ": kv_heads must be 1 to 4096";
    if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8) return ": head_dim must be a multiple of 8 up to 256";
    if (c->page_tokens < 32 || c->page_tokens > 4096 || c->page_tokens % 32)
        return ": page_tokens must be a multiple of 32 up to 4096";
    if (c->value_bytes != 1 && c->value_bytes != 2) return ": value_bytes must be 1 or 2";
    if (!memory) return nullptr;
    if (!c->data || (reinterpret_cast<uintptr_t>(c->data) & 15)) return ": the cache's data must be 16-byte aligned";
    if (c->layers < 1 || c->pages < 1 || c->pages > 0x7FFFFFFF) return ": layers and pages must be >= 1, pages below 2^31";
    return nullptr;
}

// The same of a step's rows; `pointers`: those too.
static const char *wrong_rows(const usp_cache_rows *r, const usp_cache &c, bool pointers) {
    if (!r) return ": null rows";
    if (r->rows < 0 || r->rows > (int64_t)1 << 20) return ": rows must be 0 to 2^20";
    if (r->sequences < 1 || r->sequences > (int64_t)1 << 20) return ": sequences must be 1 to 2^20";
    if (!r->offsets && r->rows != r->sequences && r->rows != 0) return ": without offsets there is one row for each sequence";
    if (r->table_pages < 1 || r->table_pages > (0x7FFFFFFF - 4096) / c.page_tokens)
        return ": table_pages must be >= 1, its tokens below 2^31 - 4096";
    if (!pointers) return nullptr;
    if (!r->table || !r->lengths) return ": null table or lengths";
    if (r->ld_table < r->table_pages) return ": ld_table must be >= table_pages";
    for (const void *p : {(const void *)r->table, (const void *)r->lengths, (const void *)r->offsets})
        if (reinterpret_cast<uintptr_t>(p) & 3) return ": table, lengths and offsets must be 4-byte aligned";
    return nullptr;
}

// Whether rows of heads of an output lie apart from each other.
static bool lie_apart(int64_t ld, int64_t head, int64_t rows, int64_t heads, int64_t dim) {
    const auto inside = [dim](int64_t inner, int64_t n, int64_t outer, int64_t m) {
        return (n == 1 || inner >= dim) && (m == 1 || (outer >= dim && (outer - dim) / (n > 1 ? n - 1 : 1) >= (n > 1 ? inner : 0)));
    };
    return inside(head, heads, ld, rows) || inside(ld, rows, head, heads);
}

static bool select_device(int device, DeviceGuard &g) {
    int ndev = 0;
    return device >= 0 && hipGetDeviceCount(&ndev) == hipSuccess && device < ndev && g.ok;
}

// What usp_cache_append and usp_cache_read check and do alike.
static usp_status cache_rows_common(const std::string &f, const usp_cache *cache, const usp_cache_rows *rows, int64_t layer,
                                    usp::HeadRows K, usp::HeadRows V, bool write, void *stream) {
    if (const char *why = wrong_cache(cache, true)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (const char *why = wrong_rows(rows, *cache, true)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (layer < 0 || layer >= cache->layers) return usp::fail(USP_ERR_INVALID_ARG, f + ": no such layer");
    if (rows->rows == 0) return USP_OK;
    if (!K.p || !V.p) return usp::fail(USP_ERR_INVALID_ARG, f + ": null K or V");
    if ((reinterpret_cast<uintptr_t>(K.p) | reinterpret_cast<uintptr_t>(V.p)) & 1)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": K and V must be 2-byte aligned");
    for (const usp::HeadRows &r : {K, V}) {
        if (r.ld < 0 || r.head < 0) return usp::fail(USP_ERR_INVALID_ARG, f + ": strides must be >= 0");
        if (!write && !lie_apart(r.ld, r.head, rows->rows, cache->kv_heads, cache->head_dim))
            return usp::fail(USP_ERR_INVALID_ARG, f + ": rows and heads of K and V must lie apart");
    }
    const usp::CacheView c = usp::cache_view(*cache, layer);
    const usp::RowsView r = usp::rows_view(*rows, *cache);
    if (!usp::cache_rows_fit(c, r)) return usp::fail(USP_ERR_UNSUPPORTED, f + ": too many rows and heads");
    DeviceGuard g(cache->device);
    if (!select_device(cache->device, g)) return usp::fail(USP_ERR_INVALID_ARG, f + ": no such device");
    const int rc = write ? usp::launch_cache_append(c, r, K, V, stream) : usp::launch_cache_read(c, r, K, V, stream);
    if (rc != 0) return hip_fail((hipError_t)rc, (f + ": launch").c_str());
    return USP_OK;
}

extern "C" {

const char *usp_last_error(void) { return g_last_error.c_str(); }

// The checks and the device part of usp_encode and usp_encode_q (scale: host scales
// of the rows, or null for fp16 values); encode fills the records.
static usp_status encode_common(const char *fn, const void *W, int64_t ldw, const uint8_t *mask, int64_t ldm,
                                const float *scale, int64_t M, int64_t K, int device, usp_matrix **out,
                                void (*encode)(const void *, int64_t, const uint8_t *, int64_t, int64_t, int64_t,
                                               usp::HostEncoding &)) {
    const std::string f(fn);
    if (out) *out = nullptr;
    if (!out || !W || !mask) return usp::fail(USP_ERR_INVALID_ARG, f + ": null pointer");
    if (M < 1 || K < 1) return usp::fail(USP_ERR_INVALID_ARG, f + ": M and K must be >= 1");
    if (ldw < K || ldm < K) return usp::fail(USP_ERR_INVALID_ARG, f + ": ldw and ldm must be >= K");
    if (M > usp::kMaxRows)
        return usp::fail(USP_ERR_UNSUPPORTED, f + ": M above 2^20 rows (the workspace's arrival counters)");
    if (scale && K > USP_MAX_K_Q) return usp::fail(USP_ERR_UNSUPPORTED, f + ": K above USP_MAX_K_Q");
    for (int64_t m = 0; scale && m < M; ++m)
        if (!std::isfinite(scale[m])) return usp::fail(USP_ERR_INVALID_ARG, f + ": scales must be finite");
    int ndev = 0;
    hipError_t e = hipGetDeviceCount(&ndev);
    if (e != hipSuccess) return hip_fail(e, (f + ": hipGetDeviceCount").c_str());
    if (device < 0 || device >= ndev) return usp::fail(USP_ERR_INVALID_ARG, f + ": no such device");

    usp::HostEncoding enc;
    std::vector<float> scales;  // of whole row blocks
    try {
        encode(W, ldw, mask, ldm, M, K, enc);
        if (scale) {
            scales.assign((size_t)enc.RB * usp::kTileRows, 0.f);
            std::copy(scale, scale + M, scales.begin());
        }
    } catch (const std::exception &) {  // bad_alloc, or length_error of sizes that no vector has
        return usp::fail(USP_ERR_OOM, f + ": host allocation failed (or encoding exceeds 64 GiB)");
    }
    DeviceGuard g(device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, f + ": cannot select device");
    usp_matrix *A = new (std::nothrow) usp_matrix();
    if (!A) return usp::fail(USP_ERR_OOM, f + ": host allocation failed");
    A->device = device;
    A->M = M;
    A->K = K;
    A->RB = enc.RB;
    A->KT = enc.KT;
    A->nnz = enc.nnz;
    A->max_chunks = enc.max_chunks;
    A->stream_bytes = enc.stream.size();
    A->d_stream = nullptr;
    A->d_off = nullptr;
    A->num_cus = 0;
    A->value_bytes = scale ? 1 : 2;
    A->d_scale = nullptr;
    A->groups = 0;
    if (hipDeviceGetAttribute(&A->num_cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess)
        A->num_cus = 0;
    // The kernels' last load of a record may read up to 1 KB past it.
    e = hipMalloc(&A->d_stream, A->stream_bytes + usp::kStreamPad);
    if (e == hipSuccess) e = hipMemset(reinterpret_cast<uint8_t *>(A->d_stream) + A->stream_bytes, 0, usp::kStreamPad);
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void **>(&A->d_off), enc.off.size() * sizeof(uint32_t));
    if (e == hipSuccess && scale) e = hipMalloc(reinterpret_cast<void **>(&A->d_scale), scales.size() * sizeof(float));
    if (e != hipSuccess) {
        release(A);
        return usp::fail(USP_ERR_OOM, f + std::string(": hipMalloc: ") + hipGetErrorString(e));
    }
    // One-time set-up of this device's scratch for usp_spmm_noalloc (outside
    // any graph capture: encoding precedes every product).
    if (e == hipSuccess) e = (hipError_t)usp::noalloc_setup(device);
    if (e != hipSuccess) {
        release(A);
        return hip_fail(e, (f + ": device scratch set-up").c_str());
    }
    e = hipMemcpy(A->d_stream, enc.stream.data(), A->stream_bytes, hipMemcpyHostToDevice);
    if (e == hipSuccess)
        e = hipMemcpy(A->d_off, enc.off.data(), enc.off.size() * sizeof(uint32_t), hipMemcpyHostToDevice);
    if (e == hipSuccess && scale)
        e = hipMemcpy(A->d_scale, scales.data(), scales.size() * sizeof(float), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        release(A);
        return hip_fail(e, (f + ": hipMemcpy").c_str());
    }
    try {
        std::lock_guard<std::mutex> lk(g_live_mu);
        g_live.insert(A);
    } catch (const std::bad_alloc &) {
        release(A);
        return usp::fail(USP_ERR_OOM, f + ": host allocation failed");
    }
    *out = A;
    return USP_OK;
}

usp_status usp_encode(const uint16_t *W, int64_t ldw, const uint8_t *mask, int64_t ldm, int64_t M, int64_t K,
                      int device, usp_matrix **out) {
    return encode_common("usp_encode", W, ldw, mask, ldm, nullptr, M, K, device, out,
                         [](const void *w, int64_t lw, const uint8_t *m, int64_t lm, int64_t rows, int64_t cols,
                            usp::HostEncoding &enc) {
                             usp::encode_host(static_cast<const uint16_t *>(w), lw, m, lm, rows, cols, enc);
                         });
}

usp_status usp_encode_q(const int8_t *W, int64_t ldw, const uint8_t *mask, int64_t ldm, const float *scale,
                        int64_t M, int64_t K, int device, usp_matrix **out) {
    if (!scale) {
        if (out) *out = nullptr;
        return usp::fail(USP_ERR_INVALID_ARG, "usp_encode_q: null pointer");
    }
    return encode_common("usp_encode_q", W, ldw, mask, ldm, scale, M, K, device, out,
                         [](const void *w, int64_t lw, const uint8_t *m, int64_t lm, int64_t rows, int64_t cols,
                            usp::HostEncoding &enc) {
                             usp::encode_host_q(static_cast<const int8_t *>(w), lw, m, lm, rows, cols, enc);
                         });
}

size_t usp_workspace_size(const usp_matrix *A, int64_t N) {
    if (!alive(A) || N < 1) return 0;
    if (A->value_bytes == 1) return usp::product_workspace_bytes(usp::product_shape(A), N);
    return usp::spmm_workspace_bytes(A, N);
}

static usp_status copy_text(const std::string &d, char *buf, size_t len) {
    const size_t n = d.size() < len - 1 ? d.size() : len - 1;
    std::memcpy(buf, d.data(), n);
    buf[n] = '\0';
    return USP_OK;
}

usp_status usp_plan(const usp_matrix *A, int64_t N, char *buf, size_t len) {
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, "usp_plan: invalid or freed handle");
    if (N < 1 || !buf || len == 0) return usp::fail(USP_ERR_INVALID_ARG, "usp_plan: need N >= 1 and a buffer");
    DeviceGuard g(A->device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, "usp_plan: cannot select device");
    const std::string d =
        A->value_bytes == 1 ? usp::describe_product(usp::product_shape(A), N) : usp::describe_plan(A, N);
    return copy_text(d, buf, len);
}

// The text of usp_spmm's refusal of a handle of the other value type, or null.
static const char *wrong_values(const usp_matrix *A, int value_bytes) {
    if (A->value_bytes == value_bytes) return nullptr;
    return A->value_bytes == 1 ? ": the handle holds 8-bit weights (use usp_spmm_q)"
                               : ": the handle holds fp16 weights (use usp_spmm)";
}

static usp_status spmm_common(const char *fn, const usp_matrix *A, const void *X, int64_t ldx, void *Y,
                              int64_t ldy, int64_t N, const usp::Epilogue &ep, void *workspace, size_t ws_bytes,
                              void *stream) {
    const std::string f(fn);
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, f + ": invalid or freed handle");
    if (const char *why = wrong_values(A, 2)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (!X || !Y) return usp::fail(USP_ERR_INVALID_ARG, f + ": null X or Y");
    if (N < 1) return usp::fail(USP_ERR_INVALID_ARG, f + ": N must be >= 1");
    if (N > (int64_t)1 << 20) return usp::fail(USP_ERR_UNSUPPORTED, f + ": N too large");
    if (ldx < A->K) return usp::fail(USP_ERR_INVALID_ARG, f + ": ldx must be >= K");
    if (ldy < A->M) return usp::fail(USP_ERR_INVALID_ARG, f + ": ldy must be >= M");
    if ((reinterpret_cast<uintptr_t>(X) & 1) || (reinterpret_cast<uintptr_t>(Y) & 1))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": X and Y must be 2-byte aligned");
    if (ep.act < USP_ACT_NONE || ep.act > USP_ACT_SILU)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": unknown activation");
    if (reinterpret_cast<uintptr_t>(ep.bias) & 1) return usp::fail(USP_ERR_INVALID_ARG, f + ": bias must be 2-byte aligned");
    if (ep.res && ((reinterpret_cast<uintptr_t>(ep.res) & 1) || ep.ldr < A->M))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": residual must be 2-byte aligned with ldr >= M");
    const size_t need = usp::spmm_workspace_min_bytes(A, N);
    if (need && (!workspace || ws_bytes < need))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": workspace too small (see usp_workspace_size)");
    if (need && (reinterpret_cast<uintptr_t>(workspace) & 15))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": workspace must be 16-byte aligned");
    DeviceGuard g(A->device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, f + ": cannot select device");
    const int rc = usp::launch_spmm(A, X, ldx, Y, ldy, N, ep, workspace, ws_bytes, stream);
    if (rc != 0) return hip_fail((hipError_t)rc, (f + ": launch").c_str());
    return USP_OK;
}

usp_status usp_spmm(const usp_matrix *A, const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t N,
                    void *workspace, size_t ws_bytes, void *stream) {
    return spmm_common("usp_spmm", A, X, ldx, Y, ldy, N, usp::Epilogue(), workspace, ws_bytes, stream);
}

usp_status usp_spmm_ex(const usp_matrix *A, const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t N,
                       const void *bias, const void *residual, int64_t ldr, int activation, void *workspace,
                       size_t ws_bytes, void *stream) {
    usp::Epilogue ep;
    ep.bias = reinterpret_cast<const uint16_t *>(bias);
    ep.res = reinterpret_cast<const uint16_t *>(residual);
    ep.ldr = ldr;
    ep.act = activation;
    return spmm_common("usp_spmm_ex", A, X, ldx, Y, ldy, N, ep, workspace, ws_bytes, stream);
}

usp_status usp_spmm_noalloc(const usp_matrix *A, const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t N,
                            void *stream) {
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, "usp_spmm_noalloc: invalid or freed handle");
    if (const char *why = wrong_values(A, 2)) return usp::fail(USP_ERR_INVALID_ARG, std::string("usp_spmm_noalloc") + why);
    if (N < 1) return usp::fail(USP_ERR_INVALID_ARG, "usp_spmm_noalloc: N must be >= 1");
    const size_t need = usp::spmm_workspace_min_bytes(A, N);
    if (need > USP_NOALLOC_SCRATCH_BYTES)
        return usp::fail(USP_ERR_UNSUPPORTED, "usp_spmm_noalloc: this product needs " + std::to_string(need) +
                                                  " bytes of workspace, above the " +
                                                  std::to_string((size_t)USP_NOALLOC_SCRATCH_BYTES) +
                                                  "-byte device scratch (use usp_spmm with a workspace)");
    void *ws = usp::noalloc_scratch(A->device);
    if (!ws) return usp::fail(USP_ERR_INTERNAL, "usp_spmm_noalloc: device scratch not set up");
    return spmm_common("usp_spmm_noalloc", A, X, ldx, Y, ldy, N, usp::Epilogue(), ws, USP_NOALLOC_SCRATCH_BYTES,
                       stream);
}

usp_status usp_densify(const usp_matrix *A, void *Wd, int64_t ldw, void *stream) {
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, "usp_densify: invalid or freed handle");
    if (!Wd) return usp::fail(USP_ERR_INVALID_ARG, "usp_densify: null output");
    if (ldw < A->K) return usp::fail(USP_ERR_INVALID_ARG, "usp_densify: ldw must be >= K");
    if (reinterpret_cast<uintptr_t>(Wd) & 1) return usp::fail(USP_ERR_INVALID_ARG, "usp_densify: misaligned output");
    DeviceGuard g(A->device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, "usp_densify: cannot select device");
    const int rc = A->value_bytes == 1 ? usp::launch_densify_q(A, Wd, ldw, stream) : usp::launch_densify(A, Wd, ldw, stream);
    if (rc != 0) return hip_fail((hipError_t)rc, "usp_densify: launch");
    return USP_OK;
}

// Copies the encoding of A back to the host.
static usp_status fetch_encoding(const std::string &f, const usp_matrix *A, usp::HostEncoding &enc) {
    try {
        enc.M = A->M;
        enc.K = A->K;
        enc.RB = A->RB;
        enc.KT = A->KT;
        enc.nnz = A->nnz;
        enc.off.resize(A->RB * A->KT + 1);
        enc.stream.resize(A->stream_bytes);
    } catch (const std::bad_alloc &) {
        return usp::fail(USP_ERR_OOM, f + ": host allocation failed");
    }
    DeviceGuard g(A->device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, f + ": cannot select device");
    hipError_t e = hipMemcpy(enc.stream.data(), A->d_stream, A->stream_bytes, hipMemcpyDeviceToHost);
    if (e == hipSuccess)
        e = hipMemcpy(enc.off.data(), A->d_off, enc.off.size() * sizeof(uint32_t), hipMemcpyDeviceToHost);
    if (e != hipSuccess) return hip_fail(e, (f + ": hipMemcpy").c_str());
    return USP_OK;
}

usp_status usp_decode(const usp_matrix *A, uint16_t *W_out, uint8_t *mask_out) {
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, "usp_decode: invalid or freed handle");
    if (A->value_bytes != 2)
        return usp::fail(USP_ERR_INVALID_ARG, "usp_decode: the handle holds 8-bit weights (use usp_decode_q)");
    if (!W_out || !mask_out) return usp::fail(USP_ERR_INVALID_ARG, "usp_decode: null output");
    usp::HostEncoding enc;
    if (const usp_status st = fetch_encoding("usp_decode", A, enc)) return st;
    if (!usp::decode_host(enc, W_out, mask_out))
        return usp::fail(USP_ERR_INTERNAL, "usp_decode: encoding is inconsistent");
    return USP_OK;
}

usp_status usp_decode_q(const usp_matrix *A, int8_t *W_out, uint8_t *mask_out, float *scale_out) {
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, "usp_decode_q: invalid or freed handle");
    if (A->value_bytes != 1)
        return usp::fail(USP_ERR_INVALID_ARG, "usp_decode_q: the handle holds fp16 weights (use usp_decode)");
    if (!W_out || !mask_out || !scale_out) return usp::fail(USP_ERR_INVALID_ARG, "usp_decode_q: null output");
    usp::HostEncoding enc;
    if (const usp_status st = fetch_encoding("usp_decode_q", A, enc)) return st;
    DeviceGuard g(A->device);
    if (!g.ok) return usp::fail(USP_ERR_HIP, "usp_decode_q: cannot select device");
    const hipError_t e = hipMemcpy(scale_out, A->d_scale, (size_t)A->M * sizeof(float), hipMemcpyDeviceToHost);
    if (e != hipSuccess) return hip_fail(e, "usp_decode_q: hipMemcpy");
    if (!usp::decode_host_q(enc, W_out, mask_out))
        return usp::fail(USP_ERR_INTERNAL, "usp_decode_q: encoding is inconsistent");
    return USP_OK;
}

usp_status usp_info(const usp_matrix *A, usp_info_t *info) {
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, "usp_info: invalid or freed handle");
    if (!info) return usp::fail(USP_ERR_INVALID_ARG, "usp_info: null output");
    std::memset(info, 0, sizeof(*info));
    info->M = A->M;
    info->K = A->K;
    info->nnz = A->nnz;
    info->device_bytes = A->stream_bytes;
    info->table_bytes = (size_t)(A->RB * A->KT + 1) * sizeof(uint32_t);
    info->format_version = A->value_bytes == 1 ? USP_FORMAT_VERSION_Q : USP_FORMAT_VERSION;
    info->tile_rows = usp::kTileRows;
    info->tile_k = usp::kTileK;
    info->device = A->device;
    return USP_OK;
}

usp_status usp_free(usp_matrix *A) {
    if (!A) return USP_OK;
    {
        std::lock_guard<std::mutex> lk(g_live_mu);
        const auto it = g_live.find(A);
        if (it == g_live.end()) return usp::fail(USP_ERR_INVALID_ARG, "usp_free: invalid or already freed handle");
        if (A->groups > 0) return usp::fail(USP_ERR_INVALID_ARG, "usp_free: a group holds this handle (usp_group_free first)");
        g_live.erase(it);
    }
    release(A);
    return USP_OK;
}

usp_status usp_quantize(const void *X, int64_t ldx, int64_t N, int64_t K, void *Xq, int64_t ldq, float *x_scale,
                        int device, void *stream) {
    if (!X || !Xq || !x_scale) return usp::fail(USP_ERR_INVALID_ARG, "usp_quantize: null pointer");
    usp_norm_args p = {};
    p.residual = X;
    p.ld_residual = ldx;
    p.out_q = Xq;
    p.ld_out_q = ldq;
    p.out_scale = x_scale;
    return norm_common("usp_quantize", p, N, K, device, stream);
}

usp_status usp_norm(const usp_norm_args *args, int64_t N, int64_t K, int device, void *stream) {
    if (!args) return usp::fail(USP_ERR_INVALID_ARG, "usp_norm: null arguments");
    return norm_common("usp_norm", *args, N, K, device, stream);
}

usp_status usp_spmm_q(const usp_matrix *A, const void *Xq, int64_t ldx, const float *x_scale, void *Y, int64_t ldy,
                      int64_t N, const void *bias, const void *residual, int64_t ldr, int activation,
                      void *workspace, size_t ws_bytes, void *stream) {
    const std::string f("usp_spmm_q");
    if (!alive(A)) return usp::fail(USP_ERR_INVALID_ARG, f + ": invalid or freed handle");
    if (const char *why = wrong_values(A, 1)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (N < 1) return usp::fail(USP_ERR_INVALID_ARG, f + ": N must be >= 1");
    if (residual && ((reinterpret_cast<uintptr_t>(residual) & 1) || ldr < A->M))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": residual must be 2-byte aligned with ldr >= M");
    usp::ProductCall c = {};
    c.X = Xq;
    c.ldx = ldx;
    c.x_rows = N;
    c.x_scale = x_scale;
    c.quantize = !x_scale;
    c.Y = Y;
    c.ldy = ldy;
    c.N = N;
    c.ep.bias = reinterpret_cast<const uint16_t *>(bias);
    c.ep.res = reinterpret_cast<const uint16_t *>(residual);
    c.ep.ldr = ldr;
    c.ep.act = activation;
    return product_common(f, usp::product_shape(A), A->device, c, workspace, ws_bytes, stream);
}

usp_status usp_group_create(const usp_matrix *const *experts, int64_t E, usp_group **out) {
    const std::string f("usp_group_create");
    if (out) *out = nullptr;
    if (!out || !experts) return usp::fail(USP_ERR_INVALID_ARG, f + ": null pointer");
    if (E < 1 || E > 4096) return usp::fail(USP_ERR_INVALID_ARG, f + ": E must be 1 to 4096");
    usp_group *G = new (std::nothrow) usp_group();
    if (!G) return usp::fail(USP_ERR_OOM, f + ": host allocation failed");
    std::vector<usp::ExpertRef> refs;
    try {
        G->experts.reserve((size_t)E);
        refs.reserve((size_t)E);
        // Held from here on, so that no other thread frees one meanwhile.
        std::lock_guard<std::mutex> lk(g_live_mu);
        const char *why = nullptr;
        for (int64_t i = 0; i < E && !why; ++i) {
            const usp_matrix *A = experts[i], *first = experts[0];
            if (!A || g_live.count(A) == 0)
                why = ": invalid or freed handle among the experts";
            else if (A->M != first->M || A->K != first->K || A->device != first->device ||
                     A->value_bytes != first->value_bytes)
                why = ": experts must have one shape, value type and device";
            else if (A->K > USP_MAX_K_Q)
                why = ": K above USP_MAX_K_Q";
        }
        if (why) {
            delete G;
            return usp::fail(USP_ERR_INVALID_ARG, f + why);
        }
        g_live_groups.insert(G);  // the last step that may fail here
        for (int64_t i = 0; i < E; ++i) {
            usp_matrix *A = const_cast<usp_matrix *>(experts[i]);
            ++A->groups;
            G->experts.push_back(A);
            refs.push_back({reinterpret_cast<const uint8_t *>(A->d_stream), A->d_off, A->d_scale});
            if (A->max_chunks > G->max_chunks) G->max_chunks = A->max_chunks;
        }
        const usp_matrix *A = experts[0];
        G->device = A->device;
        G->E = E;
        G->M = A->M;
        G->K = A->K;
        G->RB = A->RB;
        G->KT = A->KT;
        G->num_cus = A->num_cus;
        G->value_bytes = A->value_bytes;
    } catch (const std::bad_alloc &) {
        delete G;
        return usp::fail(USP_ERR_OOM, f + ": host allocation failed");
    }
    {
        DeviceGuard g(G->device);
        hipError_t e = g.ok ? hipMalloc(&G->d_experts, refs.size() * sizeof(refs[0])) : hipErrorInvalidDevice;
        const bool oom = e == hipErrorOutOfMemory;
        if (e == hipSuccess)
            e = hipMemcpy(G->d_experts, refs.data(), refs.size() * sizeof(refs[0]), hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            (void)usp_group_free(G);
            return usp::fail(oom ? USP_ERR_OOM : USP_ERR_HIP, f + ": " + hipGetErrorString(e));
        }
    }
    *out = G;
    return USP_OK;
}

usp_status usp_group_free(usp_group *G) {
    if (!G) return USP_OK;
    {
        std::lock_guard<std::mutex> lk(g_live_mu);
        if (g_live_groups.erase(G) == 0)
            return usp::fail(USP_ERR_INVALID_ARG, "usp_group_free: invalid or already freed group");
        for (usp_matrix *A : G->experts) --A->groups;
    }
    {
        DeviceGuard g(G->device);
        if (G->d_experts) (void)hipFree(G->d_experts);
    }
    delete G;
    return USP_OK;
}

size_t usp_group_workspace_size(const usp_group *G, int64_t T) {
    if (!alive(G) || T < 1) return 0;
    return usp::product_workspace_bytes(usp::product_shape(G), T);
}

usp_status usp_group_plan(const usp_group *G, int64_t T, char *buf, size_t len) {
    if (!alive(G)) return usp::fail(USP_ERR_INVALID_ARG, "usp_group_plan: invalid or freed group");
    if (T < 1 || !buf || len == 0) return usp::fail(USP_ERR_INVALID_ARG, "usp_group_plan: need T >= 1 and a buffer");
    return copy_text(usp::describe_product(usp::product_shape(G), T), buf, len);
}

usp_status usp_spmm_grouped(const usp_group *G, const void *X, int64_t ldx, int64_t x_rows, const float *x_scale,
                            const int32_t *rows, const int32_t *offsets, int64_t E, void *Y, int64_t ldy, int64_t T,
                            const void *bias, int64_t ldb, const float *row_weight, int activation,
                            void *workspace, size_t ws_bytes, void *stream) {
    const std::string f("usp_spmm_grouped");
    if (!alive(G)) return usp::fail(USP_ERR_INVALID_ARG, f + ": invalid or freed group");
    if (E != G->E) return usp::fail(USP_ERR_INVALID_ARG, f + ": E must be the group's number of experts");
    if (T < 0) return usp::fail(USP_ERR_INVALID_ARG, f + ": T must be >= 0");
    if (T == 0) return USP_OK;
    if (!offsets) return usp::fail(USP_ERR_INVALID_ARG, f + ": null offsets");
    if (x_rows < 1 || (!rows && x_rows < T))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": x_rows must be >= 1, and >= T without rows");
    if ((G->value_bytes == 1) != (x_scale != nullptr))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": x_scale belongs to experts of 8-bit weights, and to no others");
    if (bias && ldb < G->M) return usp::fail(USP_ERR_INVALID_ARG, f + ": ldb must be >= M");
    for (const void *p : {(const void *)rows, (const void *)offsets, (const void *)row_weight})
        if (reinterpret_cast<uintptr_t>(p) & 3)
            return usp::fail(USP_ERR_INVALID_ARG, f + ": rows, offsets and row_weight must be 4-byte aligned");
    usp::ProductCall c = {};
    c.X = X;
    c.ldx = ldx;
    c.x_rows = x_rows;
    c.x_scale = x_scale;
    c.rows = rows;
    c.offsets = offsets;
    c.Y = Y;
    c.ldy = ldy;
    c.N = T;
    c.ep.bias = reinterpret_cast<const uint16_t *>(bias);
    c.ep.act = activation;
    c.ldb = ldb;
    c.weight = row_weight;
    return product_common(f, usp::product_shape(G), G->device, c, workspace, ws_bytes, stream);
}

size_t usp_cache_page_bytes(const usp_cache *cache) {
    if (wrong_cache(cache, false)) return 0;
    usp_cache c = *cache;
    c.data = nullptr;
    c.layers = c.pages = 1;
    return (size_t)usp::cache_view(c, 0).page_bytes;
}

usp_status usp_cache_append(const usp_cache *cache, const usp_cache_rows *rows, int64_t layer, const void *K,
                            int64_t ld_k, int64_t head_k, const void *V, int64_t ld_v, int64_t head_v, void *stream) {
    return cache_rows_common("usp_cache_append", cache, rows, layer, {const_cast<void *>(K), ld_k, head_k},
                             {const_cast<void *>(V), ld_v, head_v}, true, stream);
}

usp_status usp_cache_read(const usp_cache *cache, const usp_cache_rows *rows, int64_t layer, void *K, int64_t ld_k,
                          int64_t head_k, void *V, int64_t ld_v, int64_t head_v, void *stream) {
    return cache_rows_common("usp_cache_read", cache, rows, layer, {K, ld_k, head_k}, {V, ld_v, head_v}, false, stream);
}

usp_status usp_cache_copy(const usp_cache *cache, const int32_t *src, const int32_t *dst, int64_t n, void *stream) {
    const std::string f("usp_cache_copy");
    if (const char *why = wrong_cache(cache, true)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (n < 0 || n > cache->pages) return usp::fail(USP_ERR_INVALID_ARG, f + ": n must be 0 to pages");
    if (n == 0) return USP_OK;
    if (!src || !dst) return usp::fail(USP_ERR_INVALID_ARG, f + ": null pages");
    std::vector<int32_t> from, to;
    try {
        std::vector<int32_t> sorted(dst, dst + n);
        std::sort(sorted.begin(), sorted.end());
        if (sorted.front() < 0 || sorted.back() >= cache->pages)
            return usp::fail(USP_ERR_INVALID_ARG, f + ": a destination is no page of the cache");
        if (std::adjacent_find(sorted.begin(), sorted.end()) != sorted.end())
            return usp::fail(USP_ERR_INVALID_ARG, f + ": a destination is named twice");
        from.reserve((size_t)n);
        to.reserve((size_t)n);
        for (int64_t i = 0; i < n; ++i) {
            if (src[i] < 0 || src[i] >= cache->pages)
                return usp::fail(USP_ERR_INVALID_ARG, f + ": a source is no page of the cache");
            if (src[i] == dst[i]) continue;
            if (std::binary_search(sorted.begin(), sorted.end(), src[i]))
                return usp::fail(USP_ERR_INVALID_ARG, f + ": a page is both a source and a destination");
            from.push_back(src[i]);
            to.push_back(dst[i]);
        }
    } catch (const std::bad_alloc &) {
        return usp::fail(USP_ERR_OOM, f + ": host allocation failed");
    }
    DeviceGuard g(cache->device);
    if (!select_device(cache->device, g)) return usp::fail(USP_ERR_INVALID_ARG, f + ": no such device");
    const int rc = usp::launch_cache_copy(usp::cache_view(*cache, 0), cache->layers, from.data(), to.data(), (int64_t)from.size(), stream);
    if (rc != 0) return hip_fail((hipError_t)rc, (f + ": launch").c_str());
    return USP_OK;
}

// Why heads of q do not go with a cache's; null where they do.
static const char *wrong_heads(const usp_cache &c, int32_t heads) {
    return heads < 1 || heads > 65536 || heads % c.kv_heads ? ": heads must be a multiple of kv_heads up to 65536" : nullptr;
}

size_t usp_attention_workspace_size(const usp_cache *cache, const usp_cache_rows *rows, int32_t heads) {
    if (wrong_cache(cache, false) || wrong_rows(rows, *cache, false) || wrong_heads(*cache, heads) || rows->rows == 0) return 0;
    return usp::attention_workspace_bytes(usp::cache_view(*cache, 0), usp::rows_view(*rows, *cache), heads);
}

usp_status usp_attention_plan(const usp_cache *cache, const usp_cache_rows *rows, int32_t heads, char *buf, size_t len) {
    const std::string f("usp_attention_plan");
    if (const char *why = wrong_cache(cache, false)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (const char *why = wrong_rows(rows, *cache, false)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (const char *why = wrong_heads(*cache, heads)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (rows->rows < 1 || !buf || len == 0) return usp::fail(USP_ERR_INVALID_ARG, f + ": need rows >= 1 and a buffer");
    return copy_text(usp::describe_attention(usp::cache_view(*cache, 0), usp::rows_view(*rows, *cache), heads), buf, len);
}

usp_status usp_attention(const usp_cache *cache, const usp_cache_rows *rows, const usp_attention_args *args,
                         void *workspace, size_t ws_bytes, void *stream) {
    const std::string f("usp_attention");
    if (const char *why = wrong_cache(cache, true)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (const char *why = wrong_rows(rows, *cache, true)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (!args) return usp::fail(USP_ERR_INVALID_ARG, f + ": null arguments");
    const usp_attention_args &p = *args;
    if (const char *why = wrong_heads(*cache, p.heads)) return usp::fail(USP_ERR_INVALID_ARG, f + why);
    if (p.layer < 0 || p.layer >= cache->layers) return usp::fail(USP_ERR_INVALID_ARG, f + ": no such layer");
    if (!(std::fabs(p.scale) <= 0x1p127f)) return usp::fail(USP_ERR_INVALID_ARG, f + ": scale must be finite, of at most 2^127");
    if (!std::isfinite(p.cap) || p.cap < 0.f) return usp::fail(USP_ERR_INVALID_ARG, f + ": cap must be >= 0 and finite");
    if (p.cap > 0.f && !std::isfinite(2.f * p.scale / p.cap * 2.f))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": scale / cap is not finite");
    if (p.window < 0) return usp::fail(USP_ERR_INVALID_ARG, f + ": window must be >= 0");
    if (rows->rows == 0) return USP_OK;
    if (!p.q || !p.out) return usp::fail(USP_ERR_INVALID_ARG, f + ": null q or out");
    if ((reinterpret_cast<uintptr_t>(p.q) | reinterpret_cast<uintptr_t>(p.out)) & 1)
        return usp::fail(USP_ERR_INVALID_ARG, f + ": q and out must be 2-byte aligned");
    for (const void *q : {(const void *)p.first, (const void *)p.last, (const void *)p.slopes})
        if (reinterpret_cast<uintptr_t>(q) & 3)
            return usp::fail(USP_ERR_INVALID_ARG, f + ": first, last and slopes must be 4-byte aligned");
    if (p.ld_q < 0 || p.head_q < 0) return usp::fail(USP_ERR_INVALID_ARG, f + ": strides must be >= 0");
    if (!lie_apart(p.ld_out, p.head_out, rows->rows, p.heads, cache->head_dim))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": rows and heads of out must lie apart");
    const usp::CacheView c = usp::cache_view(*cache, p.layer);
    const usp::RowsView r = usp::rows_view(*rows, *cache);
    if (!usp::attention_fits(c, r, p.heads)) return usp::fail(USP_ERR_UNSUPPORTED, f + ": too many rows and heads");
    const size_t need = usp::attention_workspace_bytes(c, r, p.heads);
    if (need && (!workspace || ws_bytes < need)) return usp::fail(USP_ERR_INVALID_ARG, f + ": workspace too small");
    if (need && (reinterpret_cast<uintptr_t>(workspace) & 15))
        return usp::fail(USP_ERR_INVALID_ARG, f + ": workspace must be 16-byte aligned");
    DeviceGuard g(cache->device);
    if (!select_device(cache->device, g)) return usp::fail(USP_ERR_INVALID_ARG, f + ": no such device");
    const int rc = usp::launch_attention(c, r, p, workspace, stream);
    if (rc != 0) return hip_fail((hipError_t)rc, (f + ": launch").c_str());
    return USP_OK;
}

}  // extern "C"
