/*
 * usp.h -- C ABI of the unstructured-sparse fp16 SpMM library (libusp.so).
 *
 * The library computes Y = W X for a weight matrix W (M x K, fp16) pruned to
 * moderate unstructured sparsity and a skinny dense input X (K x N, fp16, N the
 * number of tokens of a decode step), with fp32 accumulation and fp16 output.
 * This is the sparse matrix multiplication of Section 5.1 of the paper
 * (weight M x K sparse, input K x N dense, output M x N dense), the operation its
 * storage format (Section 3) and kernel (Section 4) exist to accelerate.
 *
 * W is first converted once, on the host, into a compressed device-resident
 * format (the one-time conversion of Section 5.3, "Storage Format Conversion");
 * every product then streams that format from HBM and decodes it on chip.
 *
 * Layout conventions (all strides in elements):
 *   W     row-major M x K: row m at W + m*ldw (the nn.Linear weight layout)
 *   mask  row-major M x K bytes: row m at mask + m*ldm; nonzero = kept
 *   X     token-major: column n of the logical K x N matrix at X + n*ldx,
 *         i.e. a contiguous [N, K] activation when ldx == K
 *   Y     token-major: column n of the logical M x N matrix at Y + n*ldy
 *
 * Errors: every entry point returns a usp_status; no exception crosses the
 * ABI. usp_last_error() returns a message for the calling thread's most recent
 * failure. Kernel faults surface at the caller's next synchronisation.
 * Thread safety: a handle is immutable after usp_encode; concurrent usp_spmm
 * calls on one handle are safe when each uses its own workspace.
 */
#ifndef USP_H
#define USP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct usp_matrix usp_matrix; /* opaque; owns the device memory of one encoded W */

typedef enum {
    USP_OK = 0,
    USP_ERR_INVALID_ARG = 1, /* null pointer, bad size or stride, freed handle */
    USP_ERR_UNSUPPORTED = 2, /* valid request this build does not serve (alignment, N range) */
    USP_ERR_OOM = 3,         /* host or device allocation failed */
    USP_ERR_HIP = 4,         /* a HIP runtime call failed (message has the HIP error) */
    USP_ERR_INTERNAL = 5
} usp_status;

/* Format version written by usp_encode and reported by usp_info. */
#define USP_FORMAT_VERSION 2
/* The same for usp_encode_q: records of 8-bit values. */
#define USP_FORMAT_VERSION_Q 3

/*
 * usp_encode -- one-time conversion of W and its keep-mask into the compressed
 * device format (Section 3.2 defines the paper's own format; ours is described
 * with the library). Blocking.
 *   W     host pointer, M x K fp16 bit patterns, row stride ldw >= K
 *   mask  host pointer, M x K bytes, row stride ldm >= K; nonzero = keep
 *   M, K  >= 1, M <= 2^20 (USP_ERR_UNSUPPORTED above: the workspace keeps one
 *         arrival counter per 16 rows in a fixed 256 KB region)
 *   device  HIP device ordinal that will hold the encoding
 *   out   receives the new handle; set to NULL on any error
 * Kept values are stored as opaque 16-bit words (signed zeros, subnormals,
 * NaN payloads and kept exact zeros survive bit for bit); values where the
 * mask is zero are ignored. The caller keeps ownership of W and mask.
 */
usp_status usp_encode(const uint16_t *W, int64_t ldw, const uint8_t *mask, int64_t ldm,
                      int64_t M, int64_t K, int device, usp_matrix **out);

/*
 * usp_workspace_size -- bytes of device workspace usp_spmm (of an 8-bit handle:
 * usp_spmm_q) needs for this handle and this N (0 when none). Returns 0 for a NULL
 * handle. The workspace of usp_spmm holds the split rows' arrival counters and fp32 partials and,
 * where the shared-decode or the wide kernel serves the call (33 to 256 tokens
 * on large layers, 320 and more on all), a copy of X rearranged into the order
 * its products read it (512 KT bytes per token, KT = ceil(K / 256), of at most
 * 2048 tokens), rewritten by every such call. It does not grow evenly with N: the
 * wide kernel's partials take up to 128 MiB where the rows and tokens leave it few
 * whole tiles (5120 x 5120: 33 MiB at 320 tokens, 70 at 1024, 15 at 1536; 28672 x
 * 8192: 8 MiB at 512, 144 at 1024).
 */
size_t usp_workspace_size(const usp_matrix *A, int64_t N);

/*
 * usp_spmm -- Y = W X on the handle's device, enqueued on `stream`
 * (a hipStream_t; NULL = the default stream). Asynchronous: returns after the
 * launch. Y is overwritten (no accumulation into it).
 *   X   device pointer, fp16, token-major with stride ldx >= K
 *   Y   device pointer, fp16, token-major with stride ldy >= M; must not alias X
 *   N   number of tokens, 1 <= N
 *   workspace  device pointer, 16-byte aligned, to >= usp_workspace_size(A, N)
 *       bytes (may be NULL when that size is 0); owned by the caller; must not be
 *       used by another in-flight call. It must be zero-filled before its first
 *       use; every completed call leaves it ready for the next one (with any
 *       handle and any N), so it is cleared once, not per call. From 320 tokens a
 *       smaller one is accepted too if it holds the smallest part the product can
 *       be cut into (a few MiB: 1.8 for 5120 x 5120 and 2.3 for 28672 x 8192 at
 *       1024 tokens): the call then runs in as many parts as it takes, slower, with
 *       the same bits.
 * Accumulation is fp32 in a fixed order: results are bitwise reproducible run
 * to run. The output is rounded to fp16 with round-to-nearest-even.
 * Inputs with X not 16-byte aligned, or ldx or K not a multiple of 8, are
 * read at their alignment while staged, packed or padded; some take a slower
 * kernel. No allocation and no synchronisation happens inside, and
 * the call only enqueues kernels on `stream` (no memory-set or copy operations),
 * so it may be captured into a HIP graph and the graph replayed; each replay
 * leaves the workspace ready for the next, as each call does.
 */
usp_status usp_spmm(const usp_matrix *A, const void *X, int64_t ldx, void *Y, int64_t ldy,
                    int64_t N, void *workspace, size_t ws_bytes, void *stream);

/* Activation of usp_spmm_ex, applied after the bias. */
typedef enum {
    USP_ACT_NONE = 0,
    USP_ACT_RELU = 1,      /* max(v, 0); of a NaN: 0 in usp_spmm_ex, NaN in usp_spmm_q and usp_spmm_grouped */
    USP_ACT_GELU_TANH = 2, /* 0.5 v (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))) */
    USP_ACT_SILU = 3       /* v / (1 + exp(-v)) */
} usp_activation;

/*
 * usp_spmm_ex -- usp_spmm with a linear layer's epilogue fused into the output
 * store: Y = act(W X + bias) + residual. The decode-step linear layers the
 * paper's sparse product replaces (Section 2.1; its models' projections carry a
 * bias, the FFN an activation, the block a residual add) need nothing else.
 * Per output, in fp32: the sum, + bias, the activation, + residual, then the
 * one rounding to fp16 (round to nearest even).
 *   bias       device fp16 [M] (2-byte aligned), or NULL for none
 *   residual   device fp16, logical M x N, column n at residual + n * ldr with
 *              ldr >= M (2-byte aligned), or NULL for none. It may be Y itself
 *              with ldr == ldy (an in-place add: each output reads its residual
 *              before it is written, by the same thread); otherwise it must not
 *              overlap Y.
 *   activation a usp_activation
 * Everything else -- arguments, workspace, asynchrony, reproducibility -- as
 * usp_spmm; usp_spmm(...) equals usp_spmm_ex(..., NULL, NULL, 0, USP_ACT_NONE, ...).
 * An activation outside usp_activation is USP_ERR_INVALID_ARG.
 */
usp_status usp_spmm_ex(const usp_matrix *A, const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t N,
                       const void *bias, const void *residual, int64_t ldr, int activation,
                       void *workspace, size_t ws_bytes, void *stream);

/* Bytes of the device scratch usp_spmm_noalloc uses on each GPU (32 MiB). */
#define USP_NOALLOC_SCRATCH_BYTES (32u << 20)

/*
 * usp_spmm_noalloc -- for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc. The same product as usp_spmm (same kernels, same bits), with no
 * workspace argument: its workspace is a USP_NOALLOC_SCRATCH_BYTES device array
 * the library holds on each GPU until the process ends (looked up and cleared
 * once per device inside usp_encode, so the handle's device is set up by the
 * time any product runs). This call allocates nothing and calls no allocating
 * routine. From 320 tokens a product whose workspace exceeds the scratch runs in
 * parts that fit it.
 *   A, X, ldx, Y, ldy, N, stream   as usp_spmm
 * Every call on a GPU shares that GPU's scratch, which keeps the last call's
 * contents; each completed call leaves its arrival counters at zero, as the
 * next call needs them. Calls that overlap in time on one GPU (other streams,
 * other host threads) race on the scratch and give wrong results: serialize
 * them. Returns USP_ERR_UNSUPPORTED, enqueueing nothing, when the product needs
 * more workspace than the scratch holds: up to 319 tokens usp_workspace_size(A, N)
 * > USP_NOALLOC_SCRATCH_BYTES; every configured layer up to 64 tokens fits.
 */
usp_status usp_spmm_noalloc(const usp_matrix *A, const void *X, int64_t ldx, void *Y, int64_t ldy,
                            int64_t N, void *stream);

/*
 * usp_plan -- which kernel usp_spmm (usp_spmm_q, of an 8-bit handle) runs for this
 * handle and N when X is 16-byte aligned with ldx = K (of an 8-bit handle: 8-bit tokens;
 * fp16 tokens, which a kernel brings to 8 bits first, may take another), as a short text ("row W=8",
 * "chunk S=5 W=8 nb=1 grid=200", "dma nb=4 tg=1 grid=1024", "fourwave passes=1 nt=2
 * grid=768", "wide passes=1 nb=2 grid=216"; of 8-bit handles and groups "product R=4
 * W=4 nb=1 grid=448", "wide-product R=4 nb=4 grid=216"), written to
 * buf (at most len bytes with the terminating NUL, truncated if longer). For
 * tests and tuning; enqueues nothing. USP_ERR_INVALID_ARG for a NULL handle,
 * N < 1, or no buffer.
 */
usp_status usp_plan(const usp_matrix *A, int64_t N, char *buf, size_t len);

/*
 * usp_densify -- writes W with the mask applied (pruned entries as +0) into a
 * dense row-major M x K fp16 device buffer Wd with row stride ldw >= K, by the
 * same on-chip decode the product uses; 8-bit values times their row's scale,
 * rounded to fp16. Asynchronous on `stream`. For checks.
 */
usp_status usp_densify(const usp_matrix *A, void *Wd, int64_t ldw, void *stream);

/*
 * usp_decode -- host-side inverse of usp_encode: copies the encoding back and
 * rebuilds W (masked entries as 0x0000) and the mask (0/1) into the caller's
 * host buffers of M x K entries each (contiguous rows). Blocking.
 */
usp_status usp_decode(const usp_matrix *A, uint16_t *W_out, uint8_t *mask_out);

typedef struct {
    int64_t M, K;           /* logical shape */
    int64_t nnz;            /* kept entries */
    size_t device_bytes;    /* bytes of the encoding the product streams from HBM */
    size_t table_bytes;     /* bytes of the per-tile offset table (also streamed) */
    int32_t format_version; /* USP_FORMAT_VERSION, or USP_FORMAT_VERSION_Q for 8-bit weights */
    int32_t tile_rows, tile_k; /* tile geometry of the encoding */
    int32_t device;
} usp_info_t;

/* usp_info -- shape, size and geometry of an encoding. */
usp_status usp_info(const usp_matrix *A, usp_info_t *info);

/* ---- 8-bit weights and tokens ------------------------------------------------
 *
 * W = diag(w_scale) Wq and X = Xq diag(x_scale): 8-bit integers with one fp32 scale
 * per output channel and one per token. The products are summed exactly in 32-bit
 * integers; the scales, the bias, the activation and the residual are applied in
 * fp32, then the one rounding to fp16. A handle of 8-bit weights is used with
 * usp_spmm_q, usp_densify, usp_decode_q, usp_info, usp_plan, usp_workspace_size,
 * usp_group_create and usp_free; usp_spmm and its variants and usp_decode refuse
 * it, as usp_spmm_q refuses a handle of fp16 weights (USP_ERR_INVALID_ARG).
 */

/* Most columns of an 8-bit weight (its integer sums stay below 2^31) and of the
 * experts of a group. */
#define USP_MAX_K_Q 129024

/*
 * usp_encode_q -- usp_encode for 8-bit weights.
 *   W      host pointer, M x K int8 (the whole range, -128 included), row stride ldw >= K
 *   scale  host pointer, M fp32 scales, one per row (finite)
 *   K      <= USP_MAX_K_Q
 * Everything else as usp_encode.
 */
usp_status usp_encode_q(const int8_t *W, int64_t ldw, const uint8_t *mask, int64_t ldm, const float *scale,
                        int64_t M, int64_t K, int device, usp_matrix **out);

/* usp_decode_q -- host-side inverse of usp_encode_q: M x K int8, M x K mask bytes, M scales. Blocking. */
usp_status usp_decode_q(const usp_matrix *A, int8_t *W_out, uint8_t *mask_out, float *scale_out);

/*
 * usp_quantize -- tokens in 8 bits: per token n, a = max_k |X[n, k]|, x_scale[n] = a / 127
 * and Xq[n, k] = X[n, k] * (127 / a) rounded to the nearest integer, ties to even (all in
 * fp32; a = 0 gives zeros and scale 0). A token that holds a NaN or an infinity gets zeros
 * and the scale NaN, so its products are NaN, whatever the activation.
 *   X        device pointer, fp16, token n at X + n * ldx, ldx >= K
 *   Xq       device pointer, int8, token n at Xq + n * ldq, ldq >= K
 *   x_scale  device pointer, fp32 [N]
 *   N, K     >= 1 (N up to 2^20, K up to 2^28)
 *   device   the HIP device of the pointers and of `stream`
 * Asynchronous on `stream`; no allocation, capturable.
 */
usp_status usp_quantize(const void *X, int64_t ldx, int64_t N, int64_t K, void *Xq, int64_t ldq, float *x_scale,
                        int device, void *stream);

/*
 * usp_spmm_q -- Y = act(W X + bias) + residual with 8-bit W and X, on the handle's device.
 *   Xq       device pointer, int8, token n at Xq + n * ldx, ldx >= K
 *   x_scale  device pointer, fp32 [N], 4-byte aligned; or NULL: Xq then points to fp16
 *            tokens, which are brought to 8 bits first, as usp_quantize does
 *   workspace  16-byte aligned, to >= usp_workspace_size(A, N) bytes (may be NULL when that is
 *       0); must not be used by another in-flight call. It needs no clearing, and the region that
 *       usp_spmm expects cleared is left alone, so that one workspace can serve both.
 * X is packed for the products first where many tokens or its alignment ask for it. N up to 2^20, and
 * ceil(M / 16) ceil(N / 16) below 2^31. Everything else -- Y, bias, residual, activation, asynchrony,
 * capture, reproducibility -- as usp_spmm_ex.
 */
usp_status usp_spmm_q(const usp_matrix *A, const void *Xq, int64_t ldx, const float *x_scale, void *Y, int64_t ldy,
                      int64_t N, const void *bias, const void *residual, int64_t ldr, int activation,
                      void *workspace, size_t ws_bytes, void *stream);

/* ---- Products grouped by expert ---------------------------------------------- */

typedef struct usp_group usp_group; /* opaque; a list of encoded experts */

/*
 * usp_group_create -- a group of E experts: handles of the same shape and value type (all
 * fp16 or all 8-bit) on one device, K <= USP_MAX_K_Q. An expert may occur more than once and
 * in several groups. The handles stay the caller's; while a group holds one, usp_free refuses
 * it. Blocking. 1 <= E <= 4096.
 */
usp_status usp_group_create(const usp_matrix *const *experts, int64_t E, usp_group **out);

/* usp_group_free -- releases the group (not its experts). NULL is accepted. The caller
 * guarantees that no product on it is still in flight. */
usp_status usp_group_free(usp_group *G);

/* usp_group_workspace_size -- bytes of device workspace usp_spmm_grouped needs for T rows (0 when none, or for no
 * valid group or T). */
size_t usp_group_workspace_size(const usp_group *G, int64_t T);

/* usp_group_plan -- which kernel usp_spmm_grouped runs for T >= 1 rows when X is dword-aligned, as usp_plan. */
usp_status usp_group_plan(const usp_group *G, int64_t T, char *buf, size_t len);

/*
 * usp_spmm_grouped -- for each expert e and each row t of its range offsets[e] <= t < offsets[e + 1]:
 *     Y[t] = row_weight[t] * act(W_e X[rows[t]] + bias[e])
 *   X        device pointer, x_rows rows with stride ldx >= K: fp16, or int8 for experts of
 *            8-bit weights
 *   x_scale  device fp32 [x_rows], the scales of the 8-bit rows (NULL for fp16 experts)
 *   rows     device int32 [T], the row of X that row t multiplies (a row may occur several
 *            times, as for tokens that go to several experts), or NULL: row t itself, and then
 *            x_rows >= T. An index outside [0, x_rows) stands for a row of zeros.
 *   E        the group's number of experts (any other is refused)
 *   offsets  device int32 [E + 1], not decreasing, within [0, T]. They are read on the device, so
 *            the call needs no host knowledge of the counts and may be captured; values outside
 *            [0, T] count as the nearer end and a decreasing value as the one before it. Rows of Y
 *            that no expert has are left as they were.
 *   Y        device fp16, row t at Y + t * ldy, ldy >= M; must not overlap X
 *   bias     device fp16, expert e's at bias + e * ldb (ldb >= M), or NULL
 *   row_weight  device fp32 [T], the router's weights, or NULL for ones
 *   activation  a usp_activation
 *   T        0 <= T <= 2^20 (0: nothing is done)
 *   workspace  as usp_spmm_q, of usp_group_workspace_size(G, T) bytes
 * Accumulation and rounding as in usp_spmm (fp16 experts) and usp_spmm_q; an offset or a row index
 * never makes the call read or write outside the operands.
 */
usp_status usp_spmm_grouped(const usp_group *G, const void *X, int64_t ldx, int64_t x_rows, const float *x_scale,
                            const int32_t *rows, const int32_t *offsets, int64_t E, void *Y, int64_t ldy, int64_t T,
                            const void *bias, int64_t ldb, const float *row_weight, int activation,
                            void *workspace, size_t ws_bytes, void *stream);

/* ---- Norms around a block ------------------------------------------------------ */

typedef enum {
    USP_NORM_NONE = 0,
    USP_NORM_RMS = 1,  /* v / sqrt(mean(v^2) + eps) * weight + bias */
    USP_NORM_LAYER = 2 /* (v - mean(v)) / sqrt(var(v) + eps) * weight + bias */
} usp_norm_kind;

typedef enum {
    USP_GATE_NONE = 0, /* g */
    USP_GATE_SIGMOID = 1,
    USP_GATE_TANH = 2,
    USP_GATE_SILU = 3
} usp_gate_activation;

/*
 * One token's update, all in fp32:
 *     r = residual + scale * gate_act(gate) * post(y)        (y NULL: r = residual)
 *     h = pre(r)
 * residual_out takes r and out takes h, each rounded to fp16 once (h is computed from r before
 * its rounding); out_q and out_scale take the fp16 h in 8 bits, as usp_quantize(h) does. Pointers
 * are device pointers; strides count elements.
 */
typedef struct {
    const void *residual;      /* fp16 [N, K], stride ld_residual */
    const void *y;             /* fp16 [N, K], stride ld_y: the block's output; or NULL */
    const void *gate;          /* fp16 [N, K] with stride ld_gate, or [K] with ld_gate = 0; or NULL: 1 */
    const void *post_weight;   /* fp16 [K], or NULL: 1 */
    const void *post_bias;     /* fp16 [K], or NULL: 0 */
    const void *pre_weight;
    const void *pre_bias;
    void *residual_out;        /* fp16, stride ld_residual_out; may be residual or y; or NULL */
    void *out;                 /* fp16, stride ld_out; may be y; or NULL */
    void *out_q;               /* int8, stride ld_out_q; or NULL */
    float *out_scale;          /* fp32 [N]; needed with out_q */
    int64_t ld_residual, ld_y, ld_gate, ld_residual_out, ld_out, ld_out_q;
    float scale;               /* residual scale */
    float eps;                 /* >= 0 */
    int post_kind, pre_kind;   /* usp_norm_kind; post_kind needs y */
    int gate_activation;       /* usp_gate_activation */
} usp_norm_args;

/*
 * usp_norm -- the update above for 1 to 2^20 tokens of 1 to 2^28 channels. At least one output. An output
 * that is an input has its stride and base; other overlaps are not allowed. A gate needs y.
 * Asynchronous on `stream` (of `device`); no allocation, capturable, bitwise reproducible.
 */
usp_status usp_norm(const usp_norm_args *args, int64_t N, int64_t K, int device, void *stream);

/* ---- Attention over a paged cache ------------------------------------------------
 *
 * A cache holds the keys and values of tokens that a decoder's layers have seen, in pages that
 * sequences own in any order. Its memory is the caller's: `layers` pools of `pages` pages of
 * usp_cache_page_bytes bytes each, page p of layer l at data + (l * pages + p) * page bytes. A page
 * holds page_tokens tokens of every head, in the order the matrix products read them:
 *
 *   page    kv_heads x (page_tokens / 32) blocks, a head's blocks one after the other
 *   block   32 tokens of one head: keys, then values, then for 8-bit values 32 fp32 scales of the
 *           keys and 32 of the values. W = head_dim rounded up to 32, 64, 96, 128, 192 or 256.
 *   keys    W / 8 x 32 x 8: channel d of token j at ((d / 8) * 32 + place(j)) * 8 + d % 8, place(j)
 *           being j with its bits 2 and 3 exchanged; channels from head_dim on are zeros
 *   values  4 x W x 8: channel d of token j at ((j / 8) * W + d) * 8 + j % 8; channels from head_dim on
 *           are not defined
 *
 * 8-bit keys and values are what usp_quantize makes of a head's fp16 channels: codes, and one scale a
 * token. A pool need not be cleared: nothing is read of tokens that were never written.
 */
typedef struct {
    void *data;          /* device pointer, 16-byte aligned */
    int64_t layers;      /* >= 1 */
    int64_t pages;       /* of a layer, 1 to 2^31 - 1 */
    int32_t kv_heads;    /* 1 to 4096 */
    int32_t head_dim;    /* a multiple of 8, 8 to 256 */
    int32_t page_tokens; /* a multiple of 32, 32 to 4096 */
    int32_t value_bytes; /* 2: fp16; 1: 8 bits */
    int32_t device;      /* the HIP device of every pointer of a call, and of its stream */
} usp_cache;

/* usp_cache_page_bytes -- bytes of a page of one layer (0 for a NULL or invalid description; data, pages and layers are
 * not looked at). */
size_t usp_cache_page_bytes(const usp_cache *cache);

/*
 * The rows of a step: new tokens of some sequences, sequence after sequence. Sequence s has
 * lengths[s] tokens in the cache, those of the step included, and the rows offsets[s] <= t <
 * offsets[s + 1]: row t is its token lengths[s] - offsets[s + 1] + t. Token j of it lies in page
 * table[s * ld_table + j / page_tokens]. All are read on the device, so a captured call takes what they
 * hold when it is replayed, and none makes a call read or write outside its operands: lengths count as at
 * most table_pages * page_tokens and at least 0, offsets as within [0, rows] (where they decrease, which rows are
 * computed is not defined), a token before the sequence's start is not there, and neither is one in a page outside
 * [0, pages).
 */
typedef struct {
    const int32_t *table;    /* device int32, sequences rows of table_pages entries with stride ld_table */
    int64_t ld_table;        /* >= table_pages */
    int64_t table_pages;     /* >= 1; table_pages * page_tokens below 2^31 - 4096 */
    const int32_t *lengths;  /* device int32 [sequences] */
    const int32_t *offsets;  /* device int32 [sequences + 1]; or NULL: row s is sequence s's only one */
    int64_t sequences;       /* 1 to 2^20; without offsets: rows */
    int64_t rows;            /* T, 0 to 2^20 (0: nothing is done); more than one launch takes, which begins at 2^24 rows
                                times heads, is USP_ERR_UNSUPPORTED */
} usp_cache_rows;

/*
 * usp_cache_append -- writes the step's keys and values into their pages of one layer (fp16 ones in 8 bits first, as
 * usp_quantize does for each head, where the cache holds 8-bit values).
 *   K, V        device fp16: channel d of head h of row t at t * ld + h * head_stride + d
 *   ld, heads   strides in elements, >= 0 (rows and heads may overlap)
 * Two rows of a step for one place of one page (a page that two sequences of the step have) leave one of them or a
 * mixture. Asynchronous on `stream`; no allocation, capturable.
 */
usp_status usp_cache_append(const usp_cache *cache, const usp_cache_rows *rows, int64_t layer, const void *K,
                            int64_t ld_k, int64_t head_k, const void *V, int64_t ld_v, int64_t head_v, void *stream);

/*
 * usp_cache_read -- the reverse: the step's keys and values (8-bit ones as code * scale, rounded to fp16) from their
 * pages into K and V, laid out as above with strides that keep rows and heads apart (heads at least head_dim, rows at
 * least one head, either one inside the other). Rows that are not there are left as they were.
 */
usp_status usp_cache_read(const usp_cache *cache, const usp_cache_rows *rows, int64_t layer, void *K, int64_t ld_k,
                          int64_t head_k, void *V, int64_t ld_v, int64_t head_v, void *stream);

/*
 * usp_cache_copy -- copies page src[i] to page dst[i] in every layer, for i < n: for forks whose last page the next token
 * changes, and to move pages together. src and dst are HOST pointers, read before the call returns (a captured call
 * keeps what they held). Pages outside [0, pages), a destination named twice, and a page that is a source of one pair and
 * the destination of another are USP_ERR_INVALID_ARG, and nothing is done; a pair of equal pages is left out.
 * Asynchronous on `stream`; no device allocation, capturable. 0 <= n <= pages.
 */
usp_status usp_cache_copy(const usp_cache *cache, const int32_t *src, const int32_t *dst, int64_t n, void *stream);

/*
 * Attention of each row over the tokens of its sequence. Row t, the token p of its sequence s, sees the tokens
 *     max(first[t], p - window + 1, 0) <= k < min(last[t], lengths[s])
 * where a missing `first` is 0, a missing `last` is p + 1 (causal) and window 0 is none. Packed documents: first[t] =
 * the start of t's document. A prefix that all rows see: last[t] = max(p + 1, prefix). Head h of q reads head
 * h / (heads / kv_heads) of the cache:
 *     x[k] = scale * q . K[k];   x[k] <- cap * tanh(x[k] / cap)  (cap > 0);   x[k] <- x[k] - slopes[h] * |p - k|
 *     out  = sum_k exp(x[k]) V[k] / sum_k exp(x[k]),   zeros for a row that sees nothing
 * in fp32, with one rounding to fp16 at the end. For the product with V the weights exp(x - max) are taken to 22 bits and
 * to 2^-37 of the largest where a step has few rows (the rows kernel of usp_attention_plan). In prompts (its tiles kernel)
 * they are rounded to fp16, in the sum below the line too: relative 2^-11 each down to 2^-27 of the largest, and to 2^-38
 * of it below that (2^-14 and 2^-25 where q and the biases allow scores beyond 2^25), and 2^-14 more over 8-bit caches, whose
 * values below 2^-14 are rounded to multiples of 2^-24 there. What a row does not see has no influence on it, NaN and
 * infinities included. A row that sees a NaN, or a score of +infinity, is NaN; one whose scores are all -infinity is zeros.
 * Infinities in q and K, and scores beyond fp32's range (log2(e) times them, so from 2.3e38 on), count as what they are
 * there; an infinite value as what it is under a weight of at least 2^-36 of the largest (2^-24 where scores may pass 2^25).
 */
typedef struct {
    const void *q;          /* device fp16: channel d of head h of row t at q + t * ld_q + h * head_q + d */
    void *out;              /* device fp16, laid out by ld_out and head_out; must not overlap q or the cache */
    const int32_t *first;   /* device int32 [rows], or NULL */
    const int32_t *last;    /* device int32 [rows], or NULL */
    const float *slopes;    /* device fp32 [heads], or NULL */
    int64_t ld_q, head_q;   /* strides in elements, >= 0 */
    int64_t ld_out, head_out; /* as usp_cache_read's */
    int64_t layer;
    int64_t window;         /* >= 0 */
    int32_t heads;          /* a multiple of kv_heads, up to 65536 */
    float scale;            /* finite, |scale| at most 2^127 */
    float cap;              /* >= 0, finite; 0: none */
} usp_attention_args;

/* usp_attention_workspace_size -- bytes of device workspace usp_attention needs for such a step (sequences, rows,
 * table_pages and whether there are offsets are looked at; no pointer is read); 0 when none, or for an invalid
 * description. */
size_t usp_attention_workspace_size(const usp_cache *cache, const usp_cache_rows *rows, int32_t heads);

/* usp_attention_plan -- which kernel usp_attention runs for such a step, as usp_plan. */
usp_status usp_attention_plan(const usp_cache *cache, const usp_cache_rows *rows, int32_t heads, char *buf, size_t len);

/*
 * usp_attention -- the attention above, of the rows' own tokens too once usp_cache_append has written them (on the same
 * stream, or waited for). Rows that no sequence has are left as they were.
 *   workspace  as usp_spmm's: 16-byte aligned, zero-filled before its first use, left ready for the next call of any
 *              operator; not used by another call in flight
 * The kernel is chosen by the number of rows for each sequence, so a step that mixes single tokens with
 * prompts is faster as two calls. Asynchronous on `stream`; no allocation, capturable; the same bits for the same
 * operands (which other sequences a step has, and whether a row near it has a q that allows scores beyond 2^25, may move a
 * result by roundings of its fp32 sums).
 */
usp_status usp_attention(const usp_cache *cache, const usp_cache_rows *rows, const usp_attention_args *args,
                         void *workspace, size_t ws_bytes, void *stream);

/* usp_free -- releases the handle and its device memory. NULL is accepted. A handle that a
 * group holds is refused (USP_ERR_INVALID_ARG).
 * The caller guarantees no product or usp_densify on it is still in flight.
 * Handles are looked up among the live ones before use, never dereferenced
 * blindly: passing a freed handle (or any pointer usp_encode did not return)
 * to any entry point gives USP_ERR_INVALID_ARG, unless a later usp_encode
 * happened to return the same address. */
usp_status usp_free(usp_matrix *A);

/* usp_last_error -- message of the calling thread's most recent failure ("" if none). */
const char *usp_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* USP_H */
