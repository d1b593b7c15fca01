/*
 * centrifuge.h -- C ABI of the MI355X (gfx950) token-filtered decoder-layer backward.
 *
 * The library implements the hot path of backward token filtering with
 * activation filtering (paper Sec. 3): the upstream gradient of a layer is
 * row-sparse (filtered tokens carry zero gradient), so every per-token
 * operation runs on the kept rows only ("dimension-reduced dense GEMM",
 * Sec. 3.2), and the attention backward emits dK/dV for kept tokens only
 * while dQ of a kept query still sees every key/value (Sec. 3.1, Eq. 3-4),
 * which keeps the gradient handed to the layer below row-sparse.
 *
 * Conventions (all entry points)
 *   - Every tensor pointer is a DEVICE pointer owned by the caller; the
 *     library never allocates or frees device memory and keeps no state
 *     between calls.  Scratch space is the caller-provided workspace `ws`
 *     (256-byte aligned); its required size comes from the *_workspace_bytes
 *     calls.  Pointers named *_host are HOST pointers.
 *   - Tokens are flat rows t = b*S + s.  Matrices are row-major and dense
 *     (leading dimension = number of columns).  Weights are stored [in, out]
 *     (Y = X * W).  "kept"/compact tensors have one row per kept token in
 *     ascending token order.
 *   - Size limit in CF_BF16 mode: every matrix a call touches ([T,F], [F,H], ...) must stay
 *     below 2 GiB (the GEMM kernels use 32-bit byte offsets); larger requests return
 *     CF_ERR_UNSUPPORTED before anything is launched.
 *   - dtype CF_BF16: bfloat16 storage, fp32 accumulation and fp32 row
 *     statistics; CF_F32: fp32 everywhere (check mode, not tuned).  LSE is
 *     always fp32.  In CF_BF16 mode H, Hq*d, Hkv*d and F must be multiples of
 *     8 and d must be 64 or 128 (another multiple of 8 returns CF_ERR_UNSUPPORTED);
 *     in CF_F32 mode they must be multiples of 4 and d <= 256.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Calls enqueue work and return without synchronising; the one exception
 *     (cf_build_keep_index with a host pointer) says so.
 *   - The number of kept tokens N_k is a DEVICE value after the index build.  Calls
 *     that take `n_kept_dev` + `max_kept` read it there: max_kept is the upper bound
 *     that buffers and launches are sized for, the kernels work on min(N_k, max_kept)
 *     rows, and nothing waits for the host.  Calls that take a plain `n_kept` are for
 *     callers that know the count (a fixed keep ratio, or after reading it back).
 *   - Errors: argument errors are detected on the host before anything is
 *     launched and reported as a cf_status; nothing is written in that case.
 *     A HIP runtime failure is reported as CF_ERR_HIP.
 */
#ifndef CENTRIFUGE_H
#define CENTRIFUGE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    CF_OK = 0,
    CF_ERR_NULL = 1,        /* a required pointer is NULL */
    CF_ERR_SHAPE = 2,       /* a size is non-positive, misaligned or inconsistent */
    CF_ERR_DTYPE = 3,       /* dtype enum out of range */
    CF_ERR_WORKSPACE = 4,   /* workspace missing, misaligned or too small */
    CF_ERR_UNSUPPORTED = 5, /* valid request this build does not implement */
    CF_ERR_HIP = 6          /* HIP runtime error */
} cf_status;

typedef enum { CF_BF16 = 0, CF_F32 = 1 } cf_dtype;

typedef void* cf_stream;

/* Shape of one decoder layer (RMSNorm -> GQA causal attention -> residual ->
 * RMSNorm -> SwiGLU FFN -> residual) and of the batch. */
typedef struct {
    int32_t B, S;          /* sequences, tokens per sequence; T = B*S            */
    int32_t H;             /* hidden size                                        */
    int32_t Hq, Hkv, d;    /* query heads, key/value heads (Hq % Hkv == 0), head dim */
    int32_t F;             /* SwiGLU width                                       */
    int32_t dtype;         /* cf_dtype                                           */
    float rms_eps;         /* RMSNorm epsilon                                    */
    float softmax_scale;   /* 0 => 1/sqrt(d)                                     */
} cf_layer_desc;

/* Activations saved by the forward pass, full length (T rows). */
typedef struct {
    const void* x;         /* [T,H]     layer input                              */
    const void* q;         /* [T,Hq*d]  queries as used by attention             */
    const void* k;         /* [T,Hkv*d] keys                                     */
    const void* v;         /* [T,Hkv*d] values                                   */
    const void* attn_out;  /* [T,Hq*d]  attention output before the O projection */
    const float* lse;      /* [B,Hq,S]  log-sum-exp of the scaled causal scores  */
    const void* r;         /* [T,H]     x + attn_out*Wo (input of the 2nd norm)  */
    const void* gate;      /* [T,F]     rmsnorm2(r)*Wg                           */
    const void* up;        /* [T,F]     rmsnorm2(r)*Wu                           */
    /* Rotary position embedding of q and k (optional; both NULL = none).  The paper does not
     * mention it; the evaluated model families use it.  Tables [S, d/2] fp32 for position s and
     * frequency i; the forward rotated each head of the projected q and k as
     *   out[i] = x[i]*cos - x[i+d/2]*sin,  out[i+d/2] = x[i+d/2]*cos + x[i]*sin   (i < d/2),
     * q and k above are the rotated tensors, and the layer calls apply the transposed rotation
     * to dq and dk, at the ORIGINAL position of each kept row, before the projections' backward. */
    const float* rope_cos;
    const float* rope_sin;
} cf_saved;

typedef struct {
    const void *wq, *wk, *wv;  /* [H,Hq*d], [H,Hkv*d], [H,Hkv*d] */
    const void *wo;            /* [Hq*d,H] */
    const void *wg, *wu;       /* [H,F]    */
    const void *wd;            /* [F,H]    */
    const void *g1, *g2;       /* [H] RMSNorm gains */
} cf_weights;

/* Outputs.  Parameter gradients have the shapes of the parameters.  dx is [N_k,H]
 * compact for the filtered call and [T,H] for the dense call, always overwritten.
 *   main_grad == 0: parameter gradients in the storage dtype, overwritten.
 *   main_grad == 1: the nine parameter-gradient tensors are fp32 buffers (whatever the
 *     storage dtype) and the call ADDS this batch's gradient to them, without rounding
 *     the fp32 accumulators to the storage dtype first: gradient accumulation over
 *     micro-batches in a master-precision buffer.  With no kept token nothing is added. */
typedef struct {
    void *dwq, *dwk, *dwv, *dwo, *dwg, *dwu, *dwd, *dg1, *dg2;
    void *dx;
    int32_t main_grad;
} cf_grads;

const char* cf_status_str(cf_status s);

/* Library version string (static storage). */
const char* cf_version(void);

/* ---- A1: keep-index build (Sec. 3.2: shrink the sequence dimension) --------
 * Order-preserving compaction of the keep mask (Sec. 2.1 Eq. 2: 1 = token is
 * selected; any non-zero byte counts as kept).
 *   mask        [B*S] bytes, device
 *   idx         [>= number kept] int32, device: flat row of the j-th kept token, ascending
 *   cu_kept     [B+1] int32, device: kept tokens in sequences before b; cu_kept[B] = N_k
 *   n_kept_dev  [1] int32, device (nullable)
 *   n_kept_host [1] int32, host (nullable).  When non-NULL the call copies N_k
 *               back and synchronises the stream before returning.
 *   ws          device scratch of cf_index_workspace_bytes(B*S) bytes
 * idx must have room for B*S entries unless the caller knows N_k in advance. */
size_t cf_index_workspace_bytes(int64_t n_tokens);
cf_status cf_build_keep_index(const uint8_t* mask, int32_t B, int32_t S,
                              int32_t* idx, int32_t* cu_kept, int32_t* n_kept_dev,
                              int32_t* n_kept_host, void* ws, size_t ws_bytes, cf_stream stream);

/* Masks of up to this many tokens are indexed in one launch that touches neither a workspace nor the library's own array. */
#define CF_INDEX_NO_SCRATCH_TOKENS 32768

/* The keep-index build for callers that cannot allocate device memory or carry a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc).  Same
 * arguments and results as cf_build_keep_index without the workspace and without the host copy:
 * what the first of two launches leaves for the second (a count per 8192 tokens and a bit per token) lives in a device array
 * built into the library (2.1 MB per GPU, held until the process ends), nothing is allocated, freed or copied to the host and the stream is not
 * synchronised.  At most 2^24 tokens (B*S); more returns CF_ERR_UNSUPPORTED before any launch.
 * All calls on one GPU of more than CF_INDEX_NO_SCRATCH_TOKENS tokens share that array: such calls that overlap on one GPU (two streams, two host
 * threads) race and must be serialised by the caller.  Shorter masks are indexed in one launch that does not touch it. */
cf_status cf_build_keep_index_static(const uint8_t* mask, int32_t B, int32_t S,
                                     int32_t* idx, int32_t* cu_kept, int32_t* n_kept_dev,
                                     cf_stream stream);

/* ---- A2: row gather (Sec. 3.2: remove the filtered rows of saved tensors) --
 * dst[j,:] = src[idx[j],:] for j < min(N_k, max_kept), N_k = *n_kept_dev (device; NULL: exactly
 * max_kept rows).  src is [src_rows, cols], dst has room for max_kept rows; cols*sizeof(elt) must be
 * a multiple of 4.  idx entries must lie in [0, src_rows) (not checked: they live on the device). */
cf_status cf_gather_rows(const void* src, int64_t src_rows, int64_t cols, int32_t dtype,
                         const int32_t* idx, const int32_t* n_kept_dev, int32_t max_kept, void* dst,
                         cf_stream stream);

/* ---- A3: dimension-reduced linear backward (Sec. 3.2, the two GEMM types) ---
 * For Y = X*W with W [in,out]:
 *   dx_kept [n_kept,in]  = dy_kept [n_kept,out] * W^T          (nullable: skipped)
 *   dw      [in,out]     = dw_beta*dw + x_kept^T [in,n_kept] * dy_kept   (nullable: skipped)
 * x_kept is [n_kept,in].  dw_beta is 0 (overwrite) or 1 (accumulate).  With dw_beta 0, dw may be w's own memory
 * (W is read for dx_kept first); no other output may overlap an input.
 * n_kept == 0 is valid: dw is zeroed (beta 0) or left alone (beta 1). */
cf_status cf_linear_bwd_reduced(const void* x_kept, const void* dy_kept, const void* w,
                                int32_t n_kept, int32_t in, int32_t out, int32_t dtype,
                                void* dx_kept, void* dw, float dw_beta, cf_stream stream);
/* The same with scratch (ws: 256-byte aligned, overlapping no other argument, or NULL) that lets a product of few output
 * tiles and a long contraction be cut into parts, which idle compute units work on, and summed up.  The size is 0 where
 * nothing would be cut (and for invalid sizes); a ws that is smaller is CF_ERR_WORKSPACE. */
size_t cf_linear_workspace_bytes(int32_t n_kept, int32_t in, int32_t out, int32_t dtype);
cf_status cf_linear_bwd_reduced_ws(const void* x_kept, const void* dy_kept, const void* w,
                                   int32_t n_kept, int32_t in, int32_t out, int32_t dtype,
                                   void* dx_kept, void* dw, float dw_beta, void* ws, size_t ws_bytes, cf_stream stream);

/* ---- A5: filtered attention backward (Sec. 3.1, Eq. 3 and Eq. 4) -----------
 * Kept queries attend to ALL keys/values at positions <= their own (causal on
 * original positions) for dQ; dK and dV are produced for kept tokens only.
 *   q_kept, o_kept, do_kept  [n_kept,Hq*d]   compact rows (o = attention output, do = its gradient)
 *   k_full, v_full           [T,Hkv*d]       full length
 *   lse_full                 [B,Hq,S] fp32   forward's log-sum-exp over the full causal row
 *   idx [n_kept], cu_kept [B+1]              from cf_build_keep_index
 *   dq_kept [n_kept,Hq*d], dk_kept, dv_kept [n_kept,Hkv*d]   outputs, overwritten
 * dk/dv are summed over the Hq/Hkv query heads that share a key/value head.
 * Uses only B,S,Hq,Hkv,d,dtype,softmax_scale of desc.
 * cf_attn_workspace_bytes grows with n_kept and is the same for every B and S: a workspace sized for the largest
 * n_kept serves all batch shapes of a model. */
size_t cf_attn_workspace_bytes(const cf_layer_desc* desc, int32_t n_kept);
cf_status cf_attn_bwd_filtered(const cf_layer_desc* desc, const void* q_kept, const void* k_full,
                               const void* v_full, const void* o_kept, const float* lse_full,
                               const void* do_kept, const int32_t* idx, const int32_t* cu_kept,
                               int32_t n_kept, void* dq_kept, void* dk_kept, void* dv_kept,
                               void* ws, size_t ws_bytes, cf_stream stream);

/* ---- whole layer -----------------------------------------------------------
 * cf_layer_bwd_filtered: mask -> keep index -> all reduced GEMMs, row-local backward ops (SwiGLU,
 * RMSNorm, residuals; Sec. 3.2 "G (.) g") and the filtered attention backward.  No tensor is gathered
 * by a kernel of its own: the kept rows of dy_full, gate, up, r, x are read through the index by the
 * kernels that consume them, and those of attn_out and q are copied by the attention backward's
 * row-statistics pass.  dy_full is the upstream gradient on all T rows (rows of filtered tokens are
 * ignored).  Outputs: grads->dx compact [N_k,H] (the row-sparse gradient for the layer below), all
 * parameter gradients; idx_out [T] / cu_kept_out [B+1] / n_kept_dev_out [1] (device, each nullable)
 * receive the keep index and N_k; n_kept_host (HOST, nullable; page-locked memory keeps the copy
 * asynchronous) receives N_k through a copy queued behind the call's kernels: read it after
 * synchronising with the stream.
 * The call itself never synchronises: every kernel reads N_k on the device.
 *   max_kept: upper bound of N_k that the workspace and grads->dx are sized for; 0 or a value above
 *   T means T, which is always sufficient.  A caller that knows its keep ratio saves workspace.  If
 *   the mask keeps more than max_kept tokens the call processes the first max_kept kept tokens only
 *   and the result is not the layer's gradient: compare the N_k read back with max_kept.
 * cf_layer_bwd_dense: the same kernels with every token kept and no index; dx is [T,H].
 *   When a dense call writes dx, the only saved tensor that is still read is x: dx may lie over another one that has room
 *   for it (also in cf_layer_bwd_lora without a mask).
 * cf_layer_bwd_compact: a layer BELOW the one whose call built the keep index
 * (Sec. 3.2: once the first gradient is reduced, every later gradient is; Sec. 3.1:
 * the sparsity is handed on to all front layers).  dy_kept [n_kept,H] is the compact
 * dx of the layer above; idx [n_kept] and cu_kept [B+1] (device) are the index that
 * call returned and n_kept its N_k.  Saved activations are still full length.
 * Outputs as for the filtered call.  Nothing is copied to the host and the stream is
 * not synchronised.
 * cf_layer_bwd_compact_dev: the same for a caller that has not read N_k back: n_kept_dev is the
 * device count the filtered call returned and max_kept the bound it was given, so a whole stack of
 * layers runs without a single synchronisation.
 * ws must hold cf_layer_workspace_bytes(desc, max_kept) bytes (compact call: max_kept >= n_kept).  One workspace sized
 * for the largest B, S and max_kept serves all smaller ones too; in bf16 16.8 MB of it (64 KB per compute unit) are for products in
 * parts, which a call of few kept tokens may come to whatever the shape. */
size_t cf_layer_workspace_bytes(const cf_layer_desc* desc, int32_t max_kept);
cf_status cf_layer_bwd_filtered(const cf_layer_desc* desc, const cf_saved* saved,
                                const cf_weights* w, const void* dy_full, const uint8_t* mask,
                                int32_t max_kept, cf_grads* grads, int32_t* idx_out,
                                int32_t* cu_kept_out, int32_t* n_kept_dev_out, int32_t* n_kept_host,
                                void* ws, size_t ws_bytes, cf_stream stream);
cf_status cf_layer_bwd_compact(const cf_layer_desc* desc, const cf_saved* saved,
                               const cf_weights* w, const void* dy_kept, const int32_t* idx,
                               const int32_t* cu_kept, int32_t n_kept, cf_grads* grads,
                               void* ws, size_t ws_bytes, cf_stream stream);
cf_status cf_layer_bwd_compact_dev(const cf_layer_desc* desc, const cf_saved* saved,
                                   const cf_weights* w, const void* dy_kept, const int32_t* idx,
                                   const int32_t* cu_kept, const int32_t* n_kept_dev, int32_t max_kept,
                                   cf_grads* grads, void* ws, size_t ws_bytes, cf_stream stream);
cf_status cf_layer_bwd_dense(const cf_layer_desc* desc, const cf_saved* saved,
                             const cf_weights* w, const void* dy_full, cf_grads* grads,
                             void* ws, size_t ws_bytes, cf_stream stream);

/* ---- low-rank adapters (Sec. 5.3: LoRA, rank 64, on the q, k, v and o projections) --------
 * The adapted projection is Y = X*W + scale * (X*a)*b with a [in, rank], b [rank, out]; the base
 * weights and the RMSNorm gains are frozen, so the call produces no gradient for them: every
 * linear layer only hands its input gradient on (reduced GEMM dX), and the adapters get
 *   da = scale * X_kept^T * (dY_kept * b^T),   db = scale * (X_kept * a)^T * dY_kept,
 * with dX_kept = dY_kept*W^T + scale * (dY_kept*b^T)*a^T.  Saved q, k, v, attn_out, r are the
 * tensors of the adapted forward.  rank must be a multiple of 8 (CF_BF16) or 4 (CF_F32). */
typedef struct {
    const void *aq, *bq;   /* [H,rank],    [rank,Hq*d]  */
    const void *ak, *bk;   /* [H,rank],    [rank,Hkv*d] */
    const void *av, *bv;   /* [H,rank],    [rank,Hkv*d] */
    const void *ao, *bo;   /* [Hq*d,rank], [rank,H]     */
    int32_t rank;
    float scale;           /* usually lora_alpha / rank */
} cf_lora;

/* Adapter gradients have the shapes of the adapters and are overwritten; dx is compact
 * [N_k,H] (or [T,H] when every token is kept because mask is NULL). */
typedef struct {
    void *daq, *dbq, *dak, *dbk, *dav, *dbv, *dao, *dbo;
    void *dx;
} cf_lora_grads;

/* cf_layer_bwd_lora: the filtered layer backward of a LoRA-adapted layer.  Arguments as for
 * cf_layer_bwd_filtered (max_kept, idx_out, cu_kept_out, n_kept_dev_out, n_kept_host included): the kept
 * count stays on the device, every kernel reads it there (the grouped launches of the rank-r products plan
 * their tiles and parts from it), and the call never synchronises.  mask == NULL means "every token kept" (no index, no gather: the dense
 * LoRA backward of the same library; *n_kept_host, when given, is set to T at once).
 * ws must hold cf_lora_workspace_bytes(desc, rank, max_kept) bytes (max_kept 0 or above T means T). */
size_t cf_lora_workspace_bytes(const cf_layer_desc* desc, int32_t rank, int32_t max_kept);
cf_status cf_layer_bwd_lora(const cf_layer_desc* desc, const cf_saved* saved, const cf_weights* w,
                            const cf_lora* lora, const void* dy_full, const uint8_t* mask, int32_t max_kept,
                            cf_lora_grads* grads, int32_t* idx_out, int32_t* cu_kept_out,
                            int32_t* n_kept_dev_out, int32_t* n_kept_host, void* ws, size_t ws_bytes,
                            cf_stream stream);

/* ---- query/key norm with rotary embedding (model families that normalise the heads) --------
 * Every head of the projected queries and keys is normalised by its own root mean square, scaled by a gain that all heads of
 * its kind share and, where tables are given, rotated at its token's position, all in one pass:
 *   n = x * rstd,  rstd = (mean(x^2) + rms_eps)^(-1/2),  y = R(pos) (n * g)
 * with the rotation R of cf_saved (half-split pairs).  Arithmetic is fp32; y is rounded once.
 *   Uses only S, Hq, Hkv, d, dtype and rms_eps of desc (Hq % Hkv == 0 is not asked for).  d is a power of two, 16 to 256
 *   in CF_BF16 and 8 to 256 in CF_F32; another multiple of 8 in CF_BF16 is CF_ERR_UNSUPPORTED.
 *   Row t of the full-length tensors has position positions[t], or t mod S without positions; a position outside [0, S),
 *   the rows of the tables, is taken for the nearest one inside.  n_rows and rows read through idx are at most 2^30. */
typedef struct {
    void *q, *k;                   /* rows of [Hq*d] and [Hkv*d] elements, 16-byte aligned          */
    int64_t q_stride, k_stride;    /* elements from row to row, 0 = dense; multiples of 16 bytes    */
} cf_qk;

typedef struct {
    const void *gq, *gk;           /* [d] gains of the queries' and the keys' norm                  */
    const float *rope_cos, *rope_sin;   /* [S, d/2] fp32; both NULL = no rotation                   */
    const int32_t* positions;      /* nullable                                                      */
} cf_qk_norm;

/* out = norm and rotation of in, n_rows rows of each.  out may be in itself (same pointers and strides); no other overlap. */
cf_status cf_qk_norm_rope_fwd(const cf_layer_desc* desc, const cf_qk_norm* p, const cf_qk* in, int32_t n_rows,
                              const cf_qk* out, cf_stream stream);

/* The backward pass on kept rows.  in: the tensors before the norm, full length, read through idx (NULL: row j is row j); dy,
 * dx: compact, one row per kept token; dx may be dy itself (same pointers and strides), without idx in itself too, no other overlap.  n_kept_dev and max_kept as for
 * cf_gather_rows.  dgq, dgk [d] (both or neither NULL: frozen gains): gain gradients, overwritten in the storage dtype, or
 * (main_grad 1) fp32 buffers that the call adds to; zero rows give zero gradients.  The sums' order depends on the sizes alone.
 * ws is needed for the gain gradients only. */
size_t cf_qk_norm_workspace_bytes(const cf_layer_desc* desc, int32_t max_kept);
cf_status cf_qk_norm_rope_bwd(const cf_layer_desc* desc, const cf_qk_norm* p, const cf_qk* in, const cf_qk* dy_kept,
                              const int32_t* idx, const int32_t* n_kept_dev, int32_t max_kept, const cf_qk* dx_kept,
                              void* dgq, void* dgk, int32_t main_grad, void* ws, size_t ws_bytes, cf_stream stream);

/* The layer calls for models with that norm: saved->q and saved->k are, as always, what attention used (after norm and rotation),
 * qk has the projections' outputs ahead of them and the gains.  dq and dk go back through the rotation and the norm at each kept
 * row, in place, before the projections' backward.  dgq, dgk [d]: in the storage dtype, overwritten, or with grads->main_grad fp32 and
 * added to; both NULL: frozen gains (always so in the adapter call, whose dgq and dgk have to be NULL).  Everything else as for the calls of the same name without
 * _qk (the compact call: cf_layer_bwd_compact_dev with n_kept_dev, and cf_layer_bwd_compact of max_kept rows with NULL), the workspace too, but for its
 * size: cf_layer_qk_workspace_bytes / cf_lora_qk_workspace_bytes. */
typedef struct {
    const void *q_pre, *k_pre;     /* [T,Hq*d], [T,Hkv*d] projected queries and keys                */
    const void *gq, *gk;           /* [d] gains                                                     */
    float eps;                     /* of this norm                                                  */
    void *dgq, *dgk;
} cf_layer_qk;

size_t cf_layer_qk_workspace_bytes(const cf_layer_desc* desc, int32_t max_kept);
size_t cf_lora_qk_workspace_bytes(const cf_layer_desc* desc, int32_t rank, int32_t max_kept);
cf_status cf_layer_bwd_filtered_qk(const cf_layer_desc* desc, const cf_saved* saved, const cf_weights* w, const cf_layer_qk* qk,
                                   const void* dy_full, const uint8_t* mask, int32_t max_kept, cf_grads* grads,
                                   int32_t* idx_out, int32_t* cu_kept_out, int32_t* n_kept_dev_out, int32_t* n_kept_host,
                                   void* ws, size_t ws_bytes, cf_stream stream);
cf_status cf_layer_bwd_compact_qk(const cf_layer_desc* desc, const cf_saved* saved, const cf_weights* w, const cf_layer_qk* qk,
                                  const void* dy_kept, const int32_t* idx, const int32_t* cu_kept, const int32_t* n_kept_dev,
                                  int32_t max_kept, cf_grads* grads, void* ws, size_t ws_bytes, cf_stream stream);
cf_status cf_layer_bwd_dense_qk(const cf_layer_desc* desc, const cf_saved* saved, const cf_weights* w, const cf_layer_qk* qk,
                                const void* dy_full, cf_grads* grads, void* ws, size_t ws_bytes, cf_stream stream);
cf_status cf_layer_bwd_lora_qk(const cf_layer_desc* desc, const cf_saved* saved, const cf_weights* w, const cf_layer_qk* qk,
                               const cf_lora* lora, const void* dy_full, const uint8_t* mask, int32_t max_kept,
                               cf_lora_grads* grads, int32_t* idx_out, int32_t* cu_kept_out, int32_t* n_kept_dev_out,
                               int32_t* n_kept_host, void* ws, size_t ws_bytes, cf_stream stream);

/* ---- losses of kept tokens with their gradient towards the logits --------------------------
 * What stands ahead of the layers: the gradient is [N_k,V], the compact upstream gradient of the head's reduced linear backward.
 * With s = logit_scale, l a kept token's logits and y its target, lp = s*l_y - log(sum_c exp(s*l_c)) and
 *   CF_LOSS_NLL     L = -lp                                   (Sec. 2.1 Eq. 1 with norm = 0: the mean over kept tokens)
 *   CF_LOSS_POLICY  L = -min(r*A, clip(r, 1-clip_lo, 1+clip_hi)*A) + kl_coef*k,  r = exp(lp - old_logp),
 *                   k = exp(ref_logp - lp) - (ref_logp - lp) - 1   (ref_logp NULL: k = 0)
 *   loss = sum_j w_j*L_j / norm,   dlogits[j,c] = w_j/norm * dL/dlp * s * ([c == y] - exp(s*l_c - logsumexp)),
 * with dL/dlp of the first term 0 where the clipped product is the smaller one and -r*A elsewhere.  r*A is 0 where A is, and a KL term with kl_coef 0 is in
 * stats alone, also where r or k is beyond fp32.  norm 0 stands for the number of live rows.  A row whose target lies outside [0,V) or whose weight is 0 is left out whatever it holds (infinities
 * and NaN included): its logp and its gradient are 0; it counts in the number of live rows.  A logit of -inf has probability 0.
 *   logits   [rows,V], row stride logits_stride elements (0 = V); kept row j is row idx[j] (NULL: row j).  Any alignment of rows:
 *            pointers need their element's only, multiples of 16 bytes are faster
 *   targets, old_logp, ref_logp, advantages, weights   one per row of logits, read at the same idx[j].  weights NULL: 1
 *   dlogits  [max_kept,V], row stride dlogits_stride (nullable: not wanted).  May be logits itself (same stride) without idx,
 *            and must not overlap them otherwise
 *   logp     [max_kept] fp32 (nullable): lp.  For the same logits it has the same bits with and without dlogits, so that old_logp
 *            from a call without gradient makes r exactly 1
 *   stats    [4] fp32 (nullable): loss, its first term, the mean k, the share of clipped tokens (all weighted by w/norm)
 * At least one of dlogits, logp, stats is wanted.  n_kept_dev and max_kept as for cf_gather_rows; rows behind the live ones are
 * left as they were.  ws: cf_token_loss_workspace_bytes(max_kept), 16-byte aligned. */
typedef enum { CF_LOSS_NLL = 0, CF_LOSS_POLICY = 1 } cf_loss_kind;

typedef struct {
    int32_t kind;                  /* cf_loss_kind                              */
    int32_t V;                     /* vocabulary, at most 2^30                  */
    int32_t dtype;                 /* cf_dtype of logits and dlogits            */
    float logit_scale;             /* 0 => 1 (one over a sampling temperature); times log2(e) it has to be finite */
    float clip_lo, clip_hi;        /* policy: 0 <= clip_lo <= 1, clip_hi >= 0   */
    float kl_coef;                 /* policy; 0 without ref_logp                */
    float norm;                    /* 0 => the number of live rows              */
} cf_loss_desc;

size_t cf_token_loss_workspace_bytes(int32_t max_kept);
cf_status cf_token_loss(const cf_loss_desc* desc, const void* logits, int64_t logits_stride, const int64_t* targets,
                        const float* old_logp, const float* ref_logp, const float* advantages, const float* weights,
                        const int32_t* idx, const int32_t* n_kept_dev, int32_t max_kept, void* dlogits,
                        int64_t dlogits_stride, float* logp, float* stats, void* ws, size_t ws_bytes, cf_stream stream);

/* ---- the ends of the stack of layers --------------------------------------------------------
 * Token embeddings, the norm of rows and the loss straight from the head's input: what a training step does below the lowest layer and above the
 * highest one.  n_kept_dev and max_kept as for cf_gather_rows; idx may be NULL (row j is row j); rows behind the live ones are left as they were.  H is
 * a multiple of 8 in CF_BF16 and of 4 in CF_F32; tensors of elements are dense and 16-byte aligned; workspaces 256-byte aligned.
 *
 * cf_embed_fwd: out[t,:] = scale * table[tokens[t],:], table [V,H], out [n,H]; 0 for a token outside [0,V).  out must not overlap table.
 * cf_embed_bwd: dtable[c,:] = scale * sum of the rows j of dx_kept [max_kept,H] with tokens[idx[j]] == c, fp32 sums in an
 *   order that tokens, idx and max_kept fix (no atomics).  main_grad 0: all of dtable [V,H] is written in the storage dtype, zeros where no row has the token.  main_grad 1:
 *   dtable is fp32 and is added to; rows without a token are not touched.  dx rows whose token lies outside [0,V) count for nothing, whatever they hold. */
cf_status cf_embed_fwd(const void* table, int32_t V, int32_t H, int32_t dtype, const int64_t* tokens, int64_t n, float scale, void* out,
                       cf_stream stream);
size_t cf_embed_bwd_workspace_bytes(int32_t H, int32_t max_kept);
cf_status cf_embed_bwd(const int64_t* tokens, const void* dx_kept, int32_t V, int32_t H, int32_t dtype, const int32_t* idx,
                       const int32_t* n_kept_dev, int32_t max_kept, float scale, void* dtable, int32_t main_grad, void* ws, size_t ws_bytes,
                       cf_stream stream);

/* cf_norm_fwd: y[j,:] = n * g + b of row idx[j] of x, n = (x - mu) * rstd, rstd = (mean((x - mu)^2) + eps)^(-1/2); mu is the row's mean (layer 1) or 0
 *   (layer 0: root mean square norm).  b (layer 1 only, nullable): biases.  y [max_kept,H] may be x itself without idx; no other overlap.
 *   (Overlaps are refused as far as extents are known; which rows of x an index names is not, beyond the first: y, and dx and the gradients below, have to lie elsewhere.)
 * cf_norm_bwd: with u = dy * g,  dx = rstd * (u - [layer 1] mean(u) - n * mean(u * n)),  dg = sum over rows of dy * n,  db = sum of dy (layer 1).
 *   The statistics are made again from x.  dx_kept [max_kept,H] may be dy_kept itself, without idx x itself; no other overlap.  dg, db [H] (nullable; db
 *   with dg only): in the storage dtype, overwritten, or (main_grad 1) fp32 and added to.  The sums' order depends on the sizes alone.  ws is needed for dg and db only.
 * H at most 32768 in CF_BF16 and 16384 in CF_F32 (CF_ERR_UNSUPPORTED above). */
typedef struct {
    int32_t H, dtype, layer;
    float eps;
} cf_norm_desc;

cf_status cf_norm_fwd(const cf_norm_desc* desc, const void* x, const void* g, const void* b, const int32_t* idx, const int32_t* n_kept_dev,
                      int32_t max_kept, void* y, cf_stream stream);
size_t cf_norm_bwd_workspace_bytes(const cf_norm_desc* desc, int32_t max_kept);
cf_status cf_norm_bwd(const cf_norm_desc* desc, const void* x, const void* g, const void* dy_kept, const int32_t* idx, const int32_t* n_kept_dev,
                      int32_t max_kept, void* dx_kept, void* dg, void* db, int32_t main_grad, void* ws, size_t ws_bytes, cf_stream stream);

/* cf_head_loss: the losses of cf_token_loss (same description, per-row inputs, terms and rules for rows that are left out) for the logits
 * l = x_kept * table^T, x_kept [max_kept,H] compact, table [V,H] as for the embeddings, and their gradients towards both operands:
 *   dx_kept = dlogits * table [max_kept,H] (nullable; may be x_kept itself),  dtable = dlogits^T * x_kept [V,H] (nullable; main_grad as for cf_embed_bwd,
 *   so that a tied table's two gradients share one buffer).
 * The logits are fp32 values that are never stored.  What is kept of them for the gradients is bounded by the workspace: exponentials, in the storage
 * dtype, of as many columns as it has room for; those of the others are computed again, piece by piece.  A larger workspace is faster; logp and stats do not
 * depend on it, gradients by the order of fp32 sums.  For the same rows and max_kept logp has the same bits with and without
 * gradients.  max_kept at most 2^22, in CF_BF16 with a gradient 2^22 - 65; in CF_BF16 x_kept stays below 2 GiB; the table may be larger.
 * In CF_BF16 the exponentials and the rows of x_kept times their row's factor are operands of matrix products and rounded to bf16 once each: dtable is off by up to
 * four roundings of 2^-8 a term, dx by three.  In CF_F32 products take their operands in three bf16 parts (2^-26 a product): magnitudes above 3.39e38 count as
 * infinite, and an infinite operand of a row that counts may give NaN where a sum of fp32 products is infinite.
 *   cf_head_loss_workspace_bytes: what to provide for a call with (need_dx, need_dtable): as much as is of use, at most `limit`, or the least that will do
 *   where that is more.  0 for sizes that are refused. */
size_t cf_head_loss_workspace_bytes(const cf_loss_desc* desc, int32_t H, int32_t max_kept, int32_t need_dx, int32_t need_dtable, size_t limit);
cf_status cf_head_loss(const cf_loss_desc* desc, int32_t H, const void* x_kept, const void* table, const int64_t* targets, const float* old_logp,
                       const float* ref_logp, const float* advantages, const float* weights, const int32_t* idx, const int32_t* n_kept_dev,
                       int32_t max_kept, void* dx_kept, void* dtable, int32_t main_grad, float* logp, float* stats, void* ws, size_t ws_bytes,
                       cf_stream stream);

/* ---- AdamW over many tensors ---------------------------------------------------------------
 * What takes cf_grads (and cf_lora_grads): one launch per 40 tensors of any sizes (or per 2^31 elements),
 *   g' = grad_scale * g * min(1, max_norm / (norm + 1e-6))
 *   m = beta1*m + (1-beta1)*g',  v = beta2*v + (1-beta2)*g'^2
 *   p = p - lr*weight_decay*p - lr * (m / (1-beta1^step)) / (sqrt(v / (1-beta2^step)) + eps)
 * in fp32; with 32-bit states a sqrt(v) that fp32 has no normal square of counts as a value between itself and 2^-63, 2^-64 at least.  norm_dev (device, nullable: no clipping) is what cf_grad_norm left; where it is not finite the call changes nothing.
 * step_dev, lr_dev (device, nullable) replace step and lr, for a call captured into a graph.
 *   p        CF_F32 parameters, or CF_BF16 ones with (master) or without an fp32 master copy; p is the rounded master
 *   m, v     state_bits 32: fp32.  state_bits 8: e4m3 bytes that stand for m / m_scale and sqrt(v) / v_scale, with a scale for every
 *            256 elements (ceil(n/256) of them): the block's largest absolute value / 448.  sqrt(v) is rounded up with the
 *            probability of what is cut off, by 20 bits of a hash of (seed, step, tensor's number in the call, element): to nearest, an average over
 *            1/(1-beta2) steps would stand still, since a step changes it by less than half a step of 8 bits; and never
 *            to 0 unless it is 0, which a later division by eps would blow up.  m is rounded to nearest, but in the same way (by 12 other bits of the hash, to
 *            0 too) where |g'| is at most 3/8 of |m| and |m| falls by less than half a step: an m whose gradient has ended would stand still beside
 *            a root that goes on falling.  An element whose new v is beyond fp32 keeps its moments (its update is 0, and NaN for an infinite g', as
 *            with 32 bits); NaN counts for no scale.  A finite value far above its block's others takes their resolution.
 * All pointers 16-byte aligned (scales: 4); no overlap.  The tensors array is read on the host during the call. */
typedef struct {
    void* p;
    float* master;                 /* CF_BF16 parameters: NULL or the fp32 master copy; CF_F32: NULL */
    const void* g;
    void *m, *v;
    float *m_scale, *v_scale;      /* state_bits 8                              */
    int64_t n;                     /* elements, 0 to 2^34                       */
    float weight_decay;
} cf_adamw_tensor;

typedef struct {
    double lr, beta1, beta2, eps;  /* eps >= 2^-126: its reciprocal is finite */
    int32_t step;                  /* 1 for the first                           */
    int32_t p_dtype, g_dtype;      /* cf_dtype of all parameters, of all gradients */
    int32_t state_bits;            /* 32 or 8                                   */
    uint32_t seed;                 /* state_bits 8                              */
    float grad_scale;
    float max_norm;                /* > 0 where norm_dev is given               */
    const float* norm_dev;
    const int32_t* step_dev;
    const float* lr_dev;
} cf_adamw_desc;

cf_status cf_adamw_step(const cf_adamw_desc* desc, const cf_adamw_tensor* tensors, int32_t n_tensors, cf_stream stream);

/* norm (device, [1] fp32) = |grad_scale| * sqrt(sum of the squares of all tensors' elements), summed in fp64 in a fixed order.  grads: host array
 * of n_tensors 16-byte aligned device pointers, sizes: their elements. */
size_t cf_grad_norm_workspace_bytes(int32_t n_tensors);
cf_status cf_grad_norm(const void* const* grads, const int64_t* sizes, int32_t n_tensors, int32_t g_dtype, float grad_scale,
                       float* norm, void* ws, size_t ws_bytes, cf_stream stream);

/* ---- measurement probes (for the rooflines of Sec. 3.2's GEMMs and of the gather / row-local
 * kernels; not part of the method) ------------------------------------------------------------
 * cf_probe_mfma_bf16: n_blocks blocks of four waves; every wave runs `iters` passes over an 8 x 8
 *   grid of 16x16x32 bf16 MFMA accumulators (the GEMM kernels' wave tile) with all operands in
 *   registers and pseudo-random non-zero operand values: no LDS, no global traffic.  sink: device,
 *   n_blocks*256 floats, overwritten (keeps the work alive).  *flops_out (host, nullable) receives
 *   the flop count of the launch.  Timing it gives the matrix cores' sustained rate on this chip
 *   under its power limit: the measured ceiling that the GEMM kernels are compared with.
 * cf_probe_mfma_lds_bf16: the same loop with LDS fragment reads mixed in at the GEMM kernels' ratio
 *   and nothing waiting for them inside the loop: reads = 0 none, 1 = 16 16-byte reads per 64 MFMAs
 *   (the NT kernel's), 2 = 32 transposing 8-byte reads per 64 MFMAs (the TN kernel's).  Same arguments
 *   and flop count as cf_probe_mfma_bf16; reads outside 0..2 -> CF_ERR_SHAPE.  Shows what the reads
 *   alone cost next to the MFMAs (issue slots, power), apart from the operand stream that feeds them.
 * cf_probe_copy: dst[0..bytes) = src[0..bytes) (device pointers, 16-byte aligned, bytes % 16 == 0,
 *   no overlap): a plain streaming copy, the measured HBM ceiling (bytes read + bytes written per
 *   second) for the bandwidth-bound kernels, and the reference that scales profiler byte counters. */
cf_status cf_probe_mfma_bf16(int32_t n_blocks, int32_t iters, float* sink, double* flops_out,
                             cf_stream stream);
cf_status cf_probe_mfma_lds_bf16(int32_t n_blocks, int32_t iters, int32_t reads, float* sink,
                                 double* flops_out, cf_stream stream);
cf_status cf_probe_copy(const void* src, void* dst, size_t bytes, cf_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* CENTRIFUGE_H */
