/*
 * dit_block.h -- C ABI of the MI355X (gfx950) DiT block library.
 *
 * One DiT transformer block forward on one GPU's share of a request or of a
 * packed batch of requests: the denoising stage that the GF-DiT paper names as
 * dominating execution time (section 1, Introduction), where each step computes
 * bidirectionally over the entire latent sequence (section 2.1, Rescheduling
 * Boundaries), for the Wan2.2 video and Qwen-Image workloads of its evaluation
 * (section 6.1, Experimental Setup).  The paper does not define the block; it
 * is the adaLN-Zero DiT block with QK-RMSNorm, sectioned 3D rotary embeddings,
 * full self-attention, cross-attention to text and a GELU-tanh MLP.  A
 * denoising-step executor takes a task over its artifacts -- latent state,
 * conditioning and text embeddings (section 3.1, Reschedulable Trajectory
 * Tasks) -- which is the argument set of dit_block_forward.
 *
 * Conventions shared by every entry point:
 *  - Every pointer not marked "host" is device memory on the current HIP
 *    device.  The caller owns all memory; the library allocates and frees
 *    nothing and keeps no mutable global state, so calls are thread-safe
 *    (the one exception, dit_timestep_modulation_noalloc, says so).
 *  - Tensors are row-major.  Activations are token-major [rows, width];
 *    Linear weights are [out, in] (every GEMM is A . W^T); vectors are dense.
 *  - dtype DIT_BF16: activations, weights, norm gains and biases are bfloat16;
 *    accumulation, norm statistics, softmax and the modulation vectors are
 *    fp32.  dtype DIT_F32: everything is fp32.
 *  - Every call is asynchronous on `stream` and never synchronises.  Arguments
 *    are validated on the host before anything is launched; a failed check
 *    returns DIT_ERR_INVALID_ARG or DIT_ERR_UNSUPPORTED and launches nothing.
 *    A failed launch returns DIT_ERR_HIP.  Faults inside kernels surface at the
 *    caller's next synchronisation.  dit_last_error() gives a thread-local
 *    message for the last failure.  The library never aborts or exits.
 *  - Packed batches: request r owns rows cu_seqlens[r]..cu_seqlens[r+1] (host
 *    arrays, non-decreasing, starting at 0).  Rows never interact across
 *    requests.  At most DIT_MAX_REQ requests per call.
 *  - Device pointers must be 16-byte aligned, and row strides must keep every
 *    row 16-byte aligned.
 */
#ifndef DIT_BLOCK_H
#define DIT_BLOCK_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DIT_MAX_REQ 64
#define DIT_ABI_VERSION 4

typedef enum {
  DIT_OK = 0,
  DIT_ERR_INVALID_ARG = -1, /* a null pointer, a bad size, stride or table */
  DIT_ERR_UNSUPPORTED = -2, /* valid, but a shape this build has no kernel for */
  DIT_ERR_WORKSPACE = -3,   /* workspace smaller than dit_block_workspace_size */
  DIT_ERR_HIP = -4          /* a HIP launch or runtime call failed */
} dit_status;

typedef enum { DIT_F32 = 0, DIT_BF16 = 1 } dit_dtype;

/* Epilogues of dit_linear, applied to z = A . W^T + bias per element. */
typedef enum {
  DIT_EPI_NONE = 0,           /* out = z */
  DIT_EPI_GELU_TANH = 1,      /* out = 0.5 z (1 + tanh(sqrt(2/pi)(z + 0.044715 z^3))) */
  DIT_EPI_RESIDUAL = 2,       /* out = res + z */
  DIT_EPI_GATED_RESIDUAL = 3  /* out = res + gate[req(row)] * z (per-request fp32 gate) */
} dit_epilogue;

/* Hyper-parameters of one block.  hidden = n_heads * head_dim. */
typedef struct {
  int hidden;           /* D */
  int n_heads;          /* H */
  int head_dim;         /* d: 128 for bf16; 64 or 128 for fp32 */
  int mlp_hidden;       /* Dff */
  int freq_dim;         /* F: width of the sinusoidal timestep encoding (even) */
  int rope_sections[3]; /* (d_t, d_h, d_w): even, sum == head_dim; {0,0,0} = no rotary */
  float rope_theta;     /* rotary base, 10000 */
  int qk_norm;          /* 1: per-head RMSNorm on q, k (self) and cq, ck (cross) */
  float ln_eps;         /* LayerNorm epsilon (biased variance), 1e-6 */
  float rms_eps;        /* RMSNorm epsilon, 1e-6 */
  dit_dtype dtype;
} dit_block_config;

/* Device pointers to the block's parameters ([out, in] weights, dtype of the
 * config).  Shapes: w_t1 [D,F] b_t1 [D] w_t2 [D,D] b_t2 [D] w_ada [6D,D]
 * b_ada [6D] w_qkv [3D,D] b_qkv [3D] g_q,g_k [d] w_o [D,D] b_o [D] g_ca,b_ca [D]
 * w_cq [D,D] b_cq [D] w_ckv [2D,D] b_ckv [2D] g_cq,g_ck [d] w_co [D,D] b_co [D]
 * w_up [Dff,D] b_up [Dff] w_dn [D,Dff] b_dn [D].  The gains may be NULL when
 * qk_norm == 0. */
typedef struct {
  const void *w_t1, *b_t1, *w_t2, *b_t2, *w_ada, *b_ada;
  const void *w_qkv, *b_qkv, *g_q, *g_k, *w_o, *b_o;
  const void *g_ca, *b_ca, *w_cq, *b_cq, *w_ckv, *b_ckv, *g_cq, *g_ck, *w_co, *b_co;
  const void *w_up, *b_up, *w_dn, *b_dn;
} dit_block_weights;

/* A packed batch on this GPU.  All arrays are HOST memory and are read during
 * the call only (their values are baked into the launches). */
typedef struct {
  int n_req;                     /* 1..DIT_MAX_REQ */
  const int32_t *cu_seqlens;     /* host [n_req+1]: latent rows of each request here */
  const int32_t *cu_seqlens_txt; /* host [n_req+1]: text rows of each request */
  const int32_t *grid_fhw;       /* host [n_req*3]: full (F,H,W) token grid of each request */
  const int32_t *pos_offset;     /* host [n_req] or NULL (all 0): flattened grid index of
                                    the request's first row here (sequence-parallel shard) */
} dit_varlen;

/* ---------------------------------------------------------------- the block */

/* Bytes of device workspace dit_block_forward / _pre_attention /
 * _post_attention need for this config and batch (0 if the arguments are
 * invalid). */
size_t dit_block_workspace_size(const dit_block_config *cfg, const dit_varlen *vl);

/* One block: y = Block(x; t, txt).  x, y: [rows, D]; t: device fp32 [n_req]
 * timesteps; mod: device fp32 [n_req, 6, D] modulation vectors in the order
 * of dit_timestep_modulation, or NULL to compute them from t (with mod given,
 * t may be NULL and the block's w_t1..b_ada are not read: a model whose
 * blocks share one timestep MLP passes each block's modulation here);
 * txt: [txt_rows, D] text embeddings.  y may equal x.  The workspace (ws,
 * ws_bytes) must hold dit_block_workspace_size bytes, 256-byte aligned; its
 * contents are scratch. */
dit_status dit_block_forward(const dit_block_config *cfg, const dit_block_weights *w,
                             const dit_varlen *vl, const void *x, const float *t,
                             const float *mod, const void *txt, void *y, void *ws,
                             size_t ws_bytes, hipStream_t stream);

/* The block split at self-attention, the two points where a sequence-parallel
 * runtime exchanges rows for heads (an all-to-all each way) between GPUs.
 * Both halves take the conditioning the way dit_block_forward does: either
 * timesteps t (the block's own timestep MLP and adaLN projection run) or
 * precomputed modulation vectors (a model whose blocks share one timestep
 * MLP; w_t1..b_ada are then not read).
 *
 * Steps before self-attention, on this GPU's rows: modulated LayerNorm, QKV
 * projection, per-head RMSNorm and rotary on q and k.  With t != NULL (device
 * fp32 [n_req]) the modulation mod = adaLN(t) is computed and written to mod
 * (device fp32 [n_req, 6, D]); with t == NULL, mod is read as given.
 * qkv: three planes [3, rows, D] (written): q = qkv[0], k = qkv[1],
 * v = qkv[2], each row-major with row stride D, head j in columns
 * [j*d, (j+1)*d).  Separate planes keep each row kernel's and attention's
 * reads on whole contiguous rows. */
dit_status dit_block_pre_attention(const dit_block_config *cfg, const dit_block_weights *w,
                                   const dit_varlen *vl, const void *x, const float *t,
                                   float *mod, void *qkv, void *ws, size_t ws_bytes,
                                   hipStream_t stream);

/* Steps after self-attention, on this GPU's rows: o [rows, D] is the
 * attention output (heads concatenated).  Gated output projection,
 * cross-attention to each request's text, gated GELU-tanh MLP; writes y.
 * mod: device fp32 [n_req, 6, D] (from dit_block_pre_attention or
 * dit_timestep_modulation), or NULL to compute it from t (device fp32
 * [n_req]) in the workspace.  y may equal x. */
dit_status dit_block_post_attention(const dit_block_config *cfg, const dit_block_weights *w,
                                    const dit_varlen *vl, const void *x, const void *o,
                                    const void *txt, const float *t, const float *mod, void *y,
                                    void *ws, size_t ws_bytes, hipStream_t stream);

/* --------------------------------------------------------------- the stages */

/* Timestep conditioning (adaLN-Zero): e = [cos(t w), sin(t w)] with
 * w_i = 10000^(-i/(F/2)); c = W_t2 SiLU(W_t1 e + b_t1) + b_t2;
 * mod = W_ada SiLU(c) + b_ada, written as fp32 [n_req, 6, D] in the order
 * shift_sa, scale_sa, gate_sa, shift_ff, scale_ff, gate_ff.  ws must hold
 * (F + 2D) * n_req floats. */
dit_status dit_timestep_modulation(const dit_block_config *cfg, const dit_block_weights *w,
                                   int n_req, const float *t, float *mod, void *ws,
                                   size_t ws_bytes, hipStream_t stream);

/* For callers that cannot allocate device memory -- code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation:
 * dit_timestep_modulation with the same arguments and results but no
 * workspace.  Its scratch (the sinusoidal encoding and the timestep MLP's two
 * hidden vectors, (F + 2D) * n_req floats, each part 256-byte aligned) lives
 * in a static device array of DIT_NOALLOC_SCRATCH_BYTES bytes that every GPU
 * the library runs on holds until the process ends; the library looks up its
 * address once per device, on the first call there.  Nothing is allocated or
 * freed.  A size over the array gives DIT_ERR_UNSUPPORTED (nothing launched).
 * Every call on one GPU shares that GPU's array and leaves its contents
 * behind (each call writes all it reads, so nothing needs clearing); calls
 * that overlap on one GPU (other streams or threads) race on it. */
#define DIT_NOALLOC_SCRATCH_BYTES (8u << 20)
dit_status dit_timestep_modulation_noalloc(const dit_block_config *cfg, const dit_block_weights *w,
                                           int n_req, const float *t, float *mod,
                                           hipStream_t stream);

/* Scaled dot-product attention over a packed batch, non-causal, no mask:
 * for request r and head h, O = softmax(Q K^T * softmax_scale) V with queries
 * rows cu_q[r]..cu_q[r+1] and keys/values rows cu_k[r]..cu_k[r+1] (host
 * arrays; cu_q == cu_k for self-attention).  Head h of row i starts at
 * q + i*q_row_stride + h*head_dim (strides in elements; likewise k, v, o).
 * softmax_scale 0 selects the standard 1/sqrt(head_dim); any other finite
 * value is used as given (inf or NaN: DIT_ERR_INVALID_ARG).  o must not
 * overlap q, k or v: the byte range from o's first to its last row must not
 * meet that of q, k or v (checked, DIT_ERR_INVALID_ARG); q, k and v may share
 * one buffer.  bf16 needs head_dim 128, and k_row_stride and v_row_stride of
 * at most 2^24 elements (the kernel forms a key tile's offsets in 32 bits;
 * larger: DIT_ERR_INVALID_ARG); fp32 takes 64 or 128.  A request with
 * queries but no keys gets rows of zeros. */
dit_status dit_attention_varlen(const void *q, const void *k, const void *v, void *o,
                                int64_t q_row_stride, int64_t k_row_stride,
                                int64_t v_row_stride, int64_t o_row_stride,
                                const int32_t *cu_q, const int32_t *cu_k, int n_req,
                                int n_heads, int head_dim, float softmax_scale,
                                dit_dtype dtype, hipStream_t stream);

/* Modulated LayerNorm: out[i] = LN(x[i]) * (1 + scale[r]) + shift[r] for row i
 * of request r (LN over `hidden`, biased variance, eps inside the root).
 * shift, scale: device fp32, request r's vector at shift + r*mod_stride.
 * x, out: [n_rows, hidden] with n_rows = cu_seqlens[n_req]. */
dit_status dit_adaln_modulate(const void *x, const float *shift, const float *scale,
                              int64_t mod_stride, const int32_t *cu_seqlens, int n_req,
                              int hidden, float eps, void *out, dit_dtype dtype,
                              hipStream_t stream);

/* Affine LayerNorm: out = LN(x) * gamma + beta (gamma, beta: [hidden], dtype). */
dit_status dit_layer_norm_affine(const void *x, const void *gamma, const void *beta,
                                 int64_t n_rows, int hidden, float eps, void *out,
                                 dit_dtype dtype, hipStream_t stream);

/* out = epilogue(A . W^T + bias): A [M, K] (row stride lda), W [N, K] (ldw),
 * bias [N] or NULL, out [M, N] (ldo), res [M, N] (ldr; RESIDUAL epilogues,
 * may equal out), gate: device fp32, request r's [N] vector at
 * gate + r*gate_stride (GATED_RESIDUAL), rows grouped by cu_seqlens.
 * bf16 needs K % 64 == 0 and N % 8 == 0. */
dit_status dit_linear(const void *a, int64_t lda, const void *w, int64_t ldw,
                      const void *bias, void *out, int64_t ldo, int64_t M, int N, int K,
                      dit_epilogue epi, const void *res, int64_t ldr, const float *gate,
                      int64_t gate_stride, const int32_t *cu_seqlens, int n_req,
                      dit_dtype dtype, hipStream_t stream);

/* The bf16 GEMM computes 256 x 256 output tiles, or smaller ones (256 x 192,
 * 128 x 256, 128 x 192, 128 x 128) where the rounds of tiles over the compute
 * units then take less time (few rows).  For tests and tuning: tile_n = 192
 * or 256 forces 256-row tiles of that width for every later bf16 GEMM of this
 * process (every entry point), 0 restores the choice per shape; any other
 * value gives DIT_ERR_INVALID_ARG.  Results do not depend on the tile shape.
 * Process-wide setting; not synchronised with work in flight (set it between
 * calls). */
dit_status dit_debug_gemm_tile_n(int tile_n);

/* The output tile (*tile_m x *tile_n) that a bf16 GEMM of M x N outputs over K
 * takes on a GPU of `compute_units` compute units, under the current debug
 * setting.  Host arithmetic only: no device is used. */
dit_status dit_debug_gemm_plan(int64_t M, int N, int K, int compute_units, int *tile_m, int *tile_n);

/* The bf16 self-attention (key ranges over 1024) runs its work items in
 * rounds of one workgroup per compute unit.  When the last round would be at
 * most half full (one request), its items are split into 2 or 4 key pieces
 * that run as one short round and are merged by a second kernel; the pieces
 * live in a static device array of 34 MB that every GPU holds until the
 * process ends, and calls that split are serialised on it by an event (not
 * under graph capture, where no split happens).  For tests and tuning:
 * mode 2 or 4 forces a split of the last request's last items (as many as
 * one round of pieces holds) into that many pieces, 1 disables splitting,
 * 0 restores the choice per shape; other values give DIT_ERR_INVALID_ARG.
 * Process-wide; set it between calls. */
dit_status dit_debug_attention_split(int mode);

/* The bf16 attention runs one of two kernel shapes per call: 8 waves per
 * workgroup (256 query rows, one workgroup per compute unit) or 4 waves (128
 * query rows, two workgroups per compute unit).  Key ranges up to 1024 take
 * the 4-wave shape; so does a single request whose 8-wave items would end in
 * a split last round when the call holds at most 3 x 64 key tiles of
 * 256-query items per compute unit.  For tests and tuning: waves = 4 or 8
 * forces that shape (and the split setting above then applies to the 8-wave
 * shape only), 0 restores the choice per call; other values give
 * DIT_ERR_INVALID_ARG.  Without a split both shapes give the same bits.
 * Process-wide; set it between calls. */
dit_status dit_debug_attention_shape(int waves);

/* The shape (*waves: 4 or 8) and last-round split (*split_pieces: 0, 2 or 4
 * key pieces for each of the last request's last *split_items items) that a
 * bf16 attention call with these ranges takes on a GPU of `compute_units`
 * compute units, under the current debug settings.  Host arithmetic only: no
 * device is used.  cu_q, cu_k: host arrays of n_req + 1 offsets from 0, as
 * for dit_attention_varlen; the outputs are host ints.  A call under graph
 * capture runs the same shape without the split. */
dit_status dit_debug_attention_plan(const int32_t *cu_q, const int32_t *cu_k, int n_req, int n_heads,
                                    int compute_units, int *waves, int *split_pieces, int *split_items);

/* ------------------------------------------- Linears on 8-bit integers */

/* A row y of fp32 values is held as int8 codes c and one fp32 scale s:
 *   m = max(max|y|, 127 * 2^-100),  s = m / 127,  c = 127 y / m to nearest, ties to even,
 * so |c| <= 127 and y = c s within half a step s / 2.  127 y / m is computed to
 * 2^-16 (a value nearer to the middle between two codes may take either); of
 * bf16 rows as they are and of their RMS norm (which 1 / rms leaves out of y / m),
 * exactly.  A row with a value that is not finite gets the scale NaN and codes 0.
 * A row's codes and scale do not depend on the rows beside it.  Codes are the
 * operands of dit_linear_i8: activations with one scale per token, and weights
 * [out, in] with one per output channel -- their rows -- from the same calls.
 *
 * codes: int8, rows of a multiple of 16 values, 16-byte aligned.  scales: fp32
 * [n_rows], 4-byte aligned.  What is written must not overlap what is read, but
 * where a call says so (checked, DIT_ERR_INVALID_ARG).  Calls without rows do
 * nothing, and their tensors may be NULL. */

/* The codes of x [n_rows, width] (dtype; strides in elements).  width <= 2^22. */
dit_status dit_quantize_rows(const void *x, int64_t x_row_stride, int64_t n_rows, int width,
                             int8_t *codes, int64_t codes_row_stride, float *scales,
                             dit_dtype dtype, hipStream_t stream);

/* dit_adaln_modulate with the result as codes [n_rows, hidden]: the codes of
 * LN(x[i]) * (1 + scale[r]) + shift[r], which is not rounded to dtype before.
 * The codes of dit_layer_norm_affine are those of one request with its gains
 * less 1 as scale and its offsets as shift, in fp32.
 * hidden <= 8192 (bf16) or 4096 (fp32), else DIT_ERR_UNSUPPORTED. */
dit_status dit_adaln_modulate_i8(const void *x, const float *shift, const float *scale,
                                 int64_t mod_stride, const int32_t *cu_seqlens, int n_req,
                                 int hidden, float eps, int8_t *codes, float *scales,
                                 dit_dtype dtype, hipStream_t stream);

/* Root-mean-square norm with the residual's addition:
 *   sum = x + z, rounded to dtype (z and sum NULL: sum is x, nothing written)
 *   y = sum / sqrt(mean(sum^2) + eps) * gain     (gain [hidden], dtype)
 * written to out (dtype), as codes and scales, or both; those not wanted are
 * NULL.  All rows are dense, [n_rows, hidden]; the mean of squares is fp32, so
 * it has to stay in range.  sum and out may each be x or z (the same address),
 * but not each other.  hidden as for dit_adaln_modulate_i8; a multiple of 8
 * (bf16) or 4 (fp32) suffices without codes. */
dit_status dit_add_rms_norm(const void *x, const void *z, const void *gain, int64_t n_rows,
                            int hidden, float eps, void *sum, void *out, int8_t *codes,
                            float *scales, dit_dtype dtype, hipStream_t stream);

/* dit_linear on codes: out = epilogue(z), z[m][n] = (sum_k a[m][k] w[n][k]) *
 * a_scales[m] * w_scales[n] + bias[n], with a [M, K] and w [N, K] of int8 (any
 * value, -128 too; strides lda and ldw, at most 2^22) and bias, out, res of
 * dtype; the epilogues as for dit_linear.  The sum is exact (32-bit integers),
 * the rest fp32, one rounding to dtype at the end: a row of a packed batch has
 * the same bits as alone.  K is a multiple of 16, at most 131,056; N a multiple
 * of 8, at most 2^24; M at most 2^28 and M N at most 2^44; else
 * DIT_ERR_UNSUPPORTED.  ldo and ldr are at most 2^24.
 * out may be res (the same address and stride). */
dit_status dit_linear_i8(const int8_t *a, int64_t lda, const float *a_scales, const int8_t *w,
                         int64_t ldw, const float *w_scales, const void *bias, void *out,
                         int64_t ldo, int64_t M, int N, int K, dit_epilogue epi, const void *res,
                         int64_t ldr, const float *gate, int64_t gate_stride,
                         const int32_t *cu_seqlens, int n_req, dit_dtype dtype,
                         hipStream_t stream);

/* dit_linear_i8 computes output tiles as dit_linear does (256 x 256, 256 x 192,
 * 128 x 256, 128 x 192, 128 x 128) or, for few rows, smaller ones whose sums over
 * K are shared by a workgroup's waves (64 x 64, 32 x 64, 32 x 32, 16 x 16),
 * whichever an estimate finds faster.  For tests and tuning:
 * dit_debug_linear_i8_tile forces one of these for every later call of this
 * process (the smaller ones where a call has at most 4,096 rows), 0 x 0 restores
 * the choice per shape; other values give DIT_ERR_INVALID_ARG.  Results do not
 * depend on it.  Process-wide; set it between calls.
 * dit_debug_linear_i8_plan: the tile that a call takes on a GPU of
 * `compute_units` compute units.  Host arithmetic only. */
dit_status dit_debug_linear_i8_tile(int tile_m, int tile_n);
dit_status dit_debug_linear_i8_plan(int64_t M, int N, int K, int compute_units, int *tile_m, int *tile_n);

/* In place on q and (if not NULL) k, each [rows, n_heads*head_dim] with row
 * stride `row_stride`: per-head RMSNorm with gains g_q / g_k (skipped when the
 * gain is NULL), then, if vl != NULL and the sections are not all 0, the
 * sectioned rotary embedding at each row's grid position (vl->cu_seqlens,
 * grid_fhw and pos_offset give the position; n_rows = vl->cu_seqlens[n_req]).
 * Without vl, n_rows rows get the RMSNorm only. */
dit_status dit_qk_norm_rope(void *q, void *k, int64_t row_stride, int64_t n_rows, int n_heads,
                            int head_dim, const void *g_q, const void *g_k, float eps,
                            const int rope_sections[3], float rope_theta, const dit_varlen *vl,
                            dit_dtype dtype, hipStream_t stream);

/* Standalone gated residual: out[i] = x[i] + gate[r] * (z[i] + bias) for row i
 * of request r; x, z, out [n_rows, hidden]; bias [hidden] (dtype) or NULL;
 * gate device fp32 at gate + r*gate_stride.  hidden <= 8192 (bf16) or 4096
 * (fp32), else DIT_ERR_UNSUPPORTED.  out may alias x or z. */
dit_status dit_gated_residual(const void *x, const void *z, const void *bias, const float *gate,
                              int64_t gate_stride, const int32_t *cu_seqlens, int n_req,
                              int hidden, void *out, dit_dtype dtype, hipStream_t stream);

/* ------------------------------------------------------ one denoising step */

/* One denoising step is the unit the paper schedules as a trajectory task: it
 * advances a request's latent along its diffusion trajectory by one timestep
 * and leaves a complete latent state behind (section 2.1, Rescheduling
 * Boundaries; section 3.1, Reschedulable Trajectory Tasks).  The paper does
 * not define the model, so this is the standard DiT stack around the block:
 * patch embedding of the latent, a timestep MLP shared by all blocks, B blocks
 * with per-block adaLN-Zero modulation, an adaLN output layer and a
 * flow-matching Euler update.  The text keys and values of every block's
 * cross-attention do not depend on the latent or the timestep, so they are
 * computed once per request (dit_text_kv) and reused by every step.
 *
 * Latent of request r: fp32, channel-major [C, F*pt, H*ph, W*pw] where
 * (F, H, W) = vl->grid_fhw[r] is its token grid, stored contiguously; the
 * requests follow each other in order (request r starts after the
 * C*F*pt*H*ph*W*pw values of requests 0..r-1).  Token n = (f*H + h)*W + w of
 * the request covers the latent patch at (f*pt, h*ph, w*pw); its patch vector
 * has P = C*pt*ph*pw entries in the order (c, i, j, k) with i over time,
 * j over height and k over width, and the model's output uses the same order,
 * so unpatchify is the exact inverse of patchify.  The step needs whole
 * requests: cu_seqlens[r+1] - cu_seqlens[r] = F*H*W and pos_offset NULL or 0. */
typedef struct {
  dit_block_config block; /* shared by every block */
  int n_blocks;           /* B >= 1 */
  int in_channels;        /* C: latent channels (the velocity has the same) */
  int patch[3];           /* (pt, ph, pw) >= 1; bf16 needs P % 64 == 0, fp32 P % 4 == 0 */
} dit_model_config;

/* Device pointers (dtype of the config) except `blocks`, a HOST array of
 * n_blocks block weight sets.  Shapes with P = C*pt*ph*pw: w_t1 [D,F] b_t1 [D]
 * w_t2 [D,D] b_t2 [D] (the shared timestep MLP); w_pe [D,P] b_pe [D] (patch
 * embedding); w_hmod [2D,D] b_hmod [2D] (output adaLN: shift, scale);
 * w_out [P,D] b_out [P] (output projection).  The blocks' own w_t1..b_t2 are
 * not read: every block takes its modulation W_ada SiLU(c) + b_ada from the
 * shared c. */
typedef struct {
  const void *w_t1, *b_t1, *w_t2, *b_t2;
  const void *w_pe, *b_pe;
  const void *w_hmod, *b_hmod;
  const void *w_out, *b_out;
  const dit_block_weights *blocks;
} dit_model_weights;

/* Elements (not bytes) of the text key/value cache: n_blocks * txt_rows * 2D,
 * dtype of the config.  0 if the arguments are invalid. */
size_t dit_text_kv_elems(const dit_model_config *cfg, const dit_varlen *vl);

/* The cross-attention keys and values of every block: for block b,
 * kv[b] = [RMSNorm_heads(txt W_ck^T + b_ck) | txt W_cv^T + b_cv] (the norm only
 * with qk_norm), [txt_rows, 2D] at kv + b*txt_rows*2D.  txt: [txt_rows, D]. */
dit_status dit_text_kv(const dit_model_config *cfg, const dit_model_weights *w,
                       const dit_varlen *vl, const void *txt, void *kv,
                       hipStream_t stream);

/* Bytes of device workspace dit_denoise_step needs (0 if invalid). */
size_t dit_denoise_workspace_size(const dit_model_config *cfg, const dit_varlen *vl);

/* One flow-matching Euler step of every request in the batch:
 *   x   = patchify(latent) W_pe^T + b_pe                    [rows, D]
 *   c   = W_t2 SiLU(W_t1 emb(t) + b_t1) + b_t2              per request
 *   x   = Block_b(x; c, kv[b]) for b = 0..B-1
 *   v   = (LN(x)(1 + scale) + shift) W_out^T + b_out, (shift, scale) = W_hmod SiLU(c) + b_hmod
 *   latent_out = latent + dt[r] * unpatchify(v)
 * t, dt: device fp32 [n_req] (timestep given to the model, and the step of
 * the flow time, sigma_next - sigma; negative when denoising).  latent,
 * latent_out: fp32 as described above; latent_out may equal latent.  kv: the
 * cache from dit_text_kv.  Workspace as for dit_block_forward, sized by
 * dit_denoise_workspace_size. */
dit_status dit_denoise_step(const dit_model_config *cfg, const dit_model_weights *w,
                            const dit_varlen *vl, const float *latent, const float *t,
                            const float *dt, const void *kv, float *latent_out, void *ws,
                            size_t ws_bytes, hipStream_t stream);

/* The latent <-> token steps of dit_denoise_step on their own.
 * dit_patchify: tokens [rows, P] (dtype, rounded to nearest even for bf16)
 * from the fp32 latent.  dit_unpatchify_euler: latent_out = latent +
 * dt[r] * unpatchify(v), v [rows, P] (dtype); latent_out may equal latent. */
dit_status dit_patchify(const dit_model_config *cfg, const dit_varlen *vl, const float *latent,
                        void *tokens, hipStream_t stream);
dit_status dit_unpatchify_euler(const dit_model_config *cfg, const dit_varlen *vl,
                                const float *latent, const void *v, const float *dt,
                                float *latent_out, hipStream_t stream);

/* ------------------------------------------ the paged 8-bit key/value cache */

/* Keys and values that stay from step to step -- the text keys and values of
 * every block, or the finished frames that a video continues -- in pages of
 * 8-bit values.  Requests get pages as they are admitted and as they grow, in
 * any order, and give them back one by one; block tables and lengths are
 * device memory, so a captured step serves whichever requests they name.
 *
 * A pool holds, for each of n_blocks blocks, n_pages pages of page_tokens
 * tokens x n_kv_heads heads.  The block table's row r lists the pages of
 * request r: its token i lies in page table[r * max_pages + i / page_tokens].
 *
 * A value is a float8 e4m3 code (4 significant bits, largest 448) times a power
 * of two, 2^(s - 127), with one scale byte s for each page and head, in
 * k_scale / v_scale [n_blocks, n_pages, n_kv_heads].  dit_cache_store writes s
 * from 27 to 247; pages that a caller fills keep to that range.  The tokens of a
 * page lie in groups of 32, in the order in which a matrix instruction takes them:
 *   k [n_blocks, n_pages, n_kv_heads, page_tokens / 32, head_dim / 16, 32, 16]:
 *     element (.., g, c, t, e) is token 32 g + t, channel 16 c + e;
 *   v [n_blocks, n_pages, n_kv_heads, page_tokens / 32, 2, head_dim, 16]:
 *     element (.., g, f, d, 4 i + j) is token 32 g + 8 i + 4 f + j, channel d.
 * Pools and slot maps are 16-byte aligned like all device memory here; scales
 * need no alignment, tables, lengths and the other index arrays 4 bytes.
 * Offsets are 64-bit; a pool may hold up to 2^31 - 1 groups per block
 * (n_pages * n_kv_heads * page_tokens / 32).
 *
 * Block tables, lengths and slot maps are read by the kernels and not checked
 * on the host; no value in them makes a kernel leave its buffers.  A length
 * below 0 counts as 0, one over the table's width or the call's bound as that;
 * tokens on a page outside 0 .. n_pages - 1 are not there.  A page belongs to
 * one request: entries of one slot map that name a page twice leave that page's
 * values undefined.  So does whatever is written while a call reads it: a table
 * or length that changes meanwhile leaves that call's results undefined. */
typedef struct {
  int n_blocks, n_pages, n_kv_heads;
  int head_dim;             /* 64 or 128 */
  int page_tokens;          /* 32, 64, 128 or 256 */
  int max_pages;            /* width of the block table; max_pages * page_tokens <= 2^30 */
  int table_rows;           /* requests that the table and lens have room for */
  void *k, *v;              /* device: pools */
  uint8_t *k_scale, *v_scale;
  int32_t *table;           /* device [table_rows, max_pages] */
  int32_t *lens;            /* device [table_rows]: cached tokens of each request */
} dit_kv_cache;

/* Entries that a slot map needs for n_rows input rows of n_req requests:
 * n_rows / page_tokens + 2 * n_req (0 if an argument is invalid). */
size_t dit_cache_run_bound(int page_tokens, int n_req, int64_t n_rows);

/* Gives the requests' new tokens their places: request r (row r of the table)
 * holds lens_before[r] tokens (device; NULL: 0 each) and gets added[r] more
 * (device), whose rows lie in the input from row r * rows_per_req (a padded
 * batch; n_rows = n_req * rows_per_req) or, with rows_per_req 0, packed one
 * request after another (n_rows: rows there are).  New pages come from
 * free_pages (device [n_free]) in order, requests in order: a request whose
 * new pages do not all fit gets none, nor does any later one that needs a page.
 * Such a request is refused, and so is one with a negative length, more tokens
 * than its table row holds or rows past the input; it keeps what it had.
 * Written: the new pages' entries of cache->table (no other entry);
 *   cache->lens[0 .. n_req): the lengths afterwards;
 *   runs (device [n_runs, 4], n_runs >= dit_cache_run_bound): the slot map,
 *     one entry {page, first input row, first place in the page, tokens} for
 *     each page that gets tokens, then zeros (tokens 0: nothing to write);
 *   counts (device [4]): pages taken, entries written, requests refused, tokens
 *     placed.
 * The pools are not touched, and k .. v_scale may be NULL.  What is written
 * must not overlap what is read, cache->lens and lens_before included. */
dit_status dit_cache_tables(const dit_kv_cache *cache, int n_req, const int32_t *lens_before,
                            const int32_t *added, int rows_per_req, int64_t n_rows,
                            const int32_t *free_pages, int n_free, int32_t *runs, int n_runs,
                            int32_t *counts, hipStream_t stream);

/* Writes the keys and values of a slot map's tokens to their places in one
 * block's pages.  k, v: [n_rows, n_kv_heads * head_dim] (dtype) at row strides
 * in elements; both may lie in one buffer.  The scale of a page that the entry
 * begins (place 0) is the smallest power of two 2^e, e >= -100, for which no
 * finite value of its tokens exceeds 448 * 2^e; an entry that continues a page
 * leaves the scale or makes it larger, and then brings the page's earlier codes
 * to it.  Codes are rounded to nearest, ties to even; infinities become NaN.
 * Places behind the entry's tokens and all other pages keep their bytes.  Without
 * rows (n_rows 0, k and v may be NULL) nothing is written. */
dit_status dit_cache_store(const dit_kv_cache *cache, int block, const void *k, const void *v,
                           int64_t k_row_stride, int64_t v_row_stride, int64_t n_rows,
                           const int32_t *runs, int n_runs, dit_dtype dtype, hipStream_t stream);

/* Attention of packed queries over the cache, non-causal: for request r (row r
 * of the table) and head h, O = softmax(Q K^T * softmax_scale) V over the
 * request's cached tokens, with query rows cu_q[r]..cu_q[r+1] (host array) and
 * query head h on key/value head h / (n_heads / n_kv_heads).  q, o, strides and
 * softmax_scale as for dit_attention_varlen; head_dim (64 or 128 in both
 * dtypes) and n_kv_heads, a divisor of n_heads, are the cache's; n_heads *
 * head_dim is below 2^31 (larger: DIT_ERR_UNSUPPORTED).  A request
 * without tokens gets rows of zeros; table rows from n_req on are not read.  A
 * batch without query rows does nothing (q and o may be NULL).
 * Scores, probabilities' sums and products are fp32: a score of minus infinity
 * has no weight (a row of nothing else is zeros), one of infinity gives NaN, and
 * a row's sum of |v| over its tokens has to stay in range.
 * max_len bounds the lengths (0: the table's width): longer requests are cut
 * there, and the work is divided by it.  Where whole row tiles would leave
 * compute units idle, the tokens are divided among the workgroups and what
 * they find is joined in the workspace: ws holds
 * dit_attention_cached_workspace_size bytes, 256-byte aligned (0 bytes: NULL
 * will do), its contents are scratch, and calls that may overlap in time, or
 * captured graphs that may, each need their own. */
size_t dit_attention_cached_workspace_size(const dit_kv_cache *cache, const int32_t *cu_q, int n_req,
                                           int n_heads, int max_len, dit_dtype dtype);
dit_status dit_attention_cached(const dit_kv_cache *cache, int block, const void *q, void *o,
                                int64_t q_row_stride, int64_t o_row_stride, const int32_t *cu_q,
                                int n_req, int n_heads, int max_len, float softmax_scale,
                                dit_dtype dtype, void *ws, size_t ws_bytes, hipStream_t stream);

/* dit_text_kv into a cache with n_blocks pools of the model's heads: the text
 * rows that runs names go to their places in every block's pages (from
 * dit_cache_tables with n_rows = vl->cu_seqlens_txt[n_req]).  The workspace
 * holds one block's keys and values in the config's dtype,
 * dit_text_kv_cached_workspace_size bytes, 256-byte aligned.  Prompts without
 * rows: nothing is done, and txt and ws may be NULL. */
size_t dit_text_kv_cached_workspace_size(const dit_model_config *cfg, const dit_varlen *vl);
dit_status dit_text_kv_cached(const dit_model_config *cfg, const dit_model_weights *w,
                              const dit_varlen *vl, const void *txt, const dit_kv_cache *cache,
                              const int32_t *runs, int n_runs, void *ws, size_t ws_bytes,
                              hipStream_t stream);

/* dit_denoise_step with the text keys and values of a cache: request r of the
 * batch attends to row r of the cache's table.  vl->cu_seqlens_txt is not read
 * and may be NULL.  A captured step may be replayed for other prompts: the
 * table and lens name them.  The cross-attention's work is divided by the table's
 * width, so a table for prompts is best as wide as the longest of them. */
size_t dit_denoise_cached_workspace_size(const dit_model_config *cfg, const dit_varlen *vl,
                                         const dit_kv_cache *cache);
dit_status dit_denoise_step_cached(const dit_model_config *cfg, const dit_model_weights *w,
                                   const dit_varlen *vl, const float *latent, const float *t,
                                   const float *dt, const dit_kv_cache *cache, float *latent_out,
                                   void *ws, size_t ws_bytes, hipStream_t stream);

/* -------------------------------------------------------------- diagnostics */

const char *dit_status_string(dit_status s);
/* Thread-local description of the last failure in this thread ("" if none). */
const char *dit_last_error(void);
int dit_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DIT_BLOCK_H */
