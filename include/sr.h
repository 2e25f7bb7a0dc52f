/*
 * sr.h -- C ABI of libsr, the MI355X (gfx950) hot path of Sparse-Reslim:
 * random (or top-k) token selection, gather, the n2 middle transformer blocks
 * run on the routed tokens only (forward and backward), and the residual-delta
 * scatter back into the full token sequence, plus the dense keep=100% mode.
 *
 * The operations follow the paper's statement of the method:
 *   selection            Sec. 3.2 "Random token selection"; Alg. 1 stage 2; App. A.4
 *   gather / scatter     Sec. 3.2 "Residual delta formulation", Eq. (scatter)
 *   middle stack         Eq. (sparse_forward); block of Sec. 3.3
 *   dense mode           Sec. 3.4 "Architecture-agnostic design" (r = 1)
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Tensor arguments are DEVICE pointers owned by the caller, contiguous,
 *    row-major, 16-byte aligned.  The library allocates no device memory:
 *    saved activations and scratch space are caller buffers sized by
 *    sr_workspace_bytes / sr_select_scratch_bytes.
 *  - `stream` is a hipStream_t (NULL = the default stream).  Calls enqueue work
 *    on it and return without waiting.  The blocks backward also uses one extra
 *    stream per device (created on the first call, default priority, kept until the
 *    process ends) for its weight gradients, joined to `stream` through events: all of
 *    the call's work is complete when later work on `stream` starts.
 *  - Calls can be captured into a HIP graph (after one eager call has created the second
 *    stream and its events): they record no memset and no host synchronisation, and the
 *    backward forks and joins its second stream through events on `stream`.  A replay
 *    repeats the captured scalar arguments (seed, step, sizes).
 *  - Arguments are validated on the host before anything is enqueued; on error
 *    nothing is launched, a non-zero sr_status is returned and sr_last_error()
 *    (thread-local) describes it.  SR_EHIP reports a failed launch.
 *  - Storage dtype (sr_config.dtype): SR_F32 or SR_BF16.  Activations, weights,
 *    biases, LayerNorm parameters and the conditioning vector are stored in it;
 *    all accumulation is fp32; weight gradients and dcond are always fp32.
 *  - Determinism: the same call on the same inputs gives the same bits, whatever runs beside it.
 *    A sample's bits may depend on the batch it is in: how a sum is grouped (tiles that share
 *    its range, runs of a cut attention) follows the rows B*S and the heads of the call, and
 *    with it the rounding of the stored activations.  In bf16 they no longer do once one sample
 *    fills the GPU by itself: ceil(S/64) * D/64 > 256, and H * ceil(S/256) > 128 at head dim 64
 *    or H * ceil(S/128) > 256 at head dim 32 (D = 1024 with 16 heads: from S = 2049).
 *  - Non-finite values: a NaN or Inf in a sample's inputs (tokens, conditioning) or in the
 *    parameters gives non-finite values in that sample's outputs and gradients (attention mixes
 *    every token of a sample, so all of its routed rows may be affected; which elements is not
 *    specified) and in the parameter gradients; other samples' results are unchanged and rows
 *    the scatter does not touch keep their values.  Nothing is clamped or checked on the GPU.
 *  - Debugging: with SR_DEBUG=1 in the environment (read at every call), sr_gather,
 *    sr_scatter_delta and sr_routed_blocks_fwd/bwd copy idx to the host, synchronising
 *    `stream`, and return SR_EINVAL before any launch if a row is not strictly increasing
 *    inside [0, L).  Off by default (no host synchronisation on the hot path); not for use
 *    under graph capture.
 *  - Shapes: B samples, L tokens per sample, D channels, H heads (D % H == 0),
 *    F MLP width, n_blocks middle blocks; S = K (routed) or L (dense) tokens per
 *    sample inside the stack.
 *  - Support: D % 64 == 0, F % 64 == 0, D <= 2048, head dim D/H in {32, 64, 128}
 *    (bf16 and fp32 storage each run matrix-core attention kernels with fp32 accumulation); 1 <= K <= L; B*L*D*elt < 2^31 bytes per
 *    token tensor, and for the block-stack calls also B*S*max(F, 3D)*4 < 2^31 with S the
 *    call's rows per sample (the S or K routed tokens; L for the dense calls), which size the
 *    internal fp32 buffers.  Anything else returns SR_EUNSUPPORTED.
 */
#ifndef SR_H
#define SR_H

#include <stddef.h>
#include <stdint.h>

#ifndef SR_API
#define SR_API __attribute__((visibility("default")))
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SR_OK = 0,
  SR_EINVAL = 1,        /* null pointer, negative size, bad enum value        */
  SR_ESHAPE = 2,        /* inconsistent shapes (K > L, D % H != 0, ...)        */
  SR_EDTYPE = 3,        /* unknown storage dtype                              */
  SR_EALIGN = 4,        /* a tensor pointer is not 16-byte aligned            */
  SR_EWORKSPACE = 5,    /* saved / scratch buffer smaller than required       */
  SR_EUNSUPPORTED = 6,  /* valid but not supported by this library            */
  SR_EHIP = 7           /* a HIP launch failed; sr_last_error() has the text  */
} sr_status;

typedef enum { SR_F32 = 0, SR_BF16 = 1 } sr_dtype;

/* Block kinds.
 * SR_BLOCK_PRELN: h1 = h + Attn(LN1(h)); h' = h1 + MLP(LN2(h1))  (Sec. 3.3).
 * SR_BLOCK_ADALN: (shift1,scale1,gate1,shift2,scale2,gate2) = c W_ada^T + b_ada per
 *   sample; h1 = h + gate1*Attn(LN0(h)*(1+scale1)+shift1);
 *   h' = h1 + gate2*MLP(LN0(h1)*(1+scale2)+shift2), LN0 = LayerNorm without affine
 *   (FiLM scale/shift and a gate from a global conditioning vector, as in the
 *   paper's EDM block, Sec. 2 "Generative forecasting"). */
typedef enum { SR_BLOCK_PRELN = 0, SR_BLOCK_ADALN = 1 } sr_block_kind;

/* Added to sr_config.kind (SR_BLOCK_PRELN | SR_BLOCK_SAVE8): the block calls keep a forward's activations for
 * its backward in 8 bits (SR_Q8_BLOCK, below), 10.3 instead of 24.6 KB per token and block at D = 1024 in
 * bf16, plus one block's worth of working buffers (34 KB per token, against 10).  The forward's output is bit
 * for bit that without the flag; the gradients are those of the kept values (block inputs, q, k, v, attention
 * output, residual and MLP pre-activation, each within half a step, 1/127 of the largest of its
 * 32 neighbours), with the forward's LayerNorm statistics.  The backward runs the attention of the kept q, k and v
 * again, so that its probabilities sum to one whatever the size of the logits; logits of deviation s differ from the
 * forward's by about s / 80.  sr_workspace_bytes, the
 * sparse, dense and routed block calls take it, forward and backward alike (the same flag in both); a backward
 * also writes the working part of `saved`, so calls on one `saved` must not overlap.  sr_attention_colsums
 * returns SR_EUNSUPPORTED.  Calls that do not read `kind` ignore it, the generative blocks' (sr_edm_*) among them:
 * their `saved` keeps its full size. */
enum { SR_BLOCK_SAVE8 = 16 };

/* Selectors.
 * SR_SEL_RANDOM: per sample, the K tokens with the smallest SplitMix64 keys
 *   key_i = mix(s_b + (i+1)*gamma), s_b = mix(s_step + (b+1)*gamma),
 *   s_step = mix(seed + (step+1)*gamma): a uniformly random K-subset
 *   (randperm(L)[:K]), ascending (Sec. 3.2; App. A.4).  A fresh `step` gives a
 *   fresh draw (Sec. 3.4 "Training and inference").
 * SR_SEL_TOPK_DIFFNORM: the K tokens with the largest
 *   score_i = sum_d (x_t[i,d] - x_prev[i,d])^2 (fp32, fixed evaluation order:
 *   16-byte chunks dealt round-robin to 64 partial sums, each summed in order,
 *   then combined by an xor butterfly 32,16,8,4,2,1; no fused multiply-add),
 *   ties to the lower index, ascending (deterministic routing ablation,
 *   App. "regularization decomposition"). */
typedef enum { SR_SEL_RANDOM = 0, SR_SEL_TOPK_DIFFNORM = 1 } sr_select_kind;

typedef struct {
  int32_t B, L, D, H, F, n_blocks;
  int32_t dtype;       /* sr_dtype */
  int32_t kind;        /* sr_block_kind, with SR_BLOCK_SAVE8 or without */
  float ln_eps;        /* LayerNorm epsilon (the paper leaves it unstated; 1e-6 here) */
  int32_t idx_shared;  /* 1: idx is [1,K], one index set for every sample (the
                          App. A.4 listing); 0: idx is [B,K], one set per sample */
} sr_config;

/* Parameters of one block, nn.Linear layout [out, in], storage dtype, device
 * pointers.  QKV rows are ordered q, k, v; head j owns rows j*hd .. j*hd+hd-1 of
 * each.  PRELN blocks read ln*, w_qkv..b_fc2 (w_ada/b_ada may be NULL); ADALN
 * blocks read w_qkv..b_fc2 and w_ada [6D,D] / b_ada [6D] (ln* may be NULL). */
typedef struct {
  const void *ln1_w, *ln1_b, *w_qkv, *b_qkv, *w_o, *b_o;
  const void *ln2_w, *ln2_b, *w_fc1, *b_fc1, *w_fc2, *b_fc2;
  const void *w_ada, *b_ada;
} sr_block_params;

/* Gradients of one block, fp32 device buffers shaped like the parameters.
 * They are OVERWRITTEN (not accumulated).  A NULL member skips that gradient;
 * members for parameters the block kind does not use are written with zeros. */
typedef struct {
  float *ln1_w, *ln1_b, *w_qkv, *b_qkv, *w_o, *b_o;
  float *ln2_w, *ln2_b, *w_fc1, *b_fc1, *w_fc2, *b_fc2;
  float *w_ada, *b_ada;
} sr_block_grads;

/* Text of the last error on this thread ("" if none).  The pointer stays valid
 * until the next failing call on the same thread. */
SR_API const char* sr_last_error(void);

/* Library version string. */
SR_API const char* sr_version(void);

/* Bytes of the `saved` (activations kept from forward for backward) and
 * `scratch` buffers needed by the block calls at S tokens per sample.  Neither falls when S or B
 * grows, all else equal: buffers sized for the largest call serve the smaller ones.  (Part of
 * `scratch` is room for the partial results of an attention backward with few heads, which is cut
 * into runs.  A call asks only for the rest: without that room it runs uncut, slower and with its
 * sums in another order.) */
SR_API sr_status sr_workspace_bytes(const sr_config* cfg, int32_t S, size_t* saved_bytes,
                             size_t* scratch_bytes);

/* Bytes of scratch sr_select_indices needs for `select_kind` (0 for random). */
SR_API sr_status sr_select_scratch_bytes(const sr_config* cfg, int32_t select_kind,
                                  size_t* scratch_bytes);

/* Token selection (Sec. 3.2; Alg. 1 stage 2; App. A.4).
 *   K: tokens kept per sample, K = floor(r*L) computed by the caller (1 <= K <= L).
 *   select_kind: sr_select_kind.  seed, step: the random draw (RANDOM only).
 *   x_t, x_prev: [B,L,D] storage dtype (TOPK only; NULL for RANDOM).
 *   idx: [B,K] int32 out (or [1,K] with idx_shared, drawn for sample 0),
 *        strictly increasing per row.
 *   scratch: sr_select_scratch_bytes bytes (may be NULL when that is 0). */
SR_API sr_status sr_select_indices(const sr_config* cfg, int32_t K, int32_t select_kind,
                            uint64_t seed, uint64_t step, const void* x_t,
                            const void* x_prev, int32_t* idx, void* scratch,
                            size_t scratch_bytes, void* stream);

/* sr_select_indices without a scratch argument and without allocating, for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc).  Same arguments, results and errors as sr_select_indices; the
 * SR_SEL_TOPK_DIFFNORM scores go to a device array that the library holds on each GPU it runs
 * on until the process ends (SR_SELECT_NOALLOC_MAX_TOKENS fp32 values, 4 MiB per GPU), looked
 * up once per GPU on the first call there.  B*L (L with idx_shared) above that limit returns
 * SR_EUNSUPPORTED before anything is enqueued.  Every call on one GPU shares its array: calls
 * that overlap on one GPU (different streams, threads) race and must be ordered by the caller.
 * SR_SEL_RANDOM uses no scratch and runs as in sr_select_indices. */
#define SR_SELECT_NOALLOC_MAX_TOKENS (1 << 20)
SR_API sr_status sr_select_indices_noalloc(const sr_config* cfg, int32_t K, int32_t select_kind,
                                    uint64_t seed, uint64_t step, const void* x_t,
                                    const void* x_prev, int32_t* idx, void* stream);

/* Gather (Sec. 3.2, h0 = Gather(x, I)): h0[b,k,:] = x[b, idx[b,k], :], a bit copy.
 *   x: [B,L,D] storage dtype; idx: [B,K] (or [1,K]); h0: [B,K,D] out.
 *   idx entries must lie in [0,L) (sr_select_indices guarantees it). */
SR_API sr_status sr_gather(const sr_config* cfg, int32_t K, const void* x, const int32_t* idx,
                    void* h0, void* stream);

/* Residual-delta scatter (Eq. scatter), IN PLACE on x:
 *   x[b,i,:] <- rnd( f32(x[b,i,:]) + (f32(h[b,k,:]) - f32(h0[b,k,:])) ), i = idx[b,k],
 * fp32 subtract then add, one round-to-nearest-even to the storage dtype; rows not
 * in idx are not touched (they keep x0 bit for bit).  h0 == NULL re-reads x[idx]
 * (equal to h0 by definition).  idx rows must be duplicate-free.
 * The backward of the routed step uses the same call:
 *   gather(g) -> blocks_bwd -> scatter_delta(g, dh_in, NULL, idx). */
SR_API sr_status sr_scatter_delta(const sr_config* cfg, int32_t K, void* x, const void* h,
                           const void* h0, const int32_t* idx, void* stream);

/* The n_blocks middle blocks on S tokens per sample (Eq. sparse_forward).
 *   params: host array of n_blocks sr_block_params.
 *   cond: [B,D] storage dtype (ADALN) or NULL.
 *   h_in: [B,S,D] in; h_out: [B,S,D] out (may not alias h_in).
 *   saved: activations for sr_sparse_blocks_bwd; must outlive it.
 * Inside the stack the residual stream is fp32; h_out is rounded once. */
SR_API sr_status sr_sparse_blocks_fwd(const sr_config* cfg, int32_t S,
                               const sr_block_params* params, const void* cond,
                               const void* h_in, void* h_out, void* saved,
                               size_t saved_bytes, void* scratch, size_t scratch_bytes,
                               void* stream);

/* Vector-Jacobian product of sr_sparse_blocks_fwd (same cfg, S, params, cond, saved).
 *   dh_out: [B,S,D] storage dtype in;  dh_in: [B,S,D] out (may alias dh_out).
 *   grads: host array of n_blocks sr_block_grads (fp32, overwritten).
 *   dcond: [B,D] fp32 out (ADALN; summed over blocks) or NULL. */
SR_API sr_status sr_sparse_blocks_bwd(const sr_config* cfg, int32_t S,
                               const sr_block_params* params, const void* cond,
                               const void* saved, size_t saved_bytes, const void* dh_out,
                               void* dh_in, const sr_block_grads* grads, float* dcond,
                               void* scratch, size_t scratch_bytes, void* stream);

/* Dense keep=100% mode (Sec. 3.4, r = 1): the same blocks on all L tokens. */
SR_API sr_status sr_dense_blocks_fwd(const sr_config* cfg, const sr_block_params* params,
                              const void* cond, const void* x_in, void* x_out, void* saved,
                              size_t saved_bytes, void* scratch, size_t scratch_bytes,
                              void* stream);
SR_API sr_status sr_dense_blocks_bwd(const sr_config* cfg, const sr_block_params* params,
                              const void* cond, const void* saved, size_t saved_bytes,
                              const void* dx_out, void* dx_in, const sr_block_grads* grads,
                              float* dcond, void* scratch, size_t scratch_bytes, void* stream);

/* The routed step's forward in one call (Alg. 1 stage 2): gather, the n_blocks blocks on
 * the K routed tokens, residual-delta scatter, with the gather fused into the stack's input
 * step and the scatter into the last block's output epilogue.  In place on x:
 *   x[b,i,:] <- rnd( f32(x0[b,i,:]) + (f32(h[b,k,:]) - f32(x0[b,i,:])) ),  i = idx[b,k],
 * h = the stack's output on h0 = x0[idx] rounded to the storage type; bit for bit the
 * result of sr_gather + sr_sparse_blocks_fwd + sr_scatter_delta.  Rows not in idx keep x0.
 *   idx: [B,K] (or [1,K] with idx_shared), duplicate-free rows inside [0,L).
 *   saved: sr_workspace_bytes(cfg, K) bytes; it holds what sr_routed_blocks_bwd (or
 *          sr_sparse_blocks_bwd with S = K) needs.  No scratch. */
SR_API sr_status sr_routed_blocks_fwd(const sr_config* cfg, int32_t K, const int32_t* idx,
                               const sr_block_params* params, const void* cond, void* x,
                               void* saved, size_t saved_bytes, void* stream);

/* Its backward in one call, in place on g (in: gradient of x', out: gradient of x0):
 *   g <- g + Scatter(J^T g[I] - g[I], I)  (the gradient delta rounded once, as in
 * sr_scatter_delta(g, dh_in, NULL, idx)); bit for bit the result of sr_gather(g) +
 * sr_sparse_blocks_bwd + sr_scatter_delta.  grads, dcond, scratch as for
 * sr_sparse_blocks_bwd with S = K. */
SR_API sr_status sr_routed_blocks_bwd(const sr_config* cfg, int32_t K, const int32_t* idx,
                               const sr_block_params* params, const void* cond,
                               const void* saved, size_t saved_bytes, void* g,
                               const sr_block_grads* grads, float* dcond, void* scratch,
                               size_t scratch_bytes, void* stream);

/* Asymmetric attention of the generative block's sparse middle stage (Sec. 3.4,
 * "Integration with Generative Forecasting"): queries from Sq tokens (the routed ones),
 * keys and values from Skv tokens (the whole conditioning sequence); per sample and head
 *   O = softmax(q k^T / sqrt(hd)) v   over the Skv keys,   cost O(Sq Skv D).
 * Only cfg's B, D, H and dtype are read and validated (D % 64 == 0, head dim D/H in
 * {32, 64, 128}); L, F, n_blocks, kind, ln_eps and idx_shared are ignored.
 *   q: [B,Sq,D]; kv: [B,Skv,2D] (k of head h at columns h*hd .., v at D + h*hd ..);
 *   O: [B,Sq,D] out; lse: [B,H,Sq] fp32 out, the base-2 log-sum-exp of the scaled scores.
 * Runs the self-attention kernels, given the two buffers and token counts.  Deterministic. */
SR_API sr_status sr_cross_attention_fwd(const sr_config* cfg, int32_t Sq, int32_t Skv, const void* q,
                                 const void* kv, void* O, float* lse, void* stream);

/* Its backward: dq [B,Sq,D] and dkv [B,Skv,2D] (dk, dv in kv's layout) out, from the
 * forward's q, kv, O, lse and the output gradient dO [B,Sq,D]; delta: [B,H,Sq] fp32
 * caller scratch (receives rowsum(dO * O) per head). */
SR_API sr_status sr_cross_attention_bwd(const sr_config* cfg, int32_t Sq, int32_t Skv, const void* q,
                                 const void* kv, const void* O, const void* dO,
                                 const float* lse, void* dq, void* dkv, float* delta,
                                 void* stream);

/* The generative model's block (Sec. 3.4 "Integration with Generative Forecasting", Alg. 2
 * stage 2; App. A.1 EDM table: FiLM -> self-attention -> sigma-gated cross-attention -> MLP),
 * on S tokens per sample (the K routed ones in the sparse stage, S = L for the dense block)
 * with cross-attention to all L conditioning tokens (the asymmetric design):
 *   (shift, scale) = e W_film^T + b_film;   g = sigmoid(e W_g^T + b_g)       (per sample)
 *   u  = LN0(h) (1 + scale) + shift            LN0: LayerNorm without affine parameters
 *   h1 = h + SelfAttn(u)                       w_qkv [3D,D], b_qkv, w_o [D,D], b_o (over S tokens)
 *   h2 = h1 + g * (CrossAttn(LNc(h1), Z_c) W_oc^T + b_oc)
 *        queries LNc(h1) W_q^T + b_q (S tokens), [keys values] = Z_c W_kv^T + b_kv (L tokens,
 *        rows of w_kv [2D,D] ordered k, v, head-major within each)
 *   h' = h2 + GELU(LN2(h2) W_fc1^T + b_fc1) W_fc2^T + b_fc2
 * e: the noise embedding [B,D]; Z_c: the conditioning tokens [B,L,D]; both storage dtype and
 * shared by every block.  nn.Linear layout [out, in], storage dtype. */
typedef struct {
  const void *w_film, *b_film, *w_qkv, *b_qkv, *w_o, *b_o;
  const void *lnc_w, *lnc_b, *w_q, *b_q, *w_kv, *b_kv, *w_oc, *b_oc, *w_g, *b_g;
  const void *ln2_w, *ln2_b, *w_fc1, *b_fc1, *w_fc2, *b_fc2;
} sr_edm_block_params;

/* Its gradients, fp32, shaped like the parameters, OVERWRITTEN; a NULL member skips one. */
typedef struct {
  float *w_film, *b_film, *w_qkv, *b_qkv, *w_o, *b_o;
  float *lnc_w, *lnc_b, *w_q, *b_q, *w_kv, *b_kv, *w_oc, *b_oc, *w_g, *b_g;
  float *ln2_w, *ln2_b, *w_fc1, *b_fc1, *w_fc2, *b_fc2;
} sr_edm_block_grads;

/* Bytes of `saved` and `scratch` for the generative blocks at S query tokens per sample and
 * cfg->L conditioning tokens (cfg->kind and cfg->idx_shared are not used); as above, neither falls
 * when S or B grows. */
SR_API sr_status sr_edm_workspace_bytes(const sr_config* cfg, int32_t S, size_t* saved_bytes,
                                 size_t* scratch_bytes);

/* cfg->n_blocks generative blocks on h_in [B,S,D] -> h_out [B,S,D] (may not alias), given the
 * noise embedding e [B,D] and the conditioning tokens zc [B,L,D] (L = cfg->L), storage dtype.
 * The residual stream is fp32 inside; h_out is rounded once.  saved: activations for
 * sr_edm_blocks_bwd (sr_edm_workspace_bytes), which must outlive it.  The sparse stage of
 * Alg. 2 is sr_gather -> this call with S = K -> sr_scatter_delta. */
SR_API sr_status sr_edm_blocks_fwd(const sr_config* cfg, int32_t S, const sr_edm_block_params* params,
                            const void* e, const void* zc, const void* h_in, void* h_out, void* saved,
                            size_t saved_bytes, void* stream);

/* Its vector-Jacobian product: dh_in [B,S,D] storage out (may alias dh_out); grads (host array
 * of n_blocks, fp32, overwritten); dzc [B,L,D] fp32 out, the gradient of the conditioning
 * tokens summed over the blocks, and de [B,D] fp32 out, that of the noise embedding summed over
 * the blocks (either may be NULL). */
SR_API sr_status sr_edm_blocks_bwd(const sr_config* cfg, int32_t S, const sr_edm_block_params* params,
                            const void* e, const void* zc, const void* saved, size_t saved_bytes,
                            const void* dh_out, void* dh_in, const sr_edm_block_grads* grads,
                            float* dzc, float* de, void* scratch, size_t scratch_bytes,
                            void* stream);

/* Debug check of an index set: *ok_dev (device int32) is set to 1 if every row of
 * idx is strictly increasing and inside [0,L), else 0. */
SR_API sr_status sr_validate_indices(const sr_config* cfg, int32_t K, const int32_t* idx,
                              int32_t* ok_dev, void* stream);

/* Attention received per token, for the attention-score selector (keep the K tokens that the
 * final block of the dense early stage attends to most: Sec. 4.4 "Random vs. learned token
 * selection", Tab. selection).  For block `block` (0-based) of the forward that
 * wrote `saved` on S tokens per sample (sr_sparse_blocks_fwd, or S = L for
 * sr_dense_blocks_fwd):
 *   colsum[b,h,j] = sum over i < S of P_h[i,j],  P_h = softmax_j(q_i . k_j / sqrt(hd)),
 * the forward's probabilities (recomputed from its saved q, k and row log-sum-exp).
 *   saved: that forward's buffer, at least sr_workspace_bytes(cfg, S) bytes, unchanged
 *          since the forward (the call only reads it).
 *   colsum: [B,H,S] fp32 out, overwritten.  Sums run in a fixed order (deterministic).
 * Per head, the S column sums add up to S up to rounding (every row of P sums to 1). */
SR_API sr_status sr_attention_colsums(const sr_config* cfg, int32_t S, const void* saved,
                               size_t saved_bytes, int32_t block, float* colsum,
                               void* stream);

/* Top-K by given scores: per sample b, score_j = sum over p < parts of planes[b,p,j],
 * added in fp32 in plane order starting from +0 (parts = H with sr_attention_colsums'
 * output gives the attention received summed over heads); the K largest scores are
 * kept, ties to the lower token index, idx ascending.
 *   planes: [B,parts,L] fp32 (or [1,parts,L] with idx_shared), finite and >= 0.
 *   idx: [B,K] int32 out (or [1,K] with idx_shared); 1 <= K <= L, parts >= 1. */
SR_API sr_status sr_select_topk_scores(const sr_config* cfg, int32_t K, const float* planes,
                                int32_t parts, int32_t* idx, void* stream);

/* Eight-bit activations.
 * Tokens and activations held as signed 8-bit codes, the linear layer that multiplies such codes, and
 * the weight gradient that reads them.  These calls take their sizes and sr_dtype directly (no sr_config).
 *
 * SR_Q8_ROW, for the operands of sr_linear8 (the tokens, or a weight's rows: one scale per token, one
 *   per output channel).  Per row with a = max |x|:  q = 127 x / a to the nearest integer, halves to
 *   the even one, of the exact quotient; scale = a / 127 in fp32 (value: q * scale).  A row of zeros has
 *   q = 0, scale = 0.  A row with an Inf or NaN has q = 0 and scale = NaN.
 * SR_Q8_BLOCK, for activations kept from a forward for its backward: a power of two 2^e per 32
 *   channels, e the smallest integer in [-126, 121] with max |x| <= 127 2^e, kept as the byte e + 127;
 *   q = x 2^-e to the nearest integer, halves to even, within +-127 (which only a block with values
 *   above 1.98 * 2^127 meets).  The value q * 2^e is exact in bf16 and fp32.  A block with an Inf or
 *   NaN has the byte 255 and q = 0, and reads back as NaN. */
typedef enum { SR_Q8_ROW = 0, SR_Q8_BLOCK = 1 } sr_q8_kind;

typedef enum { SR_ACT_NONE = 0, SR_ACT_GELU = 1 } sr_act;

/* x [M,N] (storage type) -> q [M,N] int8 and scale: fp32 [M] (SR_Q8_ROW) or bytes [M,N/32]
 * (SR_Q8_BLOCK).  M >= 1, N % 64 == 0, M*N*elt < 2^31 bytes. */
SR_API sr_status sr_quantize8(int32_t q8_kind, int32_t dtype, int32_t M, int32_t N, const void* x, int8_t* q,
                       void* scale, void* stream);

/* The values that q and scale stand for -> x [M,N] storage type (SR_Q8_ROW: q * scale in
 * fp32, then rounded to it; SR_Q8_BLOCK: exact).  Sizes as above. */
SR_API sr_status sr_dequantize8(int32_t q8_kind, int32_t dtype, int32_t M, int32_t N, const int8_t* q,
                         const void* scale, void* x, void* stream);

/* Linear layer on SR_Q8_ROW operands (nn.Linear layout):
 *   y[m,n] = act( xs[m] ws[n] sum_k xq[m,k] wq[n,k] + bias[n] )
 * with an exact int32 sum, the rest in fp32 and one rounding to the storage type.
 *   xq [M,K], xs [M]: the tokens;  wq [N,K], ws [N]: the weight;  bias [N] storage type or NULL;
 *   y [M,N] storage type out;  act: sr_act (the exact GELU; its limits at the
 * infinities).
 * M >= 1, N % 8 == 0, K % 64 == 0, K <= 65536; M*K, N*K and M*N*elt < 2^31 bytes. */
SR_API sr_status sr_linear8(int32_t dtype, int32_t act, int32_t M, int32_t N, int32_t K, const int8_t* xq,
                     const float* xs, const int8_t* wq, const float* ws, const void* bias, void* y,
                     void* stream);

/* Weight and bias gradient of a linear layer from the SR_Q8_BLOCK checkpoint of its input:
 *   dw[n,k] = sum_m dy[m,n] xhat[m,k],   db[n] = sum_m dy[m,n]
 *   dy [M,N] storage type;  xq [M,K], xe [M,K/32]: the checkpoint, read in 8 bits;
 *   dw [N,K] fp32 and db [N] fp32 (or NULL), overwritten.  Every product is exact (but for the bits
 *   of an fp32 dy below 2^-133) and sums are fp32, in a fixed order (deterministic).  scratch: sr_weight_grad8_scratch_bytes bytes (NULL when 0).
 * M >= 1, N % 8 == 0, K % 64 == 0, K <= 65536; M*N*elt, M*K and N*K*4 < 2^31 bytes. */
SR_API sr_status sr_weight_grad8_scratch_bytes(int32_t dtype, int32_t M, int32_t N, int32_t K,
                                        size_t* scratch_bytes);
SR_API sr_status sr_weight_grad8(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* dy, const int8_t* xq,
                          const uint8_t* xe, float* dw, float* db, void* scratch, size_t scratch_bytes,
                          void* stream);

/* The blocks' forward with weights and tokens in 8 bits, for forecasts (nothing is kept for a backward): the
 * block of sr_config.kind with its four linear layers as sr_linear8 on SR_Q8_ROW tokens (the LayerNorm outputs, the
 * attention output and GELU's output, each quantised per token) and SR_Q8_ROW weights.  LayerNorm, attention,
 * modulation and the fp32 residual stream are those of sr_sparse_blocks_fwd.
 * Parameters of one block: int8 weights [out,in] with fp32 scales [out], as sr_quantize8 (SR_Q8_ROW) gives them
 * for the rows of nn.Linear weights; the others in storage dtype (ln* for SR_BLOCK_PRELN, w_ada / b_ada for
 * SR_BLOCK_ADALN, the rest may be NULL). */
typedef struct {
  const void *ln1_w, *ln1_b, *b_qkv, *b_o, *ln2_w, *ln2_b, *b_fc1, *b_fc2, *w_ada, *b_ada;
  const int8_t *w_qkv, *w_o, *w_fc1, *w_fc2;
  const float *s_qkv, *s_o, *s_fc1, *s_fc2;
} sr_block_params8;

/* Bytes of scratch for S tokens per sample (never less for more of S or B). */
SR_API sr_status sr_blocks8_scratch_bytes(const sr_config* cfg, int32_t S, size_t* scratch_bytes);

/* h_in [B,S,D] -> h_out [B,S,D] (storage dtype; may alias h_in): n_blocks blocks; params: host array of n_blocks;
 * cond: [B,D] (ADALN) or NULL.  S is not bounded by cfg->L. */
SR_API sr_status sr_blocks8_fwd(const sr_config* cfg, int32_t S, const sr_block_params8* params, const void* cond,
                         const void* h_in, void* h_out, void* scratch, size_t scratch_bytes, void* stream);

/* Operators around the calls above, for blocks put together from them (rotary positions, dropout, the residual step
 * with its norms, linear layers on 8-bit floating point).  They take their sizes directly or in structs of their own
 * (no sr_config); any size from 1 up is taken unless a call says otherwise, also odd ones. */

/* Rotary positions with several axes.  A token stands on a grid of up to three axes (time, height, width; the last one
 * runs fastest: token l = (i_0 * grid[1] + i_1) * grid[2] + i_2) and every head turns `pairs` pairs of its channels by
 *   angle(token, p) = (origin[a] + step[a] * i_a) * f_p      p = 0 .. P-1, a the axis that owns pair p,
 * in 64 bits (a far position keeps its angle); no place of the grid may turn a pair by more than 2^45 either way, where 64 bits
 * hold an angle to 2^-8 (SR_EUNSUPPORTED).  Axis 0 owns the first pairs[0] pairs, axis 1 the next, and so on;
 * P = their sum, 2 P <= head_dim.  f_p = base^(-j / pairs[a]) for the axis's j-th pair, or freqs[p].
 *   SR_ROT_HALVES: pair p is channels (p, P + p) of the head;  SR_ROT_NEIGHBOURS: channels (2 p, 2 p + 1).
 *   (c0, c1) -> (c0 cos - c1 sin, c1 cos + c0 sin), in fp32 and rounded once; channels from 2 P on are unchanged. */
typedef enum { SR_ROT_HALVES = 0, SR_ROT_NEIGHBOURS = 1 } sr_rotary_layout;
typedef struct {
  int32_t axes;                /* 1, 2 or 3 */
  int32_t grid[3], pairs[3];   /* of each axis, slowest first; grid >= 1, pairs >= 0 */
  int32_t layout;              /* sr_rotary_layout */
  double base;                 /* > 0; not read with freqs */
  double origin[3], step[3];   /* finite; origin: e.g. the time of a frame, or a window's corner */
  const double* freqs;         /* HOST array of P values, read during the call, or NULL */
} sr_rotary_cfg;

/* x -> y: `heads` heads of head_dim channels side by side in each of B*S rows; row r starts ldx (ldy) elements after
 * row r - 1, so the queries and keys in a row of q | k | v are one call with 2 H heads, in place.  Only those
 * channels are read and written.  y may be x (with ldy = ldx) and may not overlap it otherwise.
 *   idx: [B,S] int32 ([1,S] with idx_shared), the token index of each row, as sr_select_indices gives it (any order,
 *        repeats allowed; entries in [0, grid product)), or NULL: row s of a sample is token s (S <= the grid product).
 *   inverse: 1 turns by the negative angles: the gradient of x from that of y.
 * 1 <= head_dim <= 256, heads * head_dim <= 32768; ldx, ldy >= heads * head_dim.  x and y need the alignment of their elements only. */
SR_API sr_status sr_rotary(const sr_rotary_cfg* rot, int32_t inverse, int32_t dtype, int32_t B, int32_t S, int32_t heads,
                    int32_t head_dim, const void* x, int64_t ldx, const int32_t* idx, int32_t idx_shared, void* y,
                    int64_t ldy, void* stream);

/* Dropout whose mask is never stored: it is drawn anew, the same, wherever it is needed.  A value is dropped if its
 * 16 bits are below t = p * 65536 to the nearest integer, and multiplied by 65536 / (65536 - t) (fp32) otherwise: the
 * expectation is exact for every p (p = 1 drops all).  Draw e's bits are those from 16 (e % 4) up of the word
 *   mix(key + (e / 4 + 1) gamma),   key = mix(seed + (step + 1) gamma)      (SplitMix64, as in SR_SEL_RANDOM)
 *   group = 0: element (row, n) of N columns is draw (first_row + row) * N + n;
 *   group > 0: the values of a row share the draw (first_row + row) / group (1: tokens; S: samples, that is
 *              stochastic depth).
 * Calls with the same seed and step draw the same: give every dropout of a model (both branches of a block, and each block) a seed of its
 * own, kept from its forward to its backward, and count the training steps in step.
 * first_row lets the ranks or pieces of a batch draw as the whole batch would.  step_dev (a device address, 8-byte
 * aligned, or NULL) is read by the kernel and added to step, so that every replay of a captured graph can have a draw of its own. */
typedef struct {
  float p;                     /* in [0, 1]; 0: nothing is dropped */
  int32_t group;
  uint64_t seed, step, first_row;
  const uint64_t* step_dev;
} sr_drop;

/* y = resid + drop(x), x, resid (or NULL) and y [M,N] of the storage type, one rounding.  Dropped values of x do not
 * count, NaN or not.  y may be x or resid.  The gradient of x is the same call on the gradient of y with resid NULL; that
 * of resid is the gradient of y itself. */
SR_API sr_status sr_dropout(const sr_drop* drop, int32_t dtype, int32_t M, int32_t N, const void* x, const void* resid,
                     void* y, void* stream);

/* The residual step between two branches of a block, in one pass: the norm after one branch, its dropout, gate and
 * residual scale, the sum, and the norm before the next branch.  Per row of D channels of sample b:
 *   n  = post ? Norm(y) post_w + post_b : y
 *   x1 = x + gate_b res_scale drop(n)                              rounded to the stream's type
 *   u  = (Norm(x1) pre_w + pre_b) (1 + scale_b) + shift_b          rounded to the storage type
 * SR_NORM_LAYER: Norm(z) = (z - mean) / sqrt(var + eps);  SR_NORM_RMS: z / sqrt(mean z^2 + eps).  fp32 throughout; what a sample's
 * channels are multiplied with (gate, res_scale, the factor of what dropout keeps, post_w; 1 + scale, pre_w) is first multiplied together,
 * and post_b and pre_b alike, so a result has up to three roundings of 2^-24 more than step by step. */
typedef enum { SR_NORM_LAYER = 0, SR_NORM_RMS = 1 } sr_norm;
typedef struct {
  int32_t B, S, D;             /* samples (<= 2^22), rows per sample, channels (D <= 8192) */
  int32_t dtype;               /* of y, u, the parameters post_w .. pre_b and their gradients' tokens */
  int32_t stream_dtype;        /* of x, x1, dx1, dx: SR_F32, or dtype */
  int32_t norm;                /* sr_norm, of both norms */
  int32_t post;                /* 1: the branch output is normed; 0: n = y */
  float eps;
  int64_t mod_stride;          /* elements from one sample's gate (shift, scale) to the next's */
  sr_drop drop;                /* of n; rows are numbered b S + s, columns D */
} sr_residual_norm;
/* Device pointers; a NULL member is left out of the formula (a factor of one, a summand of zero). */
typedef struct {
  const void *post_w, *post_b, *res_scale, *pre_w, *pre_b;   /* [D], storage type */
  const float *gate, *shift, *scale;                         /* [B, mod_stride] rows, 4-byte aligned */
} sr_residual_norm_params;
/* fp32, OVERWRITTEN, a NULL member skips one: [D] (summed over the samples), and [B,D] for gate, shift and scale. */
typedef struct {
  float *post_w, *post_b, *res_scale, *pre_w, *pre_b, *gate, *shift, *scale;
} sr_residual_norm_grads;

/* x, y -> x1, u.  y NULL: x1 = x, not written (x1 may be NULL), the norm before a first branch.  x1 may be x.
 *   u: [B,S,D], or NULL;  uq, ue: u as the rows of sr_quantize_f8 (SR_F8_ROW) give it, straight from the fp32 values (not
 *      through the storage type), or NULL.  u, uq and ue all NULL: no norm before a next branch.
 *   stats: [4, B*S] fp32 for the backward (mean and reciprocal deviation of y, then of x1; those that the call does not
 *          compute are not written), or NULL. */
SR_API sr_status sr_residual_norm_fwd(const sr_residual_norm* cfg, const sr_residual_norm_params* params, const void* x,
                               const void* y, void* x1, void* u, uint8_t* uq, uint8_t* ue, float* stats, void* stream);

/* Its vector-Jacobian product.  x1: the forward's (x where y was NULL).  dx1: gradient of x1 by what else reads it, or NULL
 * for none; du: gradient of u, or NULL if the forward had no u (one of the two is needed).  dx (may be dx1) and dy out; dy, y NULL together.
 * Column sums run in a fixed order (deterministic).  scratch: sr_residual_norm_scratch_bytes bytes (never less for more of B, S or D, so
 * that of the largest call serves them all). */
SR_API sr_status sr_residual_norm_scratch_bytes(const sr_residual_norm* cfg, size_t* scratch_bytes);
SR_API sr_status sr_residual_norm_bwd(const sr_residual_norm* cfg, const sr_residual_norm_params* params, const void* x1,
                               const void* y, const float* stats, const void* dx1, const void* du, void* dx, void* dy,
                               const sr_residual_norm_grads* grads, void* scratch, size_t scratch_bytes, void* stream);

/* Linear layers on 8-bit floating point: codes of 4 exponent and 3 mantissa bits (e4m3: largest 448, no infinities), with
 * a power of two per block of 128 values.  A block holds 2^e, e the smallest integer in [-126, 119] with
 * max |x| <= 448 2^e, kept as the byte e + 127; a code is x 2^-e to the nearest e4m3 value, halves to the even one,
 * within +-448 (which only a block with values above 1.75 * 2^127 meets).  A floating-point code gains
 * nothing from a scale between two powers of two, and the matrix instructions apply these ones by themselves.
 * A block with an Inf or NaN has NaN codes and e = 0.
 *   SR_F8_ROW: blocks of 128 consecutive values (tokens and gradients);
 *   SR_F8_TILE: blocks of 128 x 128 (weights: one code for both directions).
 * Layout of R rows of C values: codes [R, Cp], Cp = C rounded up to 128, zeros past C; exponents [Cp / 128, Rp], Rp = R rounded up
 * to 16, one per row and block (the rows of a tile repeat it; bytes past R belong to no value). */
typedef enum { SR_F8_ROW = 0, SR_F8_TILE = 1 } sr_f8_kind;

/* x [M,N] storage type, rows ldx elements apart -> its codes and exponents as M rows of N (q, e), and those of its
 * transpose, N rows of M (qt, et; SR_F8_ROW: blocks of 128 rows of x).  Either pair may be NULL.  One pass over x.
 * M * Np, N * Mp < 2^31;  ldx >= N. */
SR_API sr_status sr_quantize_f8(int32_t f8_kind, int32_t dtype, int32_t M, int32_t N, const void* x, int64_t ldx, uint8_t* q,
                         uint8_t* e, uint8_t* qt, uint8_t* et, void* stream);

/* y[m,n] = act( sum_k x[m,k] w[n,k] + bias[n] ), x and w the values of codes (xq, xe: M rows of K; wq, we: N rows
 * of K), sums in fp32, one rounding to y's type.  (bf16 results: the matrix instructions' sums of 8-bit floating point, which
 * drop what lies 14 bits below the largest of eight products, about 1.5e-5 of the results' deviation: 1.2 % of them lie a step from the
 * rounded sum.  fp32 results: exact products and fp32 sums of them, at half the rate; of a block with e < -124 the values to the
 * nearest multiple of 2^-133, halves to the even one.)  GELU is of the fp32 sum.  How sums are grouped follows M, N and K.  The
 * three products of a linear layer y = x w^T are
 *   (M, N, K) on x and w;   dx: (M, K, N) on dy and the transposed codes of w;
 *   dw: (N, K, M), SR_F32, on the transposed codes of dy and of x.
 *   dtype: of bias (or NULL) and y [M,N];  act: sr_act.
 *   scratch: sr_linear_f8_scratch_bytes bytes (NULL when 0; never less for more of M, N or K, so that of the largest call serves them
 *     all), for the partial sums of long rows with few results.
 * M, N >= 1; 1 <= K <= 2^24; M*Kp, N*Kp and M*N*elt < 2^31 bytes (Kp: K rounded up to 128). */
SR_API sr_status sr_linear_f8_scratch_bytes(int32_t M, int32_t N, int32_t K, size_t* scratch_bytes);
SR_API sr_status sr_linear_f8(int32_t dtype, int32_t act, int32_t M, int32_t N, int32_t K, const uint8_t* xq, const uint8_t* xe,
                       const uint8_t* wq, const uint8_t* we, const void* bias, void* y, void* scratch,
                       size_t scratch_bytes, void* stream);

/* Launch timing for measurement (not needed by the method).  After
 * sr_profile_start, every library launch group whose name contains `name_filter`
 * ("" or NULL = all) is timed with HIP events bound to its first and last kernel at launch
 * (hipExtLaunchKernelGGL), so a group's time is its kernels' own execution.  With no filter the
 * backward issues its weight-gradient GEMMs on the caller's stream (they normally run on
 * a second stream of the library, overlapping the rest), so each group is timed alone;
 * with a filter the overlap stays and the named groups are timed as they run.
 * sr_profile_stop waits for those events, stops recording and writes one line per
 * name: "<name> <launches> <total_ms> <algorithmic_flops> <algorithmic_bytes>\n"
 * into `out` (NUL-terminated, truncated to out_bytes); *needed receives the full
 * size.  Names: select_random, select_topk, select_topk_scores, attn_colsum, xattn_fwd,
 * xattn_bwd, gather,
 * scatter_delta, gather_f32, scatter_f32, ln_fwd, ln_bwd,
 * gemm_<op> (qkv, o, fc1, fc2, dx_fc2, dx_fc1, dx_o, dx_qkv, dw_<op>), attn_fwd,
 * attn_bwd_dkv, attn_bwd_dq, attn_bwd_f32 (both passes of fp32 storage), attn_bwd_delta, reduce,
 * colsum, convert, mod, quantize8, dequantize8, linear8, weight_grad8,
 * ln_quant, rotary, dropout, residual_norm_fwd, residual_norm_bwd, quantize_f8, linear_f8.  Where few workgroups make dK/dV and dQ one launch (bf16, head dim 64),
 * attn_bwd_dkv holds both passes. */
SR_API sr_status sr_profile_start(const char* name_filter);
SR_API sr_status sr_profile_stop(char* out, size_t out_bytes, size_t* needed);

/* Sustained bf16 matrix-core rate of the current device, for the denominator of a
 * measured roofline (not needed by the method).  Runs two launches of a register-only
 * kernel (one workgroup of eight waves per compute unit, independent 32x32x16 bf16 MFMAs,
 * no memory traffic in its loop; the first launch only lets the clock settle) on
 * `stream`, times the second with HIP events and waits for it.
 *   sink: device pointer to at least 4 writable bytes (the kernel stores one float there).
 *   tflops: host pointer; receives the achieved dense bf16 TFLOP/s (the datasheet peak is
 *   2500 at 2.4 GHz; the sustained rate reflects the clock under matrix load).
 * Errors: SR_EINVAL for a NULL argument, SR_EHIP if a launch or event call fails. */
SR_API sr_status sr_probe_mfma_rate(float* sink, double* tflops, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SR_H */
