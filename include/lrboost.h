/* lrboost -- C ABI of the low-rank bottleneck decoder-block hot path for one MI355X (gfx950).
 *
 * A linear map W[d_out, d_in] is replaced by  y = W_up . sigma(W_down . x)  with a rank-r
 * bottleneck (paper Sec. 2, "Low-Rank Matrix Factorization" / "Low-Rank Activation via
 * Auto-Encoder"; sigma = identity is the SVD variant of App. "Low-rank Training Algorithm").
 *
 * Conventions common to every entry point
 *  - Every pointer is a DEVICE pointer owned by the caller unless a comment says "host".  The
 *    library never allocates, frees or synchronises: each call validates its arguments on the
 *    host, enqueues kernels on `stream` (a hipStream_t passed as void*, NULL = default
 *    stream) and returns.  A large product keeps every CU until its launch ends (up to 0.5 ms at
 *    16384 tokens): what another stream enqueues meanwhile waits for that.  Scratch memory comes
 *    from the caller through (ws, ws_bytes); the matching *_workspace_bytes() call gives the size to
 *    hand over.  That may be more than the call needs, and a workspace without what is on top is
 *    accepted too, with the same results, slower: for the backward of narrow layers up to 32 MiB
 *    (room for the weight gradients' partial sums side by side, so that they share launches), for a
 *    block, forward or backward, up to a 64th of its d_ff wide activations (their rows then start
 *    on cache lines).  The queries count dense rows: a backward over x or dy whose rows span
 *    2 GiB or more in all (T * ld * 2 bytes) needs copies of them on top and returns LR_EWORKSPACE
 *    without the room.
 *  - Matrices are row-major, activations token-major: x[T, d] with leading dimension ld (in
 *    elements).  Weights use the [out, in] layout: W_down[r, d_in], W_up[d_out, r], dense.
 *  - dt selects the storage type of activations, weights and gradients (LR_F32 or LR_BF16);
 *    accumulation is always fp32.  Per-token statistics are fp32 in either case.
 *  - LR_BF16 requires d_in, r, d_out and every leading dimension to be multiples of 8 and
 *    every pointer 16-byte aligned (LR_EALIGN otherwise).  T is arbitrary.
 *  - Return value: LR_OK or a negative lr_status.  Argument, alignment, workspace and
 *    "unsupported" errors (everything but LR_ELAUNCH) are detected on the host before any launch,
 *    so such a failed call has enqueued nothing.  LR_ELAUNCH reports that the runtime rejected a
 *    kernel launch midway through a call's sequence: the kernels before it have been enqueued and
 *    the outputs are then unspecified.  Faults inside kernels surface at the caller's next
 *    synchronisation.  Outputs must not alias inputs.
 *  - Weight and gamma gradients are written in grad_dt: LR_F32 (fp32 main-gradient buffers, the
 *    usual companion of bf16 weights; always the case when dt == LR_F32) or LR_BF16 (pure bf16,
 *    App. "Low-rank Training Algorithm", costs one more rounding).  accumulate != 0 adds them
 *    into the given buffers instead of overwriting.  Activation gradients (dx) use dt.
 */
#ifndef LRBOOST_H
#define LRBOOST_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LR_OK = 0,
  LR_EINVAL = -1,       /* null pointer, non-positive size, unknown enum value            */
  LR_EUNSUPPORTED = -2, /* valid request the library cannot run (e.g. fp32 block)         */
  LR_EWORKSPACE = -3,   /* ws is NULL or ws_bytes is smaller than the call needs          */
  LR_EALIGN = -4,       /* pointer / leading-dimension / size alignment rule violated     */
  LR_ELAUNCH = -5       /* a kernel launch was rejected by the runtime                    */
} lr_status;

typedef enum { LR_F32 = 0, LR_BF16 = 1 } lr_dtype;
typedef enum { LR_ACT_IDENTITY = 0, LR_ACT_SILU = 1 } lr_act;
/* LR_NORM_ONLINE: RMSNorm folded into the down-projection GEMM (sum of squares gathered
 * inside a GEMM, 1/rms applied as a per-row scale in the epilogue; single-GPU form of the
 * paper's Alg. 1).  LR_NORM_TWO_PASS: the unfused twin (statistic pass, normalise pass,
 * plain GEMM), i.e. what Alg. 1 falls back to (Sec. 4.5 "Configuration").               */
/* LR_NORM_ONLINE takes the sum of squares from the A tiles inside the down-projection while the
 * output is at most 512 columns wide and from one pass over x (Alg. 1, its first step) beyond
 * that, where the pass is the faster of the two.  LR_NORM_ONLINE_GATHER is the same computation
 * with the in-GEMM gather at every width (bf16; fp32 storage takes the pass): no pass over x at
 * all, at the price of every column tile repeating the gather.  Same outputs, same backward.  */
/* LR_NORM_SHARD_LOCAL (lr_group_fwd only): one tensor-parallel rank's part of Alg. 1, the steps
 * before the exchange.  x[T, d_in] is the rank's slice of the features (d_in = d / TP), gamma its
 * slice of the scale, w_down_cat[G*r, d_in] the matching columns of the weights.  The rank takes its
 * local sum of squares, normalises its slice by its LOCAL rms, multiplies by its weight slice and
 * undoes the local scale on the product: z_cat[T, G*r] receives that un-normalised partial product
 * (to be summed over the ranks), stat[T] the local sum of squares (summed with it).  sigma, the
 * up-projections and y come after the exchange: act, w_up_stack, y_stack, ldy, y_batch_stride and
 * d_out are ignored (pass NULL / 0 / any positive d_out).  lr_online_rmsnorm_finish applies the
 * global rescale to the summed product.  No backward form.                                  */
typedef enum { LR_NORM_NONE = 0, LR_NORM_TWO_PASS = 1, LR_NORM_ONLINE = 2, LR_NORM_SHARD_LOCAL = 3,
               LR_NORM_ONLINE_GATHER = 4 } lr_norm;

int lr_version(void);
/* Human-readable name of a status code; static storage, never freed. */
const char* lr_status_string(int status);

/* ---- one bottleneck layer (Sec. 2: B sigma(A x)) ------------------------------------- */
/* y[T, d_out] = W_up . act(W_down . x);  z[T, r] (dense) receives the rank-r pre-activation,
 * the only tensor the backward needs besides x (Sec. 4.4).                                */
size_t lr_linear_workspace_bytes(int64_t T, int64_t d_in, int64_t r, int64_t d_out, int dt,
                                 int backward);
int lr_linear_fwd(const void* x, int64_t ldx, const void* w_down, const void* w_up, void* z,
                  void* y, int64_t ldy, int64_t T, int64_t d_in, int64_t r, int64_t d_out,
                  int act, int dt, void* ws, size_t ws_bytes, void* stream);
/* From x, z and dy[T, d_out]: dx[T, d_in], dw_down[r, d_in], dw_up[d_out, r].              */
int lr_linear_bwd(const void* x, int64_t ldx, const void* w_down, const void* w_up,
                  const void* z, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                  void* dw_down, void* dw_up, int64_t T, int64_t d_in, int64_t r,
                  int64_t d_out, int act, int dt, int grad_dt, int accumulate, void* ws,
                  size_t ws_bytes, void* stream);

/* lr_linear_fwd for callers that cannot allocate device memory or hand over a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, results and
 * error codes as lr_linear_fwd without (ws, ws_bytes): the rank-r activation between the two GEMMs is
 * kept in a device array that is part of the library image (LR_LINEAR_STATIC_SCRATCH_BYTES per GPU, held
 * from the moment the library is loaded on that GPU until the process ends).  The call allocates and
 * frees nothing.  Limit: T * r * (2 for LR_BF16, 4 for LR_F32) bytes must fit the array, otherwise
 * LR_EWORKSPACE and nothing is enqueued.  All calls on one GPU share the array: calls that may run
 * concurrently on one GPU (different streams, different host threads) race on it and must be serialised
 * by the caller.  Nothing in it needs clearing between calls (every element a call reads, it has
 * written).  The first call on a device looks up the array's address, which is a set-up step: make it
 * before a stream capture begins, not inside one.                                                    */
#define LR_LINEAR_STATIC_SCRATCH_BYTES (32u << 20)
int lr_linear_fwd_static(const void* x, int64_t ldx, const void* w_down, const void* w_up, void* z,
                         void* y, int64_t ldy, int64_t T, int64_t d_in, int64_t r, int64_t d_out,
                         int act, int dt, void* stream);

/* ---- G projections sharing one input (Sec. 4.3 and App. "Linear Grouping Details") ---- */
/* w_down_cat[G*r, d_in]: the G down-projection weights concatenated along the rank axis (one
 * GEMM); w_up_stack[G, d_out, r]: stacked up-projection weights (one batched GEMM over the
 * (input, weight) pairs).  Optional RMSNorm of x (Eq. 4; gamma[d_in], eps inside the root):
 *   z_cat[T, G*r] = RMSNorm(x) . w_down_cat^T     (dense, the rank-r checkpoint)
 *   y_g[T, d_out] = act(z_g) . w_up_g^T           at y_stack + g*y_batch_stride, ld = ldy
 *   stat[T] (fp32) = sum_j x[t,j]^2               (written when norm != LR_NORM_NONE)
 * gamma and stat may be NULL when norm == LR_NORM_NONE.                                     */
size_t lr_group_workspace_bytes(int G, int64_t T, int64_t d_in, int64_t r, int64_t d_out,
                                int dt, int backward);
int lr_group_fwd(const void* x, int64_t ldx, const void* gamma, float eps, int norm,
                 const void* w_down_cat, const void* w_up_stack, void* z_cat, float* stat,
                 void* y_stack, int64_t ldy, int64_t y_batch_stride, int G, int64_t T,
                 int64_t d_in, int64_t r, int64_t d_out, int act, int dt, void* ws,
                 size_t ws_bytes, void* stream);
/* dx[T, d_in] is the gradient w.r.t. the un-normalised x; dgamma[d_in] (grad_dt; ignored when
 * norm == LR_NORM_NONE).  stat is the forward's output.                                     */
int lr_group_bwd(const void* x, int64_t ldx, const void* gamma, float eps, int norm,
                 const void* w_down_cat, const void* w_up_stack, const void* z_cat,
                 const float* stat, const void* dy_stack, int64_t lddy,
                 int64_t dy_batch_stride, void* dx, int64_t lddx, void* dgamma,
                 void* dw_down_cat, void* dw_up_stack, int G, int64_t T, int64_t d_in,
                 int64_t r, int64_t d_out, int act, int dt, int grad_dt, int accumulate,
                 void* ws, size_t ws_bytes, void* stream);

/* ---- the decoder block ------------------------------------------------------------------
 * RMSNorm -> grouped low-rank Q/K/V -> causal attention -> low-rank O + residual -> RMSNorm
 * -> grouped low-rank gate/up -> SiLU(g)*u -> low-rank down + residual.  Seven factored
 * projections (App. "Communication volume analysis": 11dr + 3 d_ff r parameters).  Only the
 * rank-r pre-activations are kept for the backward, which re-forwards everything wider from
 * them and from x (Sec. 4.4).                                                              */
typedef struct {
  int64_t batch, seq, d_model, n_heads, head_dim;
  int64_t ffn;     /* logical MLP width                                                    */
  int64_t ffn_ld;  /* padded MLP width, multiple of 8, >= ffn; the pad rows/columns of the
                      ffn-sized weights must be zero (then their gradients stay zero)      */
  int64_t rank;
  float eps;
  int act;         /* lr_act at rank r                                                     */
  int norm;        /* LR_NORM_ONLINE, LR_NORM_ONLINE_GATHER or LR_NORM_TWO_PASS            */
  int dt;          /* LR_BF16                                                              */
  int grad_dt;     /* dtype of the weight / gamma gradient buffers: LR_F32 or LR_BF16      */
  int causal;      /* 1                                                                    */
  /* Optional rotary position embedding of q and k (LLaMA-style models, Sec. 5.2), applied
   * between the up-projections and the attention in the forward and in the re-forward, and
   * transposed on dq, dk in the backward.  DEVICE pointers to cos / sin tables [seq, 64] fp32
   * (16-byte aligned) of the angles of lr_rope below; both NULL: no rotary embedding.       */
  const float* rope_cos;
  const float* rope_sin;
  /* Chaining the norm statistic through a stack of blocks (Sec. 4.2: the sum of squares travels
   * with the GEMM that produces the normalised tensor).  stat_y_out, if not NULL: DEVICE [T] fp32,
   * receives sum_j y[t,j]^2, accumulated from the fp32 output tiles in the epilogue of the block's
   * last GEMM; it is the s1 of the block above.  stat_x_ready != 0: ckpt->s1 already holds
   * sum_j x[t,j]^2 (the stat_y_out of the block below) and the forward takes it as given instead
   * of computing it from x.                                                                    */
  int stat_x_ready;
  float* stat_y_out;
  /* Grouped-query attention (section "Discussion and Future Work": only the shapes of the K and V
   * projections change).  0 or n_heads: multi-head.  Otherwise a divisor of n_heads: the K and V
   * up-projections are [n_kv_heads * head_dim, rank], and w_up_qkv (and its gradient) is packed:
   * W_up,q [d_model, rank], then W_up,k, then W_up,v.  Everything else keeps its shape.          */
  int64_t n_kv_heads;
} lr_block_desc;

typedef struct {
  void* gamma1;    /* [d]                                                                  */
  void* w_dn_qkv;  /* [3r, d]   q, k, v concatenated along the rank axis                   */
  void* w_up_qkv;  /* [3, d, r]  (n_kv_heads < n_heads: [d + 2 n_kv_heads head_dim, r])     */
  void* w_dn_o;    /* [r, d]                                                               */
  void* w_up_o;    /* [d, r]                                                               */
  void* gamma2;    /* [d]                                                                  */
  void* w_dn_gu;   /* [2r, d]   gate, up concatenated                                      */
  void* w_up_gu;   /* [2, ffn_ld, r]                                                       */
  void* w_dn_d;    /* [r, ffn_ld]                                                          */
  void* w_up_d;    /* [d, r]                                                               */
} lr_block_params;  /* the same struct, pointing at grad_dt buffers, receives the grads    */

typedef struct {
  void* z_qkv;     /* [T, 3r]                                                              */
  void* z_o;       /* [T, r]                                                               */
  void* z_gu;      /* [T, 2r]                                                              */
  void* z_d;       /* [T, r]                                                               */
  float* s1;       /* [T] sum of squares of x                                              */
  float* s2;       /* [T] sum of squares of h1 = x + attention branch                      */
} lr_block_ckpt;    /* rank-r checkpoints, written by fwd, read by bwd; caller-allocated    */

/* 0 when the descriptor is invalid or unsupported. */
size_t lr_block_workspace_bytes(const lr_block_desc* desc, int backward);
/* Bytes of all six checkpoint buffers together (information only; the caller allocates
 * each buffer of lr_block_ckpt separately, with the shapes given above).                  */
size_t lr_block_ckpt_bytes(const lr_block_desc* desc);
/* desc, params, ckpt are HOST structs holding device pointers.  x, y: [T, d], dense.      */
int lr_block_fwd(const lr_block_desc* desc, const lr_block_params* params, const void* x,
                 void* y, const lr_block_ckpt* ckpt, void* ws, size_t ws_bytes, void* stream);
/* x must be unchanged since the forward.  dy, dx: [T, d] dense.                           */
int lr_block_bwd(const lr_block_desc* desc, const lr_block_params* params, const void* x,
                 const void* dy, const lr_block_ckpt* ckpt, void* dx,
                 const lr_block_params* grads, int accumulate, void* ws, size_t ws_bytes,
                 void* stream);

/* ---- the block with every wide activation kept ---------------------------------------------
 * The reference point of the checkpointing comparison (Sec. 4.4, Table 5: memory saved against time
 * added by keeping only rank-r activations): lr_block_fwd_save also leaves every d-wide and ffn-wide
 * activation of the forward in caller-owned buffers, and lr_block_bwd_saved reads them instead of
 * re-forwarding from the rank-r checkpoints (which it still takes: sigma and sigma' are rebuilt from z at
 * rank r).  Results equal those of lr_block_fwd / lr_block_bwd bit for bit (recomputed = stored).  Dense
 * bf16 unless noted; the backward only reads them:
 *   qkv  q [T, d], then k [T, d_kv], then v [T, d_kv], back to back (after the rotary embedding, if any)
 *   o    [T, d]        lse  [batch, n_heads, seq] fp32        h1  [T, d]
 *   gu   g [T, ffn_ld], then u [T, ffn_ld]                    m   [T, ffn_ld]
 * 2.4 GB at the 7B shape (batch 4 x seq 4096) against 0.24 GB of rank-r checkpoints.                 */
typedef struct {
  void *qkv, *o;
  float* lse;
  void *h1, *gu, *m;
} lr_block_saved;
size_t lr_block_saved_workspace_bytes(const lr_block_desc* desc, int backward);
int lr_block_fwd_save(const lr_block_desc* desc, const lr_block_params* params, const void* x,
                      void* y, const lr_block_ckpt* ckpt, const lr_block_saved* saved, void* ws,
                      size_t ws_bytes, void* stream);
int lr_block_bwd_saved(const lr_block_desc* desc, const lr_block_params* params, const void* x,
                       const void* dy, const lr_block_ckpt* ckpt, const lr_block_saved* saved,
                       void* dx, const lr_block_params* grads, int accumulate, void* ws,
                       size_t ws_bytes, void* stream);

/* ---- the LaX variant of the block (App. "LaX variant (residual low-rank)") ----------------
 * Identity gate at rank r, and every bottleneck layer adds the rank-r activation h_{i-1} of the
 * same projection in the decoder layer below before its up-projection: y_i = B_i (h_i + h_{i-1}),
 * h_i = A_i x_i.  A block's own h_i are its checkpoints z_* (lr_block_ckpt), which the caller
 * hands to the block above as h_prev_*.  In the backward, dz_next_* is the block above's
 * gradient w.r.t. this block's z_* (its dh_prev_*), and dh_prev_* receives this block's gradient
 * w.r.t. its h_prev_*.  Layouts as the checkpoints: qkv [T, 3r], o [T, r], gu [T, 2r], d [T, r],
 * bf16, dense.  Each pointer may be NULL: an absent h_prev / dz_next counts as zeros (first /
 * last block of a stack), an absent dh_prev is not written.  desc->act must be
 * LR_ACT_IDENTITY (else LR_EUNSUPPORTED); everything else as lr_block_fwd / lr_block_bwd
 * (grouped key / value heads included), same workspace sizes.                               */
typedef struct {
  const void *h_prev_qkv, *h_prev_o, *h_prev_gu, *h_prev_d;       /* forward and backward inputs  */
  const void *dz_next_qkv, *dz_next_o, *dz_next_gu, *dz_next_d;   /* backward inputs              */
  void *dh_prev_qkv, *dh_prev_o, *dh_prev_gu, *dh_prev_d;         /* backward outputs             */
} lr_block_lax;
int lr_block_lax_fwd(const lr_block_desc* desc, const lr_block_params* params, const void* x,
                     void* y, const lr_block_ckpt* ckpt, const lr_block_lax* lax, void* ws,
                     size_t ws_bytes, void* stream);
int lr_block_lax_bwd(const lr_block_desc* desc, const lr_block_params* params, const void* x,
                     const void* dy, const lr_block_ckpt* ckpt, void* dx,
                     const lr_block_params* grads, int accumulate, const lr_block_lax* lax,
                     void* ws, size_t ws_bytes, void* stream);

/* ---- rotary position embedding (optional step of the block; the paper does not describe
 * it, LLaMA-style attention has it) -------------------------------------------------------
 * In place on x[B*S, ldx] (bf16, H heads of hd = 128 from column 0): inside every head the pair
 * (v[i], v[i + 64]), i < 64, of the token at position p of its sequence becomes
 * (v[i] c - v[i+64] s, v[i+64] c + v[i] s) with c = cos_tab[p, i], s = sin_tab[p, i]
 * (DEVICE tables [S, 64] fp32).  inverse != 0 uses -s: the transpose of the rotation, which
 * is its backward.  Other dtypes / head sizes: LR_EUNSUPPORTED.                             */
int lr_rope(void* x, int64_t ldx, const float* cos_tab, const float* sin_tab, int64_t B,
            int64_t S, int64_t H, int64_t hd, int inverse, int dt, void* stream);

/* ---- causal multi-head attention (the sharded-safe op between the chunks, Sec. 4.2) ---- */
/* q, k, v, o: [B*S, H*hd] token-major, head h in columns h*hd..; lse[B, H, S] fp32.
 * bf16 only, hd = 128, and S * ld * 2 < 2^31 bytes (the kernels address one batch element with
 * 32-bit buffer offsets); otherwise LR_EUNSUPPORTED.  The backward workspace holds two [B, H, S]
 * fp32 arrays (sum_h dO*O and lse * log2(e)) and, where S is a multiple of 8, room for the score
 * gradient scale * dS^T as bf16 [B, H, S, S].  Where the work leaves CUs idle the key / value gradient
 * kernel writes it and the query gradient is one GEMM over it; where there is work for the whole chip,
 * S is not a multiple of 8 or the room would be over 24 GiB, it is formed a second time instead.  The
 * same bits either way.  The room is that of the calls of H heads on up to B * S tokens in sequences
 * of up to S that store it (0.5 GB at B 4, H 4, S 4096; 3.4 GB at B 4, H 32, S 4096, for B 5, S 3272). */
int lr_attention_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                     int64_t ld, int64_t B, int64_t S, int64_t H, int64_t hd, int causal,
                     int dt, void* stream);
size_t lr_attention_bwd_workspace_bytes(int64_t B, int64_t S, int64_t H, int64_t hd);
int lr_attention_bwd(const void* q, const void* k, const void* v, const void* o,
                     const void* dout, const float* lse, void* dq, void* dk, void* dv,
                     int64_t ld, int64_t B, int64_t S, int64_t H, int64_t hd, int causal,
                     int dt, void* ws, size_t ws_bytes, void* stream);

/* Grouped-query form (the extension named in the section "Discussion and Future Work": only the
 * shapes of the K and V projections change).  Hkv key / value heads, H % Hkv == 0; query head h
 * attends over key / value head h / (H / Hkv).  q, o, dout, dq: [B*S, ld] with H heads of hd columns;
 * k, v, dk, dv: [B*S, ldkv] with Hkv heads; lse [B, H, S].  dk and dv are the sums over the query
 * heads of each group.  Same restrictions and error behaviour as the multi-head calls, which are the
 * case Hkv = H, ldkv = ld; for Hkv < H the backward workspace additionally holds one dK and one dV
 * contribution per query head (2 * B*S*H*hd bf16), added up by a last kernel.               */
int lr_attention_gqa_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                         int64_t ld, int64_t ldkv, int64_t B, int64_t S, int64_t H, int64_t Hkv,
                         int64_t hd, int causal, int dt, void* stream);
size_t lr_attention_gqa_bwd_workspace_bytes(int64_t B, int64_t S, int64_t H, int64_t Hkv,
                                            int64_t hd);
int lr_attention_gqa_bwd(const void* q, const void* k, const void* v, const void* o,
                         const void* dout, const float* lse, void* dq, void* dk, void* dv,
                         int64_t ld, int64_t ldkv, int64_t B, int64_t S, int64_t H, int64_t Hkv,
                         int64_t hd, int causal, int dt, void* ws, size_t ws_bytes, void* stream);

/* ---- rotary tables and rotation at given positions ----------------------------------------- */
/* cos_tab, sin_tab[n, rot / 2] (fp32): mscale * cos, mscale * sin of (first + p) * w_i, p < n, with the frequencies
 * w_i = base^(-2 i / rot) scaled for contexts longer than the one trained on: context = 0 divides all of them by `factor`
 * (1: none); context > 0 goes by t_i = context * w_i / (2 pi), the turns over the trained context: a frequency of t_i <= low is divided
 * by factor, one of t_i >= high is kept, linearly in between.  Angles are formed in 64 bits, each entry is rounded once.
 * rot even, at most 8192 (else LR_EUNSUPPORTED); first >= 0, first + n <= 2^31; base > 0, factor > 0, mscale finite, low < high.  A base or
 * factor below 1 makes angles larger than the positions: above 2^31, LR_EUNSUPPORTED.
 * The tables serve lr_rope_at and lr_kv_append, and with rot = 128 lr_rope and the block (rope_cos, rope_sin).                 */
int lr_rope_table(float* cos_tab, float* sin_tab, int64_t n, int64_t rot, int64_t first, double base, double factor,
                  double context, double low, double high, double mscale, void* stream);
/* out[T, ldo] = x[T, ldx] (H heads of hd columns from column 0) with the first rot columns of every head rotated by row pos[t] (DEVICE
 * int32; NULL: t, T <= table_rows) of the tables [table_rows, rot / 2]: pairs (i, i + rot / 2), or (2i, 2i + 1) where interleaved != 0, become
 * (a c - b s, b c + a s).  inverse != 0 uses -s: the transpose, which is its gradient.  Columns rot.. of a head are copied; a row of
 * out whose position is outside the tables is left as it was, and so are columns past the heads.  out may be x with ldo = ldx (in
 * place); any other overlap is not allowed.  LR_BF16: hd and the strides multiples of 8, rot of 16, all pointers 16-byte aligned but
 * pos; LR_F32: rot even.  rot <= hd.  T may be 0, and is at most 2^24; LR_EUNSUPPORTED above 2^32 lanes (units of 16 bytes, of a pair where
 * fp32 rows do not start on 16 bytes).                                                                                         */
int lr_rope_at(const void* x, int64_t ldx, void* out, int64_t ldo, const int32_t* pos, const float* cos_tab,
               const float* sin_tab, int64_t table_rows, int64_t T, int64_t H, int64_t hd, int64_t rot, int interleaved,
               int inverse, int dt, void* stream);

/* ---- a paged key / value cache ------------------------------------------------------------- */
/* Keys and values of `batch` sequences (bf16), in pages of page_size tokens that a sequence collects in any order: key j of sequence b
 * lies in page page_table[b, j / page_size], row j % page_size.  Token t of a call belongs to the sequence b with
 * cu_q[b] <= t < cu_q[b + 1]; kv_len[b] counts b's keys including the new ones, so that its new tokens stand at positions
 * kv_len[b] - (cu_q[b + 1] - cu_q[b]) and up.  The lists are DEVICE int32 and not read on the host: a captured call takes what they
 * hold when it is replayed.  Tokens before cu_q[0] or from cu_q[batch] on belong to nobody (a padded batch): nothing is written for
 * them.  The lists may count more tokens than the call has: those it has keep their positions.  Whatever the lists hold, nothing outside the cache and the other arguments is read or written: a page number
 * outside [0, n_pages) is no page, keys past max_pages * page_size do not exist.
 * page_size, head_dim and the strides (elements) are multiples of 8, k and v 16-byte aligned (LR_EALIGN); pages of both layouts
 * [page_size, n_kv_heads, head_dim] and [n_kv_heads, page_size, head_dim] are a matter of the strides.  Limits (LR_EUNSUPPORTED):
 * 2^35 elements from the first to the last of k, 2^31 - 2048 keys of a sequence, 2^16 sequences and 2^25 tokens of a call, token_stride < 2^26.  */
typedef struct {
  void *k, *v;
  int64_t n_pages, page_size, n_kv_heads, head_dim;
  int64_t page_stride, token_stride, head_stride;
  const int32_t* page_table;   /* [batch, table_ld], max_pages columns of it */
  int64_t batch, max_pages, table_ld;
  const int32_t* cu_q;         /* [batch + 1] */
  const int32_t* kv_len;       /* [batch] */
} lr_kv_cache;                 /* a HOST struct */

/* Writes the keys k[T, ldk] and values v[T, ldv] (n_kv_heads heads of head_dim columns) of the new tokens into their pages.  With tables
 * (cos_tab, sin_tab, rot > 0: as lr_rope_at) keys are rotated by their position on the way; NULL tables with rot = 0: as they are.
 * q (NULL: none; H heads, [T, ldq]) is rotated likewise into q_out[T, ldqo], which may be q with the same stride.  A token without a
 * place (no page, no position below kv_len, no row in the tables) is left out: its row of q_out stays as it was.  Two tokens with one
 * place (a page in two rows of page_table): either one's, or a mixture.  dt: LR_BF16.                                          */
int lr_kv_append(const lr_kv_cache* cache, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q,
                 int64_t ldq, void* q_out, int64_t ldqo, int64_t T, int64_t H, const float* cos_tab, const float* sin_tab,
                 int64_t table_rows, int64_t rot, int interleaved, int dt, void* stream);

/* Causal attention of the new tokens over the cache, which holds their own keys and values already: o[T, ldo] (H heads) =
 * softmax(scale * q . k) . v over the keys at positions up to the token's own, query head h on key / value head
 * h / (H / n_kv_heads); lse[T, H] (fp32, NULL: not written) = log of the softmax's sum.  Any mixture of long and single-token sequences.
 * A token that sees no key, or only keys whose logits are -infinity, has o = 0 and lse = -infinity; a page number that is no page holds zeros.  H % n_kv_heads == 0, scale > 0,
 * scale * log2(e) finite.  Logits scale * q . k are formed in 32 bits and below 2^26 in magnitude (where neighbours are 4 apart): far above, a row may come
 * out as zeros or NaN.
 * dt LR_BF16, head_dim 128, causal 1, otherwise LR_EUNSUPPORTED.  The workspace holds the parts of sequences whose keys are split over workgroups;
 * its size depends on T, H and the cache's sizes, not on the lists.  o overlaps nothing that is read.  LR_EUNSUPPORTED also where T * H passes
 * 2^31 - 1, or the sequences' heads and rows (n_kv_heads of each sequence that can have a token, and one for every 128 of T * H) 2^24 - 2^12.  */
size_t lr_attention_paged_workspace_bytes(const lr_kv_cache* cache, int64_t T, int64_t H);
int lr_attention_paged_fwd(const lr_kv_cache* cache, const void* q, int64_t ldq, void* o, int64_t ldo, float* lse,
                           int64_t T, int64_t H, float scale, int causal, int dt, void* ws, size_t ws_bytes, void* stream);

/* ---- who holds the pages ------------------------------------------------------------------------ */
/* refs[n_pages] (DEVICE int32) counts the holders of every page: the entries of page tables that name it, and whoever else is to keep it (a
 * prompt's beginning that is held for later).  Pages of count 0 are free.  lr_kv_fork and lr_kv_compact read lists and write new ones (no output
 * overlaps an input), so the caller keeps the old state until the new one is accepted.  All lists are DEVICE int32 and not read on the host; entries
 * outside [0, n_pages) are no page.  The same lists give the same result.
 *
 * lr_kv_fork makes the page tables of n_out sequences from those of n_in: new sequence i goes on with the len_in[p] keys of p = parent[i] (outside
 * [0, n_in): a sequence without keys) and has room for grow[i] new ones (below 0: 0), len_out[i] = len_in[p] + grow[i] (at most 2^31 - 1): the kv_len
 * of lr_kv_append.  An old sequence that is nobody's parent ends.  Pages that its keys fill are shared by all children.  The half filled page
 * stays with the first child where refs is 1; any other child takes a fresh page, to which lr_kv_copy has to bring copy_rows[i] tokens of
 * copy_src[i] (copy_dst[i] the fresh page; -1, -1, 0: no copy) before new keys are appended.  The first child also keeps the pages behind.  A column that new
 * keys reach and that has no page yet takes a fresh one: the lowest free ones (refs 0 at the call: pages that it frees are free for the next), given to the
 * sequences in order.  Where there are too few, or no column is left, entries are -1 and missing[0] counts the pages that are missing.  refs_out follows all
 * entries of the old and new tables.  Up to 2^14 old and new sequences, 2^26 pages (LR_EUNSUPPORTED).                                 */
size_t lr_kv_fork_workspace_bytes(int64_t n_pages, int64_t n_in, int64_t n_out);
int lr_kv_fork(const int32_t* refs_in, int64_t n_pages, int64_t page_size, const int32_t* table_in, int64_t ld_in, const int32_t* len_in,
               int64_t n_in, const int32_t* parent, const int32_t* grow, int32_t* refs_out, int32_t* table_out, int64_t ld_out,
               int32_t* len_out, int64_t n_out, int64_t max_pages, int32_t* copy_src, int32_t* copy_dst, int32_t* copy_rows,
               int32_t* missing, void* ws, size_t ws_bytes, void* stream);
/* Moves the held pages (refs above 0) together: with H of them, page_map[n_pages] gives every held page its new number below H (-1: free), the table
 * [batch, max_pages] and refs follow it, n_live[0] = H.  The held pages from H on move, in order, into the free ones below, in order: copy_src and
 * copy_dst [n_pages / 2] list them for lr_kv_copy, -1 behind the last.                                                                 */
size_t lr_kv_compact_workspace_bytes(int64_t n_pages);
int lr_kv_compact(const int32_t* refs_in, int64_t n_pages, const int32_t* table_in, int64_t ld_in, int64_t batch, int64_t max_pages, int32_t* refs_out,
                  int32_t* table_out, int64_t ld_out, int32_t* copy_src, int32_t* copy_dst, int32_t* page_map, int32_t* n_live, void* ws,
                  size_t ws_bytes, void* stream);
/* Copies, for i < n, the first rows[i] tokens (NULL: all; taken as at least 0 and at most page_size) of page src[i] onto page dst[i], keys and values of
 * all heads.  Entries with no page in src or dst are passed over.  A page that is written is in no other entry.  Of `cache` only the pages and their
 * strides count (the lists may be NULL, batch 0).  Once for each layer whose cache the page tables describe.  At most 2^31 - 2^12 vectors of eight
 * elements in a page's keys (LR_EUNSUPPORTED).                                                                                       */
int lr_kv_copy(const lr_kv_cache* cache, const int32_t* src, const int32_t* dst, const int32_t* rows, int64_t n, void* stream);

/* ---- which sequences go on ---------------------------------------------------------------------- */
/* Beam search's choice: for each of `batch` prompts the n candidates (beam w, token v) of highest
 *   score[b, w] + logits[b * beams + w, v] - log sum_u exp(logits[b * beams + w, u])
 * in falling order, formed in 64 bits; equal ones by beam.  A beam's own are in the order of their logits, also where those are too close for 64-bit scores to
 * differ, equal logits by token: the first candidates are the same for every n.  (The order in which a sum is added up depends on batch * beams, so a prompt's scores may differ by
 * last places of 64 bits with the prompts beside it.)  logits [batch * beams, ldl] (dt), V tokens; parent [batch, n] receives the
 * row b * beams + w (what lr_kv_fork takes), token [batch, n] the token, score_out [batch, n] the score, rounded to fp32.  done [batch, beams] (int32, NULL: none):
 * a beam with done != 0 has ended; its one candidate is done_token at its score, its logits are not read.  Logits of -infinity are no candidates; a beam whose
 * score is no finite number, or whose logits hold a NaN, +infinity or nothing above -infinity, has none.  Where there are fewer than n: parent and token
 * -1, score -infinity.  beams and n at most 64, V at most 2^20, batch * beams at most 2^20 (LR_EUNSUPPORTED).  Rows may start on any
 * element.  No output overlaps an input or another one, but score_out may be score itself where n = beams.                           */
size_t lr_beam_select_workspace_bytes(int64_t batch, int64_t beams, int64_t V, int64_t n);
int lr_beam_select(const void* logits, int64_t ldl, const float* score, const int32_t* done, int64_t done_token, int32_t* parent, int32_t* token,
                   float* score_out, int64_t batch, int64_t beams, int64_t V, int64_t n, int dt, void* ws, size_t ws_bytes, void* stream);

/* ---- products of 8-bit integers ----------------------------------------------------------------- */
/* Rows as integers of 8 bits with a scale each: scale[t] = max_j |x[t, j]| / 127, at least 2^-126, and q[t, j] the whole number nearest to
 * 127 x[t, j] / max_j |x[t, j]| (ties to even; of rows below 127 * 2^-126, x[t, j] * 2^126), -127 .. 127.  A row with an infinity or a NaN: scale NaN, zeros.  Activations by token, weights
 * [out, in] by output channel.  q rows start on 16 bytes (q and ldq multiples of 16, LR_EALIGN) and are written up to the next multiple of 16 columns, with
 * zeros.  LR_BF16: n and ldx multiples of 8, x 16-byte aligned.                                                                      */
int lr_quant_rows(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t T, int64_t n, int dt, void* stream);
/* c[m, n] = sa[m] * sb[n] * sum_k a[m, k] * b[n, k], the sum exact, the product in fp32 (the row's scale first), rounded to dt.  a [M, lda], b [N, ldb]: rows
 * start on 16 bytes (pointers and strides multiples of 16) and can be read up to the next multiple of 16 columns, whatever is there.  c [M, ldc]: rows start on 16
 * bytes; N is any.  K at most 131071 (2^31 / 128^2), lda and ldb at most 2^22, ldc 2^20 (LR_EUNSUPPORTED).                                       */
int lr_matmul_q8(const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb, const float* sb, void* c, int64_t ldc, int64_t M,
                 int64_t N, int64_t K, int dt, void* stream);
/* The forward of one bottleneck layer with both weights in 8 bits: y = Q(act(Q(x) . W_down^T)) . W_up^T, Q = lr_quant_rows and back; z and act(z) are
 * fp32 and not rounded in between: a row of y has the bits that lr_quant_rows, lr_matmul_q8 and lr_act_fwd in fp32 give it, however many there are.  w_down [r, ld_down], s_down [r], w_up [d_out, ld_up], s_up [d_out] as lr_matmul_q8 takes b.  x, y: as lr_linear_fwd (y's rows start on 16
 * bytes in LR_F32 too).                                                                                                             */
size_t lr_linear_q8_workspace_bytes(int64_t T, int64_t d_in, int64_t r);
int lr_linear_q8_fwd(const void* x, int64_t ldx, const int8_t* w_down, int64_t ld_down, const float* s_down, const int8_t* w_up, int64_t ld_up,
                     const float* s_up, void* y, int64_t ldy, int64_t T, int64_t d_in, int64_t r, int64_t d_out, int act, int dt, void* ws,
                     size_t ws_bytes, void* stream);

/* ---- measurement aid (not on the compute path) ------------------------------------------ */
/* Between begin and end every bf16 MFMA GEMM launch the library makes, and each attention forward /
 * backward call of the block, is bracketed by two HIP events on its stream.  end waits for the last one
 * and writes one record per bracketed launch, in launch order, into records[0 .. max_records) (HOST
 * memory; *n_records receives the number of launches seen, which may exceed max_records).  begin creates
 * max_launches event pairs and end destroys them: the one place where the library creates runtime
 * objects, and only on request.  Process-global and not thread-safe: one measuring thread, no compute
 * calls from other threads meanwhile.  Used by the benchmark for the per-class GEMM and attention rates
 * (Sec. 5.3 of the paper measures the same quantity per linear layer: kernel time and utilisation).
 * Products that otherwise share a launch (small independent ones; the MLP's gate and up pair, where that
 * is faster) each have their own meanwhile: same results, but not the launches of an untimed call.
 * tag: the GEMM's epilogue class (0 store, 1 down-projection: row scale + sigma, 2 / 10 / 11 up-projection
 * + residual, 3 sigma' (+ row statistic), 4 / 12 / 13 RMSNorm backward, 5 weight gradient,
 * 6 SwiGLU backward, 7 SwiGLU forward, 8 / 9 the LaX forms), or LR_TAG_ATTN_FWD / LR_TAG_ATTN_BWD.
 * flops: 2 M N K batch for a GEMM; causal-halved 2 S^2 hd per (batch, head) and product for attention
 * (2 products forward, 5 backward: S, dP, dV, dK, dQ, also where S and dP are formed twice).       */
#define LR_TAG_ATTN_FWD 32
#define LR_TAG_ATTN_BWD 33
typedef struct {
  int tag, M, N, K, batch;
  float ms;
  double flops;
} lr_launch_record;
int lr_launch_timer_begin(int max_launches);
int lr_launch_timer_end(lr_launch_record* records, int max_records, int* n_records);
/* Rows and columns of the output tile that a bf16 product of `batch` members C[M, N] over K runs on: form 0 both
 * operands k-contiguous (activation . weight^T), 1 the second one k-major (gradient . weight), 2 both k-major (weight
 * gradient, not accumulated, nothing folded in); tag: its epilogue class, as above.  Makes no GPU call.   */
int lr_gemm_tile(int M, int N, int K, int batch, int form, int tag, int* rows, int* cols);
/* The same of lr_matmul_q8's product of these sizes, and of lr_linear_q8_fwd's where it does not quantise rows on the way in.    */
int lr_matmul_q8_tile(int64_t M, int64_t N, int64_t K, int* rows, int* cols);
/* Sustained rate of the bf16 matrix pipes fed from registers alone (no LDS, no memory traffic):
 * 2048 wavefronts, 8 independent 32x32x16 accumulator tiles each, iters instructions per tile and
 * launch, `launches` timed launches after up to 4 untimed ones, on `stream`; *tflops (HOST pointer)
 * receives the rate.  random_operands = 0 uses smooth operand values, otherwise pseudo-random ones in
 * (-1, 1): the clock the chip holds under matrix load depends on how much the operand bits toggle,
 * so the second figure is the ceiling for a GEMM on trained-weight-like data.  Creates and destroys
 * two HIP events and waits for the launches.  iters in 1..2^20, launches in 1..1000, else
 * LR_EINVAL.  The utilisation of Sec. 5.3 is read against this figure and the published peak.    */
int lr_mfma_probe(int random_operands, int iters, int launches, double* tflops, void* stream);

/* ---- standalone memory-bound kernels: the unfused twins of the fused epilogues ---------- */
/* stat[t] = sum_j x[t,j]^2  (Alg. 1 line 1).                                               */
int lr_rms_stat(const void* x, int64_t ldx, float* stat, int64_t T, int64_t d, int dt,
                void* stream);
/* xhat = x * gamma / sqrt(stat/d + eps)  (Eq. 4).                                          */
int lr_rmsnorm_apply(const void* x, int64_t ldx, const void* gamma, const float* stat,
                     float eps, void* xhat, int64_t ldo, int64_t T, int64_t d, int dt,
                     void* stream);
/* The steps of Alg. 1 after the exchange: z[t, j] = h_sum[t, j] / sqrt(stat_sum[t] / d_total + eps) for
 * j < n, where h_sum[T, n] is the sum over the ranks of the partial products of LR_NORM_SHARD_LOCAL calls,
 * stat_sum[T] (fp32) the sum of their local statistics and d_total the full feature width (Eq. 5: the
 * result equals RMSNorm over the full width followed by the full projection).                  */
int lr_online_rmsnorm_finish(const void* h_sum, int64_t ldh, const float* stat_sum, int64_t d_total,
                             float eps, void* z, int64_t ldz, int64_t T, int64_t n, int dt,
                             void* stream);
/* Reverse mode of Eq. 4: dx = (dn - n*c)/rms [+ dres], dn = dxhat*gamma, n = x/rms,
 * c = mean_j(dn*n); dgamma_part[nparts, d] fp32 partial column sums of dxhat*n, where
 * nparts = lr_rmsnorm_bwd_parts(T) (the caller, or lr_colsum, adds them up).  dres may be
 * NULL.                                                                                    */
int64_t lr_rmsnorm_bwd_parts(int64_t T);
int lr_rmsnorm_bwd(const void* x, int64_t ldx, const void* gamma, const float* stat, float eps,
                   const void* dxhat, int64_t lddxh, const void* dres, int64_t lddres,
                   void* dx, int64_t lddx, float* dgamma_part, int64_t T, int64_t d, int dt,
                   void* stream);
/* a = act(z) elementwise on a [T, n] tensor.                                               */
int lr_act_fwd(const void* z, int64_t ldz, void* a, int64_t lda, int64_t T, int64_t n,
               int act, int dt, void* stream);
/* m = SiLU(g) * u    and its reverse  dg = dm*u*SiLU'(g), du = dm*SiLU(g).                 */
int lr_swiglu_fwd(const void* g, const void* u, void* m, int64_t ld, int64_t T, int64_t f,
                  int dt, void* stream);
int lr_swiglu_bwd(const void* g, const void* u, const void* dm, void* dg, void* du, int64_t ld,
                  int64_t T, int64_t f, int dt, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LRBOOST_H */
