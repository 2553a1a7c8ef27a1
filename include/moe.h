/*
 * moe.h -- C ABI of the MI355X (gfx950) mixture-of-experts FFN block.
 *
 * The block is the expert layer of a Qwen3-30B-A3B-style MoE reranker: the
 * paper (§3, Expert-Parallel MoE Training) routes each token to its top-8 of
 * 128 experts and, under expert parallelism, dispatches routed tokens to the
 * ranks that hold their experts (§3, "Expert parallelism and topology").  The
 * operations below are, in order:
 *
 *   forward   z = x W_r (fp32 logits); per valid token the top-k experts
 *             (descending logit, ties to the lower expert index) and gates
 *             g = softmax over the k selected logits; a stable permutation of
 *             the routed (token, slot) pairs into expert-major, token-ascending
 *             rows; Xp[r] = x[row_token[r]]; per expert e on its rows
 *             G = Xp W_gate[e], U = Xp W_up[e], A = silu(G) * U, O = A W_down[e];
 *             Y[t] = sum_j g[t,j] O[row_of[t,j]].
 *   backward  dO = g dY and dg = <dY, O> per routed row; dA = dO W_down^T;
 *             dG = dA U s (1 + G (1 - s)), dU = dA silu(G) with s = sigmoid(G);
 *             dXp = dG W_gate^T + dU W_up^T; dW_down = A^T dO,
 *             dW_gate = Xp^T dG, dW_up = Xp^T dU per expert (zero for experts
 *             with no rows); dz = g (dg - sum_j g dg) on the selected experts;
 *             dW_r = x^T dz; dX[t] = sum_j dXp[row_of[t,j]] + dz[t] W_r^T.
 *
 * The paper does not print these equations; the readings taken where it is
 * silent (selection precision, tie-break, gate placement, padding, dropless
 * routing, auxiliary router losses off unless asked for) are the ones stated
 * above and at moe_dims.
 *
 * Conventions shared by every entry point
 *   - All tensors are row-major and live in device memory owned by the
 *     caller; the library never allocates or frees device memory (the one
 *     static scratch array of moe_fwd_noalloc aside, which the HIP runtime
 *     reserves on each GPU when it loads the library's device code).
 *   - "bf16" tensors are IEEE bfloat16 (2 bytes); accumulation is fp32.
 *   - Every device pointer must be 16-byte aligned, but for those of moe_sample
 *     (aligned to their elements).
 *   - Calls are asynchronous on `stream` (a hipStream_t; NULL = the null
 *     stream) and never synchronise the host; counts stay on the device.
 *   - All argument checks happen before any launch: on an error nothing is
 *     launched and an MOE_ERR_* code is returned; moe_last_error() then
 *     describes it (thread-local string, valid until the next call on the
 *     same thread).
 *   - Results are deterministic: two calls with the same inputs produce the
 *     same bits (no atomics decide any floating-point summation order).
 *   - No thread safety is promised for concurrent calls sharing buffers.
 */
#ifndef MOE_MI355X_H
#define MOE_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* return codes */
#define MOE_OK 0
#define MOE_ERR_ARG (-1)       /* null pointer, non-positive size, k not in [1, E], E too large,
                                * a router-loss coefficient negative or not finite */
#define MOE_ERR_SHAPE (-2)     /* H or F not a multiple of 128, E not a multiple of 8 */
#define MOE_ERR_ALIGN (-3)     /* a device pointer not 16-byte aligned */
#define MOE_ERR_WORKSPACE (-4) /* workspace smaller than the size query returns */
#define MOE_ERR_HIP (-5)       /* the HIP runtime reported an error on launch */

/* limits */
#define MOE_MAX_EXPERTS 256
#define MOE_MAX_TOPK 32

/* flags (moe_dims.flags, moe_experts_dims.flags) */
#define MOE_F_MASK 1u    /* token_mask is given: tokens with mask 0 are not routed */
#define MOE_F_DW_FP32 2u /* weight gradients (dW_r, dW_gate, dW_up, dW_down) are fp32, else bf16 */
#define MOE_F_RECOMPUTE 4u /* the forward keeps no G and U (their saved views are NULL and the
                            * saved buffer shrinks by 2 * R_cap * F * 2 bytes); the backward
                            * recomputes them from Xp with the forward's own kernel, one more
                            * gate/up product, so every output is bit-identical to a run
                            * without the flag */

/* Sizes of the full block.  T tokens (T >= 1), hidden size H, E experts,
 * expert width F, top_k experts per token.
 *
 * Router losses (the paper is silent on them; 0 = off, the default):
 *   aux_loss_coef  load-balancing loss  L_aux = aux_loss_coef * E * sum_e f_e P_e,
 *                  f_e = rows of expert e / (T_v k), P_e = mean over valid
 *                  tokens of the full softmax of the logits;
 *   z_loss_coef    z-loss  L_z = z_loss_coef * mean over valid tokens of
 *                  (log sum_e exp z[t,e])^2.
 * With either non-zero, moe_fwd writes {L_aux, L_z} (moe_saved_view.router_loss)
 * and moe_bwd adds their gradient (f held constant) to the router-logit
 * gradient, i.e. the losses join the objective with weight 1.  Both must be
 * finite and >= 0. */
typedef struct moe_dims {
  int32_t T, H, E, F, top_k;
  uint32_t flags;
  float aux_loss_coef, z_loss_coef;
} moe_dims;

/* Device pointers into a `saved` buffer filled by moe_fwd (see
 * moe_saved_views).  R_cap = T * top_k rows are reserved; the routed row
 * count R = offsets[E] <= R_cap lives on the device. */
typedef struct moe_saved_view {
  float* logits;      /* [T, E]      fp32 router logits (masked tokens: computed, not used) */
  int32_t* topk_idx;  /* [T, k]      selected experts, descending logit; -1 for masked tokens */
  float* gates;       /* [T, k]      fp32 gates, sum 1 per valid token; 0 for masked tokens */
  int32_t* counts;    /* [E]         rows per expert */
  int32_t* offsets;   /* [E + 1]     exclusive prefix sum of counts; offsets[E] = R */
  int32_t* row_token; /* [R_cap]     token of row r for r < R, -1 beyond */
  int32_t* row_of;    /* [T, k]      row of (token, slot); -1 for masked tokens */
  void* xp;           /* [R_cap, H]  bf16 permuted tokens (rows >= R undefined) */
  void* g;            /* [R_cap, F]  bf16 gate projection G (NULL with MOE_F_RECOMPUTE) */
  void* u;            /* [R_cap, F]  bf16 up projection U (NULL with MOE_F_RECOMPUTE) */
  void* a;            /* [R_cap, F]  bf16 SwiGLU activation A = silu(G) * U */
  void* o;            /* [R_cap, H]  bf16 expert outputs O (ungated) */
  float* router_loss; /* [2]         {L_aux, L_z}, written when a router-loss coefficient is non-zero */
} moe_saved_view;

/* Bytes of the caller-owned `saved` buffer that carries routing and
 * activations from moe_fwd to moe_bwd.  0 if d is invalid. */
size_t moe_saved_bytes(const moe_dims* d);

/* Bytes of scratch each call needs (contents not preserved across calls).
 * 0 if d is invalid. */
size_t moe_fwd_workspace_bytes(const moe_dims* d);
size_t moe_bwd_workspace_bytes(const moe_dims* d);

/* Fill `view` with device pointers into `saved` (no device work).
 * Returns MOE_OK or MOE_ERR_ARG. */
int moe_saved_views(const moe_dims* d, void* saved, moe_saved_view* view);

/* Forward of the block: the top-k router and the expert FFNs of the paper's
 * MoE layer (§3, Expert-Parallel MoE Training), the forward equations in the
 * header above, with the routed rows grouped per expert as expert-parallel
 * dispatch delivers them to an expert's owner (§3, "Expert parallelism and
 * topology").
 *   x          [T, H]  bf16 tokens
 *   w_r        [H, E]  bf16 router weight
 *   w_gate     [E, H, F], w_up [E, H, F], w_down [E, F, H]  bf16 expert weights
 *   token_mask [T] uint8 (nonzero = real token) when d->flags has MOE_F_MASK,
 *              else ignored (may be NULL)
 *   y          [T, H]  bf16 output (masked tokens: 0)
 *   saved      moe_saved_bytes(d) bytes, filled for moe_bwd
 *   ws         moe_fwd_workspace_bytes(d) bytes of scratch
 */
int moe_fwd(const moe_dims* d, const void* x, const void* w_r, const void* w_gate,
            const void* w_up, const void* w_down, const uint8_t* token_mask, void* y,
            void* saved, void* ws, size_t ws_bytes, void* stream);

/* Backward of the block (the training step of §3, Expert-Parallel MoE
 * Training): the backward equations in the header above, from the `saved`
 * buffer of the matching moe_fwd (same d, x and weights).
 *   dy      [T, H] bf16 upstream gradient
 *   dx      [T, H] bf16
 *   dw_r    [H, E], dw_gate [E, H, F], dw_up [E, H, F], dw_down [E, F, H]:
 *           bf16, or fp32 with MOE_F_DW_FP32; overwritten (not accumulated)
 *   ws      moe_bwd_workspace_bytes(d) bytes of scratch
 */
int moe_bwd(const moe_dims* d, const void* x, const void* w_r, const void* w_gate,
            const void* w_up, const void* w_down, const void* dy, const void* saved,
            void* dx, void* dw_r, void* dw_gate, void* dw_up, void* dw_down, void* ws,
            size_t ws_bytes, void* stream);

/* Allocation-free forward, for callers that cannot allocate device memory or
 * must not see an allocation happen: code under HIP graph capture, tight
 * serving or training loops, harnesses that forbid hipMalloc.  The same
 * operation, arguments (minus the workspace) and outputs as moe_fwd, bit for
 * bit; its scratch is a static array of MOE_NOALLOC_SCRATCH_BYTES bytes
 * inside the library, one per GPU (reserved on each GPU the library runs on
 * until the process ends).  It calls no allocation routine of any kind.
 *   Limit: moe_fwd_workspace_bytes(d) <= MOE_NOALLOC_SCRATCH_BYTES (about
 *   13 bytes per token and expert, with the router losses on: T <= 40000 at
 *   E = 128); larger sizes return MOE_ERR_WORKSPACE before any launch.
 *   Every call on one GPU shares that GPU's array: calls that overlap on one
 *   GPU (two streams, two host threads) race and must be serialised by the
 *   caller.  Nothing in the array needs to start at zero (the kernels clear
 *   what they count into), and its contents after a call are unspecified. */
#define MOE_NOALLOC_SCRATCH_BYTES (64u << 20)
int moe_fwd_noalloc(const moe_dims* d, const void* x, const void* w_r, const void* w_gate,
                    const void* w_up, const void* w_down, const uint8_t* token_mask, void* y,
                    void* saved, void* stream);

/* Expert LoRA (§3, "LoRA target groups for MoE"; §4.3): rank-r adapters on
 * every expert's fused gate/up projection and its down projection, with the
 * base expert weights and the router frozen.  Per expert e the effective
 * weights are
 *   W_gate[e] + scale a1[e] b1_gate[e],  W_up[e] + scale a1[e] b1_up[e],
 *   W_down[e] + scale a2[e] b2[e],
 * applied through the rank-r intermediates P1 = scale Xp a1 and
 * P2 = scale A a2 (bf16, kept in the saved buffer after the block's own
 * layout, so moe_saved_views applies to it unchanged).  The backward writes dX
 * and the five adapter gradients (bf16, or fp32 with MOE_F_DW_FP32) and no base
 * or router weight gradients; dX includes the router term (the router is
 * frozen, not detached).  MOE_F_MASK, MOE_F_RECOMPUTE and the router-loss
 * coefficients behave as in moe_fwd / moe_bwd. */
typedef struct moe_lora {
  int32_t rank;        /* r: 16, 32, 48 or 64 */
  float scale;         /* multiplies every adapter product (alpha / r in the usual parametrisation) */
  const void* a1;      /* [E, H, r] bf16 */
  const void* b1_gate; /* [E, r, F] bf16 */
  const void* b1_up;   /* [E, r, F] bf16 */
  const void* a2;      /* [E, F, r] bf16 */
  const void* b2;      /* [E, r, H] bf16 */
} moe_lora;

/* Bytes of the LoRA saved buffer and of the scratch either LoRA call needs
 * (0 if d or rank is invalid). */
size_t moe_lora_saved_bytes(const moe_dims* d, int32_t rank);
size_t moe_lora_workspace_bytes(const moe_dims* d, int32_t rank);

/* Forward with the adapters; arguments as moe_fwd plus `lora`. */
int moe_lora_fwd(const moe_dims* d, const void* x, const void* w_r, const void* w_gate,
                 const void* w_up, const void* w_down, const moe_lora* lora,
                 const uint8_t* token_mask, void* y, void* saved, void* ws, size_t ws_bytes,
                 void* stream);

/* Backward with the adapters, from the saved buffer of the matching
 * moe_lora_fwd (same d, x, weights and adapters).
 *   dy    [T, H] bf16;  dx  [T, H] bf16
 *   da1 [E, H, r], db1_gate [E, r, F], db1_up [E, r, F], da2 [E, F, r],
 *   db2 [E, r, H]: overwritten; zero for experts with no rows */
int moe_lora_bwd(const moe_dims* d, const void* x, const void* w_r, const void* w_gate,
                 const void* w_up, const void* w_down, const moe_lora* lora, const void* dy,
                 const void* saved, void* dx, void* da1, void* db1_gate, void* db1_up, void* da2,
                 void* db2, void* ws, size_t ws_bytes, void* stream);

/* Forward-only pass of the block for serving (reranking scores a batch of
 * query-passage pairs in one prefill pass, §4.2 "Inference throughput"): the Y of
 * moe_fwd, bit for bit, without a saved buffer.  Routing, A and O live in the
 * workspace, G and U are never stored, and the gate/up product reads its rows
 * of x through the permutation instead of a gathered copy (a copy is made in
 * the workspace only when T * H * 2 bytes exceed 2^31 - 1).  MOE_F_MASK as in
 * moe_fwd; MOE_F_DW_FP32, MOE_F_RECOMPUTE and the router-loss coefficients
 * are ignored.
 *   x, w_r, w_gate, w_up, w_down, token_mask, y   as in moe_fwd
 *   ws    moe_infer_workspace_bytes(d) bytes of scratch
 */
size_t moe_infer_workspace_bytes(const moe_dims* d);
int moe_infer(const moe_dims* d, const void* x, const void* w_r, const void* w_gate,
              const void* w_up, const void* w_down, const uint8_t* token_mask, void* y,
              void* ws, size_t ws_bytes, void* stream);

/* One expert-parallel rank's share (§3, "Expert parallelism and topology"):
 * the rows dispatched to this rank's E local experts, already grouped
 * expert-major.  rows = capacity of the row buffers (rows >= 1). */
typedef struct moe_experts_dims {
  int32_t rows, H, E, F;
  uint32_t flags; /* MOE_F_DW_FP32, MOE_F_RECOMPUTE */
} moe_experts_dims;

/* Device pointers into an experts `saved` buffer. */
typedef struct moe_experts_saved_view {
  int32_t* offsets; /* [E + 1] exclusive prefix sum of counts, clamped to rows */
  void* g;          /* [rows, F] bf16 (NULL with MOE_F_RECOMPUTE) */
  void* u;          /* [rows, F] bf16 (NULL with MOE_F_RECOMPUTE) */
  void* a;          /* [rows, F] bf16 */
} moe_experts_saved_view;

size_t moe_experts_saved_bytes(const moe_experts_dims* d);
size_t moe_experts_workspace_bytes(const moe_experts_dims* d);
int moe_experts_saved_views(const moe_experts_dims* d, void* saved, moe_experts_saved_view* view);

/* Forward of the local experts.
 *   xp      [rows, H] bf16 dispatched rows, expert-major
 *   counts  [E] int32 on the device: rows of each local expert, in order.  Rows
 *           past the capacity (prefix sum beyond `rows`) are dropped: not read,
 *           not computed, not written.  Output rows past sum(counts) are not written.
 *   o       [rows, H] bf16 expert outputs (ungated)
 */
int moe_experts_fwd(const moe_experts_dims* d, const void* xp, const int32_t* counts,
                    const void* w_gate, const void* w_up, const void* w_down, void* o,
                    void* saved, void* ws, size_t ws_bytes, void* stream);

/* Backward of the local experts from the matching moe_experts_fwd `saved`
 * (which holds the row offsets; counts are not passed again).
 *   d_o     [rows, H] bf16 gradient of o
 *   dxp     [rows, H] bf16
 *   dw_*    as in moe_bwd (overwritten; zero for experts with no rows)
 */
int moe_experts_bwd(const moe_experts_dims* d, const void* xp, const void* w_gate, const void* w_up, const void* w_down, const void* d_o,
                    const void* saved, void* dxp, void* dw_gate, void* dw_up, void* dw_down,
                    void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ 8-bit serving
 * The forward-only pass with int8 weights and activations, and the attention
 * beside it over an int8 cache.  Bytes are the bound of serving, so weights
 * and cache are held in 8 bits; every sum is exact (int32) or fp32.
 *
 * Integer rows ("int8 rows"): a row x of K values is held as
 *   q_k = rint(127 x_k / a), a = max |x_k|, and the scale s = a / 127,
 * so x ~ s q.  A row of zeros has s = 0; a row with an infinity or NaN has
 * s = NaN and q = 0, so everything computed from it is NaN.
 *
 * What is held in fewer bits than fp32 beside the int8 rows and bf16 outputs:
 *   - softmax weights enter the product with the values in fp16, times 2^7 to
 *     2^15 against the largest: 2^-11 of each, and those below 2^-32 of the
 *     largest may be 0 there (the sum they are divided by is of the fp32 weights);
 *     scales of values below 2^-80 count as that there;
 *   - queries are fp16 over a power of two per row: exact but for elements under
 *     2^-17 of the row's largest, which are off by 2^-25 of it at most;
 *   - exponentials and the reciprocals of the sigmoid and of value scales are
 *     the hardware's, within an ulp or two of fp32.
 */

/* flags (moe_i8_dims.flags, moe_kv_attn.flags) */
#define MOE_F_OUT_FP32 8u /* moe_i8_dims: the output is fp32, else bf16 */
#define MOE_F_CAUSAL 16u  /* moe_kv_attn: a token sees the keys up to its own position, else all */

#define MOE_I8_MAX_K 131072 /* sums of K products of int8 are at most 2^31 in magnitude */

/* Rows of x ([rows, K] bf16, row pitch ldx elements) as int8 rows: q [rows, K],
 * scale [rows].  rows >= 1; K a multiple of 16, at most MOE_I8_MAX_K; ldx >= K,
 * a multiple of 8. */
int moe_i8_quant_rows(int32_t rows, int32_t K, const void* x, int64_t ldx, int8_t* q, float* scale, void* stream);

/* Weights laid out for the int8 products, once: w [E, K, N] bf16 -> q [E, N, K],
 * one int8 row and scale[e][n] per output channel.  E, N >= 1; K as above. */
int moe_i8_quant_weight(int32_t E, int32_t K, int32_t N, const void* w, int8_t* q, float* scale, void* stream);

/* Product of int8 rows: out[m][n] = a_scale[m] b_scale[n] sum_k a[m][k] b[n][k].
 * M, N >= 1, K a multiple of 16. */
typedef struct moe_i8_dims {
  int32_t M, N, K;
  uint32_t flags; /* MOE_F_OUT_FP32 */
} moe_i8_dims;

/*   a [M, K], a_scale [M]; b [N, K], b_scale [N]
 *   out  [M, N] bf16 or fp32, row pitch ldo >= N elements */
int moe_i8_matmul(const moe_i8_dims* d, const int8_t* a, const float* a_scale, const int8_t* b, const float* b_scale,
                  void* out, int64_t ldo, void* stream);

/* The same from bf16 rows x ([M, K], row pitch ldx), quantised on the way.
 *   ws  moe_i8_linear_workspace_bytes(d) bytes of scratch */
size_t moe_i8_linear_workspace_bytes(const moe_i8_dims* d);
int moe_i8_linear(const moe_i8_dims* d, const void* x, int64_t ldx, const int8_t* b, const float* b_scale, void* out,
                  int64_t ldo, void* ws, size_t ws_bytes, void* stream);

/* Expert weights in int8 (moe_i8_quant_weight of [E, H, F] and [E, F, H]). */
typedef struct moe_i8_experts {
  const int8_t* w_gate;  /* [E, F, H] */
  const int8_t* w_up;    /* [E, F, H] */
  const int8_t* w_down;  /* [E, H, F] */
  const float* s_gate;   /* [E, F] */
  const float* s_up;     /* [E, F] */
  const float* s_down;   /* [E, H] */
} moe_i8_experts;

/* moe_experts_fwd in 8 bits, forward only: O = A W_down, A = silu(G) U held as
 * int8 rows, G and U int8 products of the int8 rows of xp.  d->flags must be 0.
 *   ws  moe_experts_i8_workspace_bytes(d) bytes of scratch */
size_t moe_experts_i8_workspace_bytes(const moe_experts_dims* d);
int moe_experts_i8(const moe_experts_dims* d, const void* xp, const int32_t* counts, const moe_i8_experts* w, void* o,
                   void* ws, size_t ws_bytes, void* stream);

/* moe_infer with the experts in 8 bits; the router stays bf16 (its selection is
 * moe_infer's), the combine fp32.  Arguments as moe_infer.
 *   ws  moe_infer_i8_workspace_bytes(d) bytes of scratch */
size_t moe_infer_i8_workspace_bytes(const moe_dims* d);
int moe_infer_i8(const moe_dims* d, const void* x, const void* w_r, const moe_i8_experts* w, const uint8_t* token_mask,
                 void* y, void* ws, size_t ws_bytes, void* stream);

/* A paged cache of keys and values in 8 bits.  Block i holds block_tokens
 * tokens of one request; per block and head one scale each for keys and
 * values: key = k_scale k.  Values are stored token-last, the layout in which
 * the attention's product reads them. */
typedef struct moe_kv_cache {
  int32_t n_blocks;     /* >= 1 */
  int32_t block_tokens; /* 16, 32, 64 or 128 */
  int32_t kv_heads;     /* >= 1 */
  int32_t head_dim;     /* 64 or 128 */
  int8_t* k;            /* [n_blocks, kv_heads, block_tokens, head_dim] */
  int8_t* v;            /* [n_blocks, kv_heads, head_dim, block_tokens] */
  float* k_scale;       /* [n_blocks, kv_heads] */
  float* v_scale;       /* [n_blocks, kv_heads] */
} moe_kv_cache;

/* A batch of B requests whose new tokens are packed request after request
 * into T rows: rows row_start[b] .. row_start[b + 1] (non-decreasing) are the
 * last of request b's kv_len[b] tokens.  A row_start may pass T, as those of
 * moe_kv_plan do when T is too small: kv_len then counts tokens that have no
 * row, the rows there are keep their positions, and the tokens past them are
 * not written and not seen.  Token p lies in block
 * block_table[b][p / block_tokens]; entries outside [0, n_blocks) and tokens
 * past W blocks have no place: they are not written, and no query sees them.
 * All three arrays are on the device. */
typedef struct moe_kv_batch {
  int32_t B, T, W;
  const int32_t* row_start;   /* [B + 1] */
  const int32_t* kv_len;      /* [B] */
  const int32_t* block_table; /* [B, W] */
} moe_kv_batch;

/* Tables of one step, built on the device from request lengths: request b has
 * old_len[b] tokens in the cache and gets new_len[b] more (negative counts as
 * 0, and what exceeds 2^30 - 1 as that).  Blocks its table lacks are taken in request order from the top of the
 * stack free_ids[0 .. n_free).
 *   block_table [B, W]  the blocks taken are written (-1 once the stack is
 *                       empty), all other entries are left alone
 *   row_start [B + 1], kv_len [B]   as in moe_kv_batch: of all new tokens, also
 *                       where T is too small for them
 *   positions, slots, seq [T]       per packed token its position in its
 *                       request, block * block_tokens + offset (-1: no place)
 *                       and its request; -1 past the last token
 *   state [2]           {blocks left on the stack, blocks that were missing}
 * A step's kv_len and state[0] are the next one's old_len and n_free: kv_len
 * may be old_len or new_len itself, and state begin at n_free (one launch
 * more).  Nothing else that is written may overlap what is read. */
typedef struct moe_kv_plan_dims {
  int32_t B, T, W;      /* B, W >= 1, T >= 0 */
  int32_t n_blocks, block_tokens;
  int32_t free_cap;     /* entries of free_ids (0: free_ids is not looked at) */
} moe_kv_plan_dims;
int moe_kv_plan(const moe_kv_plan_dims* d, const int32_t* old_len, const int32_t* new_len, int32_t* block_table,
                const int32_t* free_ids, const int32_t* n_free, int32_t* row_start, int32_t* kv_len,
                int32_t* positions, int32_t* slots, int32_t* seq, int32_t* state, void* stream);

/* Write the batch's new keys and values (k, v: T rows of [kv_heads, head_dim]
 * bf16, row pitch ld elements, a multiple of 8) into their blocks.  A block's
 * scale is that of the largest value written to it since its first token
 * (largest / 127 in fp32): it only grows, and the tokens it already holds are
 * rounded again when it does.  A value is rounded as rint(x / scale) in fp32,
 * with the scale as it is stored.
 * A non-finite key or value makes the scale of its block and head NaN. */
int moe_kv_append(const moe_kv_cache* c, const moe_kv_batch* b, const void* k, const void* v, int64_t ld,
                  void* stream);

/* Read the first kv_start[b + 1] - kv_start[b] tokens of each request back as
 * bf16 rows kv_start[b] .. (kv_start [B + 1] on the device, non-decreasing,
 * clamped to [0, total]): k_out, v_out [total, kv_heads, head_dim].  Tokens
 * without a place read as 0; rows before kv_start[0] and from kv_start[B] on
 * are not written. */
int moe_kv_read(const moe_kv_cache* c, int32_t B, int32_t W, const int32_t* block_table, const int32_t* kv_start,
                int32_t total, void* k_out, void* v_out, void* stream);

/* Attention of the batch's new tokens over their requests' cache: per head
 *   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale <q, k_j>),
 * over the keys the token sees (none: out = 0).  Query head i reads kv head
 * i / (heads / kv_heads).  Rows of no request are not written.
 *   q, out  T rows of [heads, head_dim] bf16, row pitches ldq and ldo elements (multiples of 8) */
typedef struct moe_kv_attn {
  int32_t heads;  /* a multiple of kv_heads */
  int32_t max_q;  /* no request has more new tokens (rows past it are not written) */
  int32_t max_kv; /* no request has more tokens (keys past it are not seen); at most W * block_tokens counts */
  float scale;    /* finite */
  uint32_t flags; /* MOE_F_CAUSAL */
} moe_kv_attn;
size_t moe_kv_attention_workspace_bytes(const moe_kv_cache* c, const moe_kv_batch* b, const moe_kv_attn* a);
int moe_kv_attention(const moe_kv_cache* c, const moe_kv_batch* b, const moe_kv_attn* a, const void* q, int64_t ldq,
                     void* out, int64_t ldo, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ a decoding step
 * What a step needs around the products and the attention: the sum with the
 * residual and its norm (with a backward, for training), the expert layer for
 * a few tokens, and the next token from the logits. */

/* Root-mean-square norm of rows, of their sum with a residual where there is
 * one:
 *   h = bf16(x + residual),  s = 1 / sqrt(mean_c h^2 + eps),  v = h s w (fp32),
 *   y = bf16(v),  q, scale = the int8 rows of v.
 * The norm is that of the sum as stored.  A row whose squares pass fp32 has
 * s = 0; one with an infinity or NaN holds NaN where that was times s, and as
 * an int8 row its scale is NaN. */
#define MOE_NORM_MAX_H 32768
typedef struct moe_norm_dims {
  int32_t T, H;   /* T >= 1 rows of H: a multiple of 8 (of 16 for int8 rows), at most MOE_NORM_MAX_H */
  uint32_t flags; /* MOE_F_DW_FP32: the backward's dw is fp32, else bf16 */
  float eps;      /* a positive normal number */
} moe_norm_dims;

/*   x         [T, H] bf16, row pitch ldx elements (a multiple of 8)
 *   residual  the same with ldr, or NULL (ldr is ignored)
 *   w         [H] bf16
 *   h         [T, H] bf16 or NULL; NULL without a residual
 *   y         [T, H] bf16 or NULL
 *   q, scale  [T, H] int8 and [T], or both NULL; y or q is given
 * h or y may be x or residual itself where that has pitch H; apart from this
 * nothing that is written may overlap anything else. */
int moe_norm_fwd(const moe_norm_dims* d, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* w,
                 void* h, void* y, int8_t* q, float* scale, void* stream);

/* Backward.  With n = h s and g = dy w:
 *   dx = s (g - n mean_c(g n)) + dh,  dw = sum_t dy n
 * dx is the gradient of x and of the residual alike.  A row whose squares pass fp32
 * (s = 0) has dx = dh, or NaN where the sum of dy w h passes fp32 too.
 *   h   the rows that were normed (the stored sum; x without a residual), pitch ldh
 *   dy  [T, H] bf16, pitch lddy;  dh the gradient that reaches h past the norm, pitch lddh, or NULL
 *   dx  [T, H] bf16; may be dy or dh itself where that has pitch H, else overlaps nothing
 *   dw  [H] bf16, or fp32 with MOE_F_DW_FP32; overwritten
 *   ws  moe_norm_bwd_workspace_bytes(d) bytes of scratch */
size_t moe_norm_bwd_workspace_bytes(const moe_norm_dims* d);
int moe_norm_bwd(const moe_norm_dims* d, const void* h, int64_t ldh, const void* w, const void* dy, int64_t lddy,
                 const void* dh, int64_t lddh, void* dx, void* dw, void* ws, size_t ws_bytes, void* stream);

/* moe_infer for at most MOE_DECODE_MAX_T tokens: the same layer with the same
 * selection and gates, bit for bit, in tiles for few rows.  G, U and O stay
 * fp32, and A enters the down product whole (as three bf16 that add up to it, 2^-25
 * of it or 2^-125 aside), so Y is closer to the equations than moe_infer's and not its bits; an
 * infinite weight gives what it gives there.  Arguments and flags as
 * moe_infer.
 *   ws  moe_decode_workspace_bytes(d) bytes of scratch, enough for fewer tokens too */
#define MOE_DECODE_MAX_T 64
size_t moe_decode_workspace_bytes(const moe_dims* d);
int moe_decode(const moe_dims* d, const void* x, const void* w_r, const void* w_gate, const void* w_up,
               const void* w_down, const uint8_t* token_mask, void* y, void* ws, size_t ws_bytes, void* stream);

/* The same with the experts in 8 bits, as in moe_infer_i8 (O stays fp32).
 *   ws  moe_decode_i8_workspace_bytes(d) bytes of scratch */
size_t moe_decode_i8_workspace_bytes(const moe_dims* d);
int moe_decode_i8(const moe_dims* d, const void* x, const void* w_r, const moe_i8_experts* w, const uint8_t* token_mask,
                  void* y, void* ws, size_t ws_bytes, void* stream);

/* The next token of each of B rows of V logits, from a given number u in [0, 1)
 * per row.  Larger logits come first, equal ones by lower index.
 *   weights  e^((logit - largest) / temperature), held to 2^-43 of the largest, or
 *            to 2^-52 |logit| / temperature of themselves where that is more
 *   top_k    the first top_k stay; 0 or less, or V or more: all
 *   top_p    of those the shortest prefix whose weights reach top_p of their
 *            sum stays, one at least; 1 or more: all
 *   min_p    of those the weights of at least min_p times the largest stay
 *            (more than 1 counts as 1); 0 or less: all
 *   token    of what stays the lowest index at which the running sum of
 *            weights, in index order, passes u times their sum
 * A temperature of 0 or less (or NaN) takes the first in the order.  NaN in
 * top_p or min_p turns that filter off; u below 0 or NaN counts as 0, u of 1
 * and more takes the last of any weight.  A logit of -infinity or NaN is never taken; +infinity
 * leaves only its like.  A row without a logit to take has token -1 and
 * logprob -infinity.  Weights are summed by chunks of 8192 logits, counted from the
 * 16 bytes that the row begins in, and each sum is rounded to 2^-43 of the row's
 * largest weight: a draw or a border nearer than that to the next token may be that
 * token's where the row begins elsewhere within its 16 bytes. */
#define MOE_SAMPLE_MAX_V 1048576
typedef struct moe_sample_dims {
  int32_t B, V;   /* 1 <= B <= 65535, 1 <= V <= MOE_SAMPLE_MAX_V */
  uint32_t flags; /* MOE_F_LOGITS_FP32 */
} moe_sample_dims;
#define MOE_F_LOGITS_FP32 32u /* moe_sample_dims: the logits are fp32, else bf16 */

/*   logits       [B, V], row pitch ld >= V elements; like all but ws it
 *                may begin at any element (not only on 16 bytes)
 *   temperature, top_p, min_p  [B] fp32, top_k [B] int32, each on the device, or NULL: off (temperature: 1)
 *   u            [B] fp32
 *   token        [B] int32
 *   logprob      [B] fp32 or NULL: log of the token's share of the weights that stay (0 at temperature 0)
 *   ws           moe_sample_workspace_bytes(d) bytes of scratch */
size_t moe_sample_workspace_bytes(const moe_sample_dims* d);
int moe_sample(const moe_sample_dims* d, const void* logits, int64_t ld, const float* temperature,
               const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token,
               float* logprob, void* ws, size_t ws_bytes, void* stream);

/* Per-kernel timing.  With tracing on, every kernel the library launches is
 * bracketed by two HIP events recorded on its launch stream (no host
 * synchronisation at launch time).  moe_trace_read waits for the recorded
 * events, writes per kernel id the summed milliseconds and the number of
 * launches since the last read (arrays of n entries; either may be NULL), and
 * returns the number of kernel ids (or MOE_ERR_HIP).  moe_trace_name(id) is a
 * kernel's name ("" for an unknown id).  Not thread-safe; off by default. */
int moe_trace_enable(int on);
int moe_trace_read(double* total_ms, int32_t* launches, int n);
const char* moe_trace_name(int id);

/* Message describing the last error on this thread ("" if none). */
const char* moe_last_error(void);

/* Library version, major * 10000 + minor * 100 + patch. */
int moe_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MOE_MI355X_H */
