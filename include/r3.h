/*
 * r3.h - C ABI of the replayed-routing MoE layer for AMD MI355X (gfx950).
 *
 * The calls follow Section 4.1 ("Implementation") of "Stabilizing MoE
 * Reinforcement Learning by Aligning Training and Inference Routers"
 * (arxiv 2510.11370): the MoE layer of the training pass is run with the
 * expert mask recorded at inference, while the softmax is still taken over the
 * training logits so that the router keeps its gradient.
 *
 * Notation: T tokens, d hidden size, E experts (the paper's M), K selected
 * experts per token, F width of one SwiGLU expert.  A slot is one (token t, j)
 * pair with id t*K + j; there are T*K slots.  "row" is a slot's position after
 * the slots are sorted by expert.
 *
 * Conventions for every call
 *  - All data pointers are DEVICE pointers owned by the caller.  The calls
 *    declared in this header allocate nothing, free nothing and keep no state
 *    between calls (the one exception is spelled out at r3_permute_static: a
 *    fixed scratch array and its cached address).  Scratch comes from a caller
 *    workspace of at least r3_workspace_bytes(desc, op) bytes, 256-byte
 *    aligned.  (The measurement aids of r3_profile.h are not part of the
 *    method and do keep state: event pools and an on/off flag.)
 *  - `stream` is a hipStream_t (NULL = the default stream).  Calls enqueue work
 *    and return; there is no hidden synchronisation.
 *  - Matrices are row-major and dense.  Activations and weights have the dtype
 *    desc->act (bf16 or f32); gates, logits and weight gradients are f32;
 *    counts, offsets and permutations are int32.
 *  - The return value is an r3_status.  Errors the host can see (NULL pointer,
 *    bad sizes, misaligned pointer, small workspace) are returned before
 *    anything is launched.  Errors only the device can see (an expert id >= E,
 *    a duplicate id inside a token, a non-finite logit) OR bits into the
 *    optional device word `status_word` (R3_DATA_*); the affected token's
 *    outputs are then unspecified but no access goes out of bounds.
 *  - Every result is deterministic: the same inputs give the same bits.  A
 *    token's logits and gates, and for f32 its rows of y and dx, are the same
 *    bits whatever other tokens the call has.
 */
#ifndef R3_H
#define R3_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum r3_status {
    R3_OK = 0,
    R3_ERR_INVALID_ARG = 1, /* NULL pointer, size <= 0, K > E, misaligned pointer  */
    R3_ERR_UNSUPPORTED = 2, /* index dtype too narrow for E, E or K above a kernel limit */
    R3_ERR_WORKSPACE = 3,   /* workspace NULL or smaller than r3_workspace_bytes   */
    R3_ERR_HIP = 4          /* a launch failed                                     */
} r3_status;

enum { R3_BF16 = 0, R3_F32 = 1 };     /* desc->act   */
enum { R3_IDX_U8 = 0, R3_IDX_U16 = 1 }; /* desc->idx   */

/* bits of the device status word */
enum { R3_DATA_IDX_RANGE = 1, R3_DATA_IDX_DUP = 2, R3_DATA_NONFINITE = 4, R3_DATA_CACHE_ADDR = 8 };

typedef enum r3_op {
    R3_OP_REPLAY_GATE = 0,
    R3_OP_PERMUTE = 1,
    R3_OP_GROUPED_FFN = 2,
    R3_OP_BACKWARD = 3,
    R3_OP_FORWARD = 4       /* r3_moe_forward */
} r3_op;

enum { R3_FLAG_GATED_H = 1 };         /* desc->flags */

typedef struct r3_layer_desc {
    int32_t T, d, E, K, F;
    int32_t act;              /* R3_BF16 or R3_F32                                  */
    int32_t idx;              /* R3_IDX_U8 (E <= 256) or R3_IDX_U16 (E <= 65536)     */
    int32_t flags;            /* 0, or R3_FLAG_GATED_H for r3_moe_backward after
                                 r3_moe_forward (see there)                          */
    int64_t idx_token_stride; /* elements between two tokens' records; 0 means K.
                                 K gives a layer-major record [L][T][K]; L*K a
                                 token-major one [T][L][K] (Section 4.2: the
                                 inference side appends per token).               */
} r3_layer_desc;

/* Limits of this build: E <= 4096, K <= 64, K <= E. */

/* Bytes of workspace `op` needs for this layer (0 is possible). */
size_t r3_workspace_bytes(const r3_layer_desc *desc, r3_op op);

/* Human-readable build string. */
const char *r3_version(void);

/*
 * TopKMask(s, K) of Section 4.1 (second equation; used on the inference logits
 * to make the record I_infer).  For each of the T rows of `logits` ([T, ld]
 * f32, first E columns used) write the ids of the K largest entries to
 * `idx_out` ([T] records of K ids, stride desc->idx_token_stride), ascending by
 * id.  Ties go to the lower id; NaN ranks below every number; -0 equals +0.
 * A NaN or infinity sets R3_DATA_NONFINITE.
 */
int r3_record_topk(const r3_layer_desc *desc, const float *logits, int64_t ld,
                   void *idx_out, int32_t *status_word, void *stream);

/*
 * Router logits and replay gate of Section 4.1: s = x W_r (+ bias), then
 * g[t,j] = exp(s[t,idx[t,j]]) / sum_i exp(s[t,idx[t,i]]) over the K recorded
 * experts (replay-gate equation).  x [T,d] act, W_r [d,E] act, bias [E] f32 or
 * NULL, idx the record, gates [T,K] f32 aligned with idx.  Logits are
 * accumulated and kept in f32.  Optional outputs: logits_out [T,E] f32;
 * agree_out int64[2] which is INCREMENTED by {tokens whose own top-K set equals
 * the recorded set, total experts the two sets share} (Section 3.2, router
 * level; zero it before the first call).
 */
int r3_replay_gate(const r3_layer_desc *desc, const void *x, const void *W_r,
                   const float *bias, const void *idx, float *gates,
                   float *logits_out, int64_t *agree_out, int32_t *status_word,
                   void *ws, size_t ws_bytes, void *stream);

/*
 * Dispatch implied by the replay-output equation of Section 4.1: sort the T*K
 * slots by recorded expert, stably (ascending slot id inside an expert).
 * counts [E], offsets [E+1] (exclusive prefix sum), inv_perm [T*K] slot -> row,
 * perm [T*K] row -> slot, Xp [T*K,d] act with Xp[row] = x[perm[row] / K]
 * (Xp may be NULL to skip the row gather).  Sets R3_DATA_IDX_RANGE /
 * R3_DATA_IDX_DUP for a bad record.
 */
int r3_permute(const r3_layer_desc *desc, const void *x, const void *idx,
               int32_t *counts, int32_t *offsets, int32_t *inv_perm, int32_t *perm,
               void *Xp, int32_t *status_word, void *ws, size_t ws_bytes,
               void *stream);

/*
 * r3_permute for callers that cannot allocate or carry a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, results and status bits as r3_permute, without `ws`: the
 * scratch (per-chunk expert histograms and their running sums) is a fixed
 * array of R3_STATIC_SCRATCH_BYTES inside the library's device code, one copy
 * per GPU, held until the process ends; nothing is allocated or freed, by
 * this call or by anything it uses.  Its device address is looked up on the
 * first call on each device (with that device current) and kept.
 * Returns R3_ERR_UNSUPPORTED when r3_workspace_bytes(desc, R3_OP_PERMUTE)
 * exceeds R3_STATIC_SCRATCH_BYTES (that is (T*K/1024 rounded up, at most 512)
 * * E * 8 bytes: E <= 1024 always fits), R3_ERR_HIP when the address lookup
 * fails.  All calls on one GPU share the one array, on every stream: two calls
 * that overlap in time on a GPU race; calls ordered by a stream or an event
 * are fine (every word that is read is written first by the same call).
 */
#define R3_STATIC_SCRATCH_BYTES (4u << 20)
int r3_permute_static(const r3_layer_desc *desc, const void *x, const void *idx,
                      int32_t *counts, int32_t *offsets, int32_t *inv_perm, int32_t *perm,
                      void *Xp, int32_t *status_word, void *stream);

/*
 * The expert networks E_i of the replay-output equation, as bias-free SwiGLU:
 * for expert e and its rows r in [offsets[e], offsets[e+1]):
 *   A = Xp W_gate[e], B = Xp W_up[e], H = silu(A) * B, Yp = H W_down[e].
 * Xp [T*K,d]; W_gate, W_up [E,d,F]; W_down [E,F,d]; Yp [T*K,d]; H [T*K,F]
 * (required: it is the second GEMM's input and the backward's saved value).
 * FA_save, FB_save [T*K,F] or both NULL (forward only): what the backward
 * needs of the pre-activations, as the two factors its SwiGLU step multiplies
 * with: FA = B * silu'(A) (so that dA = dh * FA) and FB = silu(A) (dB = dh * FB),
 * silu'(a) = s (1 + a (1 - s)), s = sigmoid(a).  A and B themselves are not
 * stored.  All act dtype; f32 accumulation; `offsets` is read on the device.
 * Xp may be NULL when x [T,d] and perm [T*K] (from r3_permute) are given: row
 * r is then read as x[perm[r] / K] inside the first contraction's tile loads
 * and no gathered copy of the tokens is needed (r3_permute may be called with
 * Xp = NULL as well); needs T*d*sizeof(act) < 2^31.  x and perm are ignored
 * when Xp is given.
 */
int r3_grouped_ffn(const r3_layer_desc *desc, const void *Xp, const void *x, const int32_t *perm,
                   const int32_t *offsets, const void *W_gate, const void *W_up, const void *W_down,
                   void *Yp, void *H, void *FA_save, void *FB_save, void *ws,
                   size_t ws_bytes, void *stream);

/*
 * Replay output of Section 4.1: y[t] = sum_j gates[t,j] * Yp[inv_perm[t*K+j]],
 * j ascending, f32 accumulation, one rounding to act.  y [T,d].
 */
int r3_combine(const r3_layer_desc *desc, const void *Yp, const float *gates,
               const int32_t *inv_perm, void *y, void *stream);

/*
 * Gradients of r3_combine and of r3_permute's rows as calls of their own, for
 * expert networks that are not this library's (adapters, other activations or
 * number formats): r3_permute, the caller's experts on the rows of Xp,
 * r3_combine; back: r3_combine_backward, the caller's gradients, then
 * r3_permute_backward.  (r3_moe_backward has the two in its own steps.)
 *
 * r3_combine_backward: given dy [T,d], for the K slots of every token
 *   dYp[inv_perm[t*K+j]] = gates[t,j] dy[t]              ([T*K,d], one rounding)
 *   dgates[t,j] = <dy[t], Yp[inv_perm[t*K+j]]>           ([T,K] f32, f32 sums;
 *                 Yp as r3_combine takes it, without the gate)
 *   dz[t,j] = gates[t,j] (dgates[t,j] - sum_i gates[t,i] dgates[t,i])
 * dz [T,K] f32 is the gradient of the K selected logits where the gates are
 * r3_replay_gate's softmax of them.  dYp, dgates and dz may each be NULL, but
 * not all three; Yp is needed (and read) for dgates and dz only.  dYp may be
 * Yp itself, and dgates or dz may be gates itself (not a part of it); otherwise
 * no output may share bytes with another array.
 *
 * r3_permute_backward: dx[t] = add[t] + sum_j dXp[inv_perm[t*K+j]], j
 * ascending, f32 sums, one rounding.  dXp [T*K,d], dx [T,d], add [T,d] (act) or
 * NULL; add is for what else reaches x (the router's dz W_r^T, a residual), and
 * may be dx itself (not a part of it); dx may share no bytes with another array.
 * Both refuse arrays that do (R3_ERR_INVALID_ARG).
 *
 * A token's results are the same bits whatever other tokens the call has.
 * A row outside [0, T*K) in inv_perm (a bad record) is left out: nothing is
 * written for the slot, it adds nothing and its dgates is 0.  desc->flags and
 * the record's fields are ignored.  No workspace.  R3_ERR_UNSUPPORTED where
 * T * ceil(d * sizeof(act) / 1024) exceeds 2^24.
 */
int r3_combine_backward(const r3_layer_desc *desc, const void *dy, const void *Yp, const float *gates,
                        const int32_t *inv_perm, void *dYp, float *dgates, float *dz, void *stream);
int r3_permute_backward(const r3_layer_desc *desc, const void *dXp, const int32_t *inv_perm,
                        const void *add, void *dx, void *stream);

/*
 * The replayed forward in one call (Section 4.1: router logits, replay gate,
 * and the replay-output equation y = sum_i g_i E_i(x) over the recorded
 * experts).  Same results as r3_replay_gate, r3_permute (without the gathered
 * copy), r3_grouped_ffn and r3_combine in a row, to the same tolerance, with
 * the gate folded into the expert network: the first contraction's epilogue
 * stores g_r * silu(A) * B for row r (g_r the gate of the row's slot), so the
 * down projection yields the gated rows g_i E_i(x) and the combination is a
 * plain sum of each token's K rows (j ascending, f32, one rounding).  The
 * gradient of W_down then finds its row operand ready, and the backward
 * neither forms g * dy per slot nor reads the expert outputs.
 * Outputs: y [T,d]; gates [T,K]; counts, offsets, inv_perm, perm as
 * r3_permute; H [T*K,F] = g * silu(A) * B (NOT r3_grouped_ffn's H); FA_save,
 * FB_save [T*K,F] as r3_grouped_ffn (both NULL: forward only); Yp [T*K,d] =
 * the gated rows.  logits_out, agree_out, status_word: as r3_replay_gate and
 * r3_permute.  ws: r3_workspace_bytes(desc, R3_OP_FORWARD).  desc->flags is
 * ignored.  To differentiate, pass these tensors to r3_moe_backward with
 * desc->flags = R3_FLAG_GATED_H.  Needs T*d*sizeof(act) < 2^31.
 */
int r3_moe_forward(const r3_layer_desc *desc, const void *x, const void *W_r, const float *bias,
                   const void *idx, const void *W_gate, const void *W_up, const void *W_down,
                   void *y, float *gates, int32_t *counts, int32_t *offsets, int32_t *inv_perm,
                   int32_t *perm, void *Yp, void *H, void *FA_save, void *FB_save,
                   float *logits_out, int64_t *agree_out, int32_t *status_word, void *ws,
                   size_t ws_bytes, void *stream);

/*
 * Backward of the replayed layer (Section 4.1, purpose (b): the gradient still
 * reaches the router logits through the softmax; the recorded mask is a
 * constant).  Given dy [T,d] act and the forward's tensors (FA, FB, H as
 * r3_grouped_ffn saved them), writes the gradient of sum(dy*y):  dx [T,d] act;
 * dW_r [d,E], dW_gate, dW_up [E,d,F], dW_down [E,F,d] f32;  dbias [E] f32 or
 * NULL.  accumulate = 0 overwrites the weight gradients, 1 adds to them.
 * Experts outside a token's recorded set get exactly zero router gradient from
 * that token.
 * bf16 with d and F multiples of 256: perm is
 * required and T*d*sizeof(act) < 2^31 (else R3_ERR_UNSUPPORTED).  The expert
 * gradients read the rows of dy (and of x when Xp is NULL) through perm inside
 * their tile loads, and the softmax backward takes its dot products
 * <dy_t, o_j> from the down projection's gradient GEMM (<dy, H W_down> =
 * <dy W_down^T, H>), so no per-slot copy of dy is made and Yp is not read: Yp
 * and Xp may be NULL.  Other shapes and f32 need Yp, and Xp or perm; perm is
 * not read when Xp is given (unless desc->flags asks for it, see below).
 * desc->flags = R3_FLAG_GATED_H: H and Yp are the gate-scaled tensors that
 * r3_moe_forward wrote (H = g silu(A) B, Yp = g o); perm is then required on
 * every path and Xp may be NULL on every path.
 */
int r3_moe_backward(const r3_layer_desc *desc, const void *dy, const void *x,
                    const void *W_r, const void *idx, const float *gates,
                    const int32_t *inv_perm, const int32_t *perm,
                    const int32_t *offsets, const void *Xp, const void *FA,
                    const void *FB, const void *H, const void *Yp, const void *W_gate,
                    const void *W_up, const void *W_down, void *dx, float *dW_r,
                    float *dW_gate, float *dW_up, float *dW_down, float *dbias,
                    int accumulate, void *ws, size_t ws_bytes, void *stream);

/*
 * Routing differences between two records of the same tokens (Section 3.2:
 * router-level, token-level and sequence-level comparison).  idx_a, idx_b:
 * device records of L layers, dtype desc->idx, K ids per router in any order;
 * the ids of token t in layer l start at element l*layer_stride +
 * t*token_stride (token_stride = desc->idx_token_stride, K if 0; layer-major
 * [L][T][K]: layer_stride = T*K; token-major [T][L][K]: token stride L*K,
 * layer_stride = K).  d = K - |A n B| is the number of differing choices of
 * one router.  Outputs (device): router_hist [K+1] int64, ADDED to (clear it
 * first): routers with d = 0..K;  token_choices [T] int32: d summed over the
 * layers;  token_routers [T] int32: layers with d > 0;  seq_mean [nseq] f64
 * or NULL: mean of token_routers over tokens seq_offsets[s]..seq_offsets[s+1]
 * (device int32 [nseq+1], ascending, within [0,T]).  Only T, K, E, idx and
 * idx_token_stride of desc are used.  All counts are exact.
 */
int r3_routing_diff(const r3_layer_desc *desc, int L, const void *idx_a, const void *idx_b,
                    int64_t layer_stride, const int32_t *seq_offsets, int nseq,
                    int64_t *router_hist, int32_t *token_choices, int32_t *token_routers,
                    double *seq_mean, void *stream);

/*
 * Policy discrepancy over n response tokens (Section 3.1): from the float32
 * log-probabilities of the sampled tokens under the training engine
 * (logp_train) and the inference engine (logp_infer), both device [n],
 *   *kl_out   = mean of r - 1 - log r,  r = exp(logp_train - logp_infer)
 *               (the k3 estimate of KL(pi_train || pi_infer), "KL Divergence
 *               Estimation"; evaluated in f64, fixed summation order),
 *   frac_out[i] = share of tokens with max(r, 1/r) > tau[i] (the extreme token
 *               distribution function F(tau)); the test |log r| > log tau is
 *               taken in float32 on the float32 difference, with
 *               log tau = float32(log(float64(tau))).
 * tau: HOST pointer, ntau <= 8 values >= 1 (read during the call); kl_out,
 * frac_out: device f64.  ws: device workspace of r3_policy_workspace_bytes().
 */
int r3_policy_discrepancy(int64_t n, const float *logp_train, const float *logp_infer, int ntau,
                          const float *tau, double *kl_out, double *frac_out, void *ws,
                          size_t ws_bytes, void *stream);
size_t r3_policy_workspace_bytes(void);

/*
 * Log-probabilities of given tokens under a row of logits each, with entropy
 * and the most probable alternatives: what the recompute and update stages
 * need of the model's head, and r3_policy_discrepancy's input.
 * logits: device [n, V], row i at logits + i*ld elements (ld >= V; rows may
 * start at any element), dtype R3_BF16 or R3_F32.  scale = 1 / temperature, in
 * [1e-6, 1e6].  With m = max_v z_v, S = sum_v exp(scale (z_v - m)) and
 * l_v = scale (z_v - m) - log S, row i's outputs (f32, each may be NULL, but
 * not all) are
 *   logp[i] = l_target[i],  entropy[i] = -sum_v exp(l_v) l_v,
 *   stats[i] = {m, S} ([n,2]; what r3_token_logprobs_backward reads),
 *   top_logp[i], top_id[i] ([n,top]): the `top` largest l_v, descending, and
 *     their ids; ties go to the lower id, -0 equals +0.
 * target: device int32 [n], or NULL (every row counts; logp must be NULL).
 * Row i is left out if target[i] is -1 (prompt, padding): its logits do not
 * matter, its logp, entropy and stats are 0 and it has no alternatives.  Other
 * values outside [0, V) do the same and set R3_DATA_IDX_RANGE.
 * A logit of -inf is a masked token: probability 0, logp -inf, never an
 * alternative (missing ones: id -1, logp -inf).  The lowest finite value is an
 * ordinary logit.  A row of nothing but -inf: logp -inf, entropy 0, stats
 * {-inf, 0}.  A NaN or +inf in a row sets R3_DATA_NONFINITE and makes its
 * floating outputs NaN and its ids -1.
 * No logp is above 0, no entropy below 0, whatever rounding does.
 * Sums are f32.  With more than 256 rows, and for V <= 4096, a row's results are
 * the same bits whatever other rows the call has (where the same outputs are
 * asked for and the row starts at the same place of a 16-byte unit).  Fewer,
 * longer rows get more threads, and up to 128 rows of 256 KB and more are cut
 * over several work-groups and joined by a second launch: their last bits can
 * depend on n.
 * top <= R3_MAX_TOP; 0: top_logp and top_id are not read.  n = 0 is a no-op.
 * n < 2^31, V < 2^31 - 65536, n * ld <= 2^48, else R3_ERR_UNSUPPORTED.
 * ws: device workspace of r3_token_logprobs_workspace_bytes(n, V, top) (0 is
 * possible; then, and for bf16 rows of fewer than 131072 logits, which are not
 * cut, ws may be NULL).
 * No output, nor ws, may lie between another array's first element and its last,
 * padding of the rows included (R3_ERR_INVALID_ARG).
 *
 * r3_token_logprobs_backward: the gradient of sum_i (dlogp[i] logp[i] +
 * dentropy[i] entropy[i]) with respect to the logits,
 *   dlogits[i,v] = scale ([v = target[i]] dlogp[i]
 *                         - exp(l_v) (dlogp[i] + dentropy[i] (l_v + entropy[i]))),
 * from the forward's logits, target, scale, stats and entropy.  dlogp, dentropy
 * [n] f32: one may be NULL (then zero); entropy is needed with dentropy, target
 * with dlogp.  dlogits: [n, V] of the logits' dtype, row i at dlogits + i*ldd,
 * one rounding; columns past V are not written.  Rows left out and rows of
 * nothing but -inf get zeros; a masked token gets [v = target] dlogp scale.
 * dlogits may be logits itself with ldd = ld; otherwise no array that is read may
 * lie between dlogits' first element and its last (R3_ERR_INVALID_ARG).
 */
#define R3_MAX_TOP 32
size_t r3_token_logprobs_workspace_bytes(int64_t n, int64_t V, int top);
int r3_token_logprobs(int64_t n, int64_t V, int dtype, const void *logits, int64_t ld, float scale,
                      const int32_t *target, float *logp, float *entropy, float *stats, int top,
                      float *top_logp, int32_t *top_id, int32_t *status_word, void *ws, size_t ws_bytes,
                      void *stream);
int r3_token_logprobs_backward(int64_t n, int64_t V, int dtype, const void *logits, int64_t ld, float scale,
                               const int32_t *target, const float *stats, const float *entropy,
                               const float *dlogp, const float *dentropy, void *dlogits, int64_t ldd,
                               void *stream);

/*
 * Clipped policy loss over packed sequences, and its gradient: between
 * r3_token_logprobs, whose logp and entropy it reads, and
 * r3_token_logprobs_backward, which takes its dlogp and dentropy.
 * n tokens; sequence q has tokens seq_start[q] .. seq_start[q+1]-1 (device int32
 * [nseq+1], ascending, within [0,n]; NULL: one sequence of all n, nseq ignored).
 * Token i is live if it is in a sequence and target[i] >= 0 (target NULL: all
 * are); what the other arrays hold for the rest does not matter.
 * For a live token with advantage A (advantage [n], or [nseq] with
 * R3_FLAG_SEQ_ADVANTAGE), all f32:
 *   d = logp - logp_old (logp_old NULL: it is logp, d = 0);  R3_RATIO_SEQUENCE:
 *       the mean of that over the sequence's live tokens;    r = exp(d)
 *   used = min(r, 1 + clip_high) if A > 0, max(r, 1 - clip_low) if A < 0, and in
 *       the latter case at most dual_clip unless that is 0
 *   w = min(exp(logp_old - logp_infer), weight_cap), a constant; 1 without logp_infer
 *   k = exp(q) - 1 - q, q = logp_ref - logp
 *   l = -w used A + kl_coef k - entropy_coef entropy
 *   loss = sum_i nu_i l_i;  nu = scale / live tokens (R3_MEAN_TOKENS), scale /
 *       (sequences with live tokens * the sequence's live tokens)
 *       (R3_MEAN_SEQUENCES), scale (R3_SUM)
 *   dlogp = nu (-w A r [used = r] + kl_coef (1 - exp(q))); R3_RATIO_SEQUENCE: the
 *       first part is the mean over the sequence's live tokens.  A token that
 *       clipping holds, or whose A is 0, adds nothing to it.
 *   dentropy = -entropy_coef nu
 * Borders are compared in 64 bits.  Tokens that are not live get 0.
 * stats [8] f32: loss, sum nu (-w used A), sum nu k / scale, sum nu entropy /
 * scale, share of live tokens that clipping holds, mean w, live tokens, sequences
 * with live tokens (shares and means of nothing: 0).  Sums are made in 64 bits.
 * kl_coef needs logp_ref, entropy_coef needs entropy, unless they are 0: then the
 * term is in the statistics alone, if its array is there.  dlogp,
 * dentropy [n]: may be NULL.  A live token whose loss or gradient is not finite
 * sets R3_DATA_NONFINITE.  0 <= clip_low <= 1, clip_high >= 0, dual_clip 0 or > 1,
 * weight_cap > 0; they and the coefficients finite, but for weight_cap, which may
 * be infinite.  n = 0 gives stats of 0.  n, nseq < 2^31 - 2^16.
 * No output, nor ws, may share bytes with another array.
 * ws: device workspace of r3_policy_loss_workspace_bytes(desc), 256-byte aligned;
 * enough with seq_start and without.
 */
enum { R3_RATIO_TOKEN = 0, R3_RATIO_SEQUENCE = 1 };
enum { R3_MEAN_TOKENS = 0, R3_MEAN_SEQUENCES = 1, R3_SUM = 2 };
enum { R3_FLAG_SEQ_ADVANTAGE = 1 };   /* r3_policy_desc.flags */
typedef struct r3_policy_desc {
    int64_t n;
    int32_t nseq, ratio, norm, flags;
    float clip_low, clip_high, dual_clip, weight_cap, kl_coef, entropy_coef, scale;
} r3_policy_desc;
size_t r3_policy_loss_workspace_bytes(const r3_policy_desc *desc);
int r3_policy_loss(const r3_policy_desc *desc, const float *logp, const float *logp_old, const float *logp_infer,
                   const float *logp_ref, const float *entropy, const float *advantage, const int32_t *target,
                   const int32_t *seq_start, float *dlogp, float *dentropy, float *stats, int32_t *status_word, void *ws,
                   size_t ws_bytes, void *stream);

/*
 * Load-balance loss of the recorded routing with the router's z-loss, and the
 * gradient of the router's logits (r3_replay_gate's logits_out).  Groups: the
 * nseq sequences of seq_start (as for r3_policy_loss), or with NULL the whole
 * batch.  Of a group with N tokens:
 *   counts[e] = slots of its tokens that the record gives expert e   (int32)
 *   probs[e]  = mean over its tokens of p_te, p_t = softmax(logits[t])   (f32)
 *   f_e = E counts[e] / (K N)
 * loss = balance_coef * balance + z_coef * z, where balance is the mean over the
 * groups that hold tokens of sum_e f_e probs[e] and z the mean over their tokens
 * of the squared log-sum-exp of the logits.  f is a constant:
 *   dlogits[t,e] = balance_coef / (groups N) p_te (f_e - sum_i f_i p_ti)
 *                  + 2 z_coef / tokens lse_t p_te
 * (a user's router then has dx += dlogits W_r^T, dW_r += x^T dlogits).
 * Outputs: counts, probs [groups,E]; stats [3] f32: loss, balance, z; dlogits
 * f32, row t at dlogits + t*ldd.  counts, probs, dlogits may be NULL.  Tokens of
 * no group get zeros in dlogits.  Groups without tokens have counts and probs 0.
 * A logit of -inf is a masked expert: probability and gradient 0.  A row of
 * nothing but -inf has probabilities, gradient and lse of 0 and counts as a
 * token.  A NaN or +inf in a row makes its gradient NaN and sets
 * R3_DATA_NONFINITE; an id >= E is not counted and sets R3_DATA_IDX_RANGE.
 * Of desc T, E, K, idx and idx_token_stride are used.  Rows are ld elements apart
 * (ld, ldd >= E; they may start at any element).  dlogits may be logits itself
 * with ldd = ld; otherwise no output, nor ws, may lie between another array's
 * first element and its last.  T * max(ld, ldd) <= 2^48, nseq < 2^31 - 2^16.
 * A token's gradient is the same bits whatever the other groups' logits are.
 * Exponential, logarithm and reciprocal are the hardware's, each within a unit in
 * the last place; sums over a row are f32, those over tokens 64 bits but for the
 * probabilities' of a piece of a group.
 * ws: device workspace of r3_balance_loss_workspace_bytes(), 256-byte aligned.
 */
size_t r3_balance_loss_workspace_bytes(const r3_layer_desc *desc, int nseq);
int r3_balance_loss(const r3_layer_desc *desc, const float *logits, int64_t ld, const void *idx, const int32_t *seq_start, int nseq,
                    float balance_coef, float z_coef, int32_t *counts, float *probs, float *stats, float *dlogits, int64_t ldd,
                    int32_t *status_word, void *ws, size_t ws_bytes, void *stream);

/*
 * Orthogonalised updates: a batch of gradients (dW_gate, dW_up, dW_down or dW_r
 * as r3_moe_backward writes them, or momenta of them) by Newton-Schulz
 * products, for optimisers whose update keeps a gradient's singular vectors and
 * levels its singular values.  For each of `batch` matrices G [rows,cols],
 *   X = G / (|G|_F + eps),  `steps` times  X <- a X + (b A + c A A) X,  A = X X^T,
 *   out = scale X,
 * which takes every singular value s of G to scale f(f(... s / (|G|_F + eps))),
 * f(x) = a x + b x^3 + c x^5 (a tall matrix is worked on transposed; the result
 * is the same).  coef: HOST pointer to {a, b, c}, or NULL for
 * {3.4445, -4.775, 2.0315}, with which singular values of 0.002 and more come
 * to lie in [0.68, 1.21] after five steps.
 * G and out: dense [batch, rows, cols], dtype R3_BF16 or R3_F32 each.  The
 * products' operands are f16 numbers with f32 sums; for dtype_out R3_F32, and
 * where rows or cols are at most 128, they are sums of two such, 22 bits.
 * Errors of five steps, relative to each result in the Frobenius norm, beside a
 * bf16 result's own rounding (1.7e-3): bf16 1e-3 where many directions count, 8e-3
 * where G has one to four (it is spread over all the others: 2e-3 in the 2-norm),
 * with a side of at most 128 less than 1e-4; f32 3e-6, and 1e-4 with one to four
 * directions (6e-6 and 2e-5 in the 2-norm), as the same steps in f32 have.
 * A matrix of zeros gives zeros.  A NaN or an infinity in a matrix makes its
 * result NaN and sets R3_DATA_NONFINITE; the other matrices are as without it.
 * A matrix's bits do not depend on what the call's other matrices hold, but may
 * on how many they are.
 * rows, cols <= 32768, batch * rows * cols <= 2^46, and coefficients with which
 * no element of X, A or b A + c A A (|G|_2 <= |G|_F bounds them), nor a or
 * a + b + c, can leave (-15, 15), else R3_ERR_UNSUPPORTED.
 * 1 <= steps <= R3_MAX_STEPS, eps >= 0.
 * out may be G itself if the types are the same; otherwise no output, nor ws,
 * may share bytes with another array.  batch = 0 is a no-op.
 * ws: device workspace of r3_orthogonalize_workspace_bytes(), 256-byte aligned.
 */
#define R3_MAX_STEPS 64
size_t r3_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, int dtype_out);
int r3_orthogonalize(int64_t batch, int64_t rows, int64_t cols, int dtype_in, const void *G, int dtype_out, void *out, int steps,
                     const float *coef, float eps, float scale, int32_t *status_word, void *ws, size_t ws_bytes, void *stream);

/*
 * Router-mask cache (Section 4.2: routing masks stored with the KV cache per
 * layer and token prefix, so that a prefix that hits the cache brings its masks
 * and is not prefilled again).  Masks live in `pages`, a device pool
 * [num_pages][P][L][K] of ids (idx_dtype R3_IDX_U8 / R3_IDX_U16): P tokens per
 * page, one token's L*K ids contiguous.  block_table: device int32
 * [nseq][max_blocks]; entry b of sequence s is the page that holds its tokens
 * b*P .. b*P+P-1 (negative: none).  A prefix shared by several sequences is the
 * same page ids in their rows; the library never allocates or frees pages.
 *
 * r3_mask_cache_append: ids of n new tokens (device; element (l, i, k) at
 * idx_new[l*layer_stride + i*token_stride + k], so both [n][L][K] and the
 * [L][n][K] that L calls of r3_record_topk leave are accepted) go to the slot of
 * token position[i] (0-based) of sequence seq_id[i] (device int32 [n]).  Two
 * entries that name the same slot race.
 *
 * r3_mask_cache_gather: the layer-major record out[L][T][K] of a packed batch:
 * sequence s owns tokens seq_start[s] .. seq_start[s+1]-1 (device int32
 * [nseq+1], ascending from 0 to T) and its j-th token is read from page
 * block_table[s][j / P], slot j % P.  The result is what r3_replay_gate,
 * r3_permute and r3_moe_backward take as idx, layer by layer.
 *
 * A token whose sequence, position or page is out of range is skipped by
 * append and zero-filled by gather, and R3_DATA_CACHE_ADDR is set in
 * *status_word (device, may be NULL); nothing is accessed out of bounds.
 * Pure copies: results are bit-exact.  pages, idx_new, out: aligned to the id
 * size.  n = 0 / T = 0 are no-ops.
 */
int r3_mask_cache_append(int idx_dtype, int L, int K, int P, void *pages, int64_t num_pages,
                         const int32_t *block_table, int nseq, int max_blocks, int64_t n,
                         const int32_t *seq_id, const int32_t *position, const void *idx_new,
                         int64_t layer_stride, int64_t token_stride, int32_t *status_word,
                         void *stream);
int r3_mask_cache_gather(int idx_dtype, int L, int K, int P, const void *pages, int64_t num_pages,
                         const int32_t *block_table, int nseq, int max_blocks,
                         const int32_t *seq_start, int64_t T, void *out, int32_t *status_word,
                         void *stream);

#ifdef __cplusplus
}
#endif
#endif /* R3_H */
