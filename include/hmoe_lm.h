/*
 * hmoe_lm.h -- C ABI of the operators around the hard mixture that answer with its model and adapt
 * it: log-probabilities of given tokens, the whole mixture layer for a few samples, low-rank
 * adapters beside a shared projection.  A "token" is an entry of the decoder's vocabulary, a tag.
 *
 * The conventions are hmoe.h's: device pointers, the caller's workspace, one stream, no
 * allocation, no state and no host synchronisation, argument errors before any launch
 * (hmoe_last_error), HMOE_F32 or HMOE_BF16 data with sums in fp32 or wider, calls that can be
 * captured into HIP graphs.  Workspaces are 16-byte aligned, too (HMOE_ESHAPE).
 */
#ifndef HMOE_LM_H_
#define HMOE_LM_H_

#include "hmoe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ token log-probabilities */

/* Log-probabilities of given tokens, entropies and the most probable alternatives of n rows of
 * logits, in one pass over them.  With z_v = scale * logit_v, for row i:
 *   logp[i]     = z_t - ln sum_v exp z_v,  t = token[i]; a token outside [0, vocab) marks a row
 *                 without one: 0
 *   entropy[i]  = -sum_v p_v ln p_v,       p = softmax(z)
 *   lse[i]      = ln sum_v exp z_v
 *   top_idx[i][q], top_logp[i][q], q < m: the m largest logits in decreasing order, equal ones in
 *                 increasing index order, and their log-probabilities
 *   stat[i]     = (max_v logit_v, ln sum_v exp(z_v - max z)), what the backward needs of the row
 *
 *   logits [n][vocab] in dtype dt, rows ld elements apart (ld >= vocab), any vocab >= 1, aligned to
 *     their element.  With anchor (float, HMOE_ANCHOR_*; then ld = vocab, a multiple of 8, and both
 *     16-byte aligned) a logit is anchor + stored value, formed in fp32, as hmoe_moe_forward keeps them.
 *   0 < scale <= 2^127 (an inverse temperature).  token int32[n] or NULL (logp is then not written).
 *   logp, entropy, lse float[n], stat float[n][2], top_idx int32[n][m], top_logp float[n][m]: each may be
 *     NULL (top_idx and top_logp if m = 0, top_logp always).  0 <= m <= min(16, vocab).
 * A logit of -inf is a masked entry: probability 0, and nothing in the entropy.  A row of nothing
 * else has lse, logp and top_logp -inf and entropy 0.  A row with NaN or +inf has NaN for all of
 * its numbers; NaN ranks last among the alternatives, whose indexes are always in [0, vocab).
 * Errors: HMOE_EINVAL (NULL logits, m, vocab, ld or scale out of range, m > 0 without top_idx),
 * HMOE_ESHAPE (anchored logits with a stride or an alignment), HMOE_EDTYPE, HMOE_EWORKSPACE. */
size_t hmoe_token_logprob_workspace(int64_t n, int32_t vocab, int32_t m, hmoe_dtype_t dt);
int hmoe_token_logprob(const void* logits, int64_t ld, const float* anchor, hmoe_dtype_t dt, int64_t n,
                       int32_t vocab, float scale, const int32_t* token, int32_t m, float* logp,
                       float* entropy, float* lse, float* stat, int32_t* top_idx, float* top_logp,
                       void* ws, size_t ws_bytes, void* stream);

/* The gradient of  sum_i g_logp[i] logp[i] + g_entropy[i] entropy[i]  with respect to the logits:
 *   dlogits[i][v] = scale * (g_logp ([v = t] - p_v) - g_entropy p_v (ln p_v + entropy))
 * with p_v = exp(scale (logit_v - stat[0]) - stat[1]).  Rows without a token take nothing from g_logp;
 * rows of masked entries alone get 0, and so do masked entries of other rows -- but for the row's own token, whose
 * entry gets scale * g_logp there, as the formula with p = 0 has it.
 *   stat and entropy are the forward's.  g_logp, g_entropy float[n], either may be NULL (zeros); entropy
 *   is needed with g_entropy, token with g_logp.
 *   dlogits [n][vocab] in dtype dt, rows ld_out >= vocab elements apart; it may be logits itself (without
 *   anchors, ld_out = ld) and overlap it in no other way.  One pass, no workspace. */
int hmoe_token_logprob_backward(const void* logits, int64_t ld, const float* anchor, hmoe_dtype_t dt, int64_t n,
                                int32_t vocab, float scale, const int32_t* token, const float* stat,
                                const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits,
                                int64_t ld_out, void* stream);

/* ------------------------------------------------------------------ mixture layer of a few samples */

/* What an expert does between its layers. */
enum {
  HMOE_ACT_RELU = 0,      /* h = max(0, W1 x + b1), W1 [K][d_hid][d_in], b1 [K][d_hid]: hmoe_moe_params_t's */
  HMOE_ACT_SILU_GATED = 1 /* h = silu(g) u, silu(g) = g / (1 + e^-g); W1 [K][2 d_hid][d_in], b1 [K][2 d_hid]: the
                           * first d_hid rows give g, the others u */
};

#define HMOE_FEW_ROWS 64  /* most rows of the entry points for a few of them */
#define HMOE_FEW_EXPERTS 8 /* most experts of a sample */
#define HMOE_FEW_WIDTH (1 << 20) /* largest d_in, d_hid and d_out */

/* A mixture layer that routes by itself.  R [K][d_in] the router's rows, r_bias float[K] or NULL; W2
 * [K][d_out][d_hid], b2 [K][d_out]; biases may be NULL; matrices and biases in dtype dt.
 * The gater of Eq. 2 over centres C is R = C, r_bias[e] = -|C_e|^2 / 2, top_k = 1: the nearest centre has the
 * largest x . C_e - |C_e|^2 / 2. */
typedef struct {
  int32_t K, d_in, d_hid, d_out, top_k;
  hmoe_dtype_t dt;
  int32_t act; /* HMOE_ACT_* */
  const void* R;
  const float* r_bias;
  const void *W1, *b1, *W2, *b2;
} hmoe_few_params_t;

/* The whole layer for 1 <= n <= HMOE_FEW_ROWS samples, for serving: no sort, no padding, an
 * expert's weights read once for every 16 samples that chose it.  For row i of X [n x d_in]:
 *   s_e = R_e . x + r_bias[e];  expert[i][0 .. top_k) = the top_k largest, in decreasing order, equal ones in
 *   increasing e (NaN ranks last);  weight[i][j] = softmax of those top_k scores;
 *   Y[i] = sum_j weight[i][j] (W2_e h + b2_e), e = expert[i][j].
 * A weight below 2^-126, the smallest normal float, is 0, and an expert of weight 0 is not evaluated: one
 * with a score of -inf (r_bias[e] = -inf: it is off) never is.  A row of nothing else has Y = 0.
 * Scores, sums, h and weights are held in fp32; the second product of bf16 data takes h as two bf16 numbers, good to
 * 2^-16 of it, and Y is rounded to bf16 once.
 *   expert int32[n][top_k], weight float[n][top_k], Y [n x d_out] in dtype dt: out.
 * 1 <= top_k <= min(HMOE_FEW_EXPERTS, K).  Errors: HMOE_EINVAL (n, K, top_k or act out of range, NULL pointer),
 * HMOE_ESHAPE (width not a multiple of 8, misaligned pointer), HMOE_EDTYPE, HMOE_EWORKSPACE. */
size_t hmoe_moe_few_workspace(const hmoe_few_params_t* p, int64_t n);
int hmoe_moe_few(const hmoe_few_params_t* p, int64_t n, const void* X, int32_t* expert, float* weight, void* Y,
                 void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ low-rank adapters */

#define HMOE_LORA_RANK 128          /* largest rank */
#define HMOE_LORA_WIDTH (1 << 21)   /* largest d_in and d_out */
#define HMOE_LORA_ROWS (1 << 28)    /* most rows */

/* A projection W [d_out][d_in] with bias b [d_out] (or NULL) that all rows share, and E adapters beside it:
 * A [E][rank][d_in], B [E][d_out][rank], scale float[E] (NULL: ones); matrices and b in dtype dt.  With
 * adapter a, or none:
 *   y = W x + b + scale[a] B_a (A_a x).
 * d_in, d_out and rank are multiples of 8 up to the limits above, 1 <= E <= 4096.  A hard mixture's experts can
 * be such adapters (one per cluster), and so can its decoders, beside one D. */
typedef struct {
  int32_t E, d_in, d_out, rank;
  hmoe_dtype_t dt;
  const void *W, *b, *A, *B;
  const float* scale;
} hmoe_lora_t;

/* For serving: n <= HMOE_FEW_ROWS rows X [n x d_in] of any mix of requests, adapter int32[n] (an id outside
 * [0, E): none); Y [n x d_out] out.  W is read once, of each adapter that is used B once and A once for every 16 of
 * its rows (and A by every workgroup, from the caches, where one row and a narrow A take one launch).  Y is rounded to
 * the data type as it is: bf16 logits have no anchors here and are good to 2^-9 of their size. */
size_t hmoe_lora_few_workspace(const hmoe_lora_t* p, int64_t n);
int hmoe_lora_few(const hmoe_lora_t* p, int64_t n, const void* X, const int32_t* adapter, void* Y, void* ws,
                  size_t ws_bytes, void* stream);

/* Many rows, in adapter order as hmoe_moe_dispatch leaves them: X_sorted [n x d_in], rows [offsets[a],
 * offsets[a + 1]) with adapter a and rows from offsets[E] on without one; offsets int32[E + 1] starts at 0.
 * perm int32[n] (slot -> sample, a permutation), or NULL: Y's rows are in slot order too.
 *   Y [n x d_out] out, sample order; rounded as above.
 *   U [n][hmoe_lora_saved_width] out, dtype dt: scale A x of every row with an adapter, for the
 *     backward, in fp32: with bf16 data as three bf16 numbers a value, in blocks of 16 values. */
int32_t hmoe_lora_saved_width(int32_t rank, hmoe_dtype_t dt);
size_t hmoe_lora_workspace(const hmoe_lora_t* p, int64_t n);
int hmoe_lora_forward(const hmoe_lora_t* p, int64_t n, const void* X_sorted, const int32_t* offsets,
                      const int32_t* perm, void* U, void* Y, void* ws, size_t ws_bytes, void* stream);

/* Gradients with respect to the adapters and the input; W, b and scale are fixed.  With V = scale B_a^T dY:
 *   dA[a] = sum over a's rows of V x^T, dB[a] = sum of dY U^T: float, A's and B's shapes, zeros for adapters
 *   without rows, sums in a fixed order;  dX [n x d_in] (dtype dt, sample order) = W^T dY + A_a^T V.
 *   dY [n x d_out] in sample order (slot order without perm).  dX, dA and dB may each be NULL.
 * Errors of the four: HMOE_EINVAL (n, E or rank out of range, NULL pointer), HMOE_ESHAPE (width not a multiple
 * of 8, misaligned pointer), HMOE_EDTYPE, HMOE_EWORKSPACE. */
int hmoe_lora_backward(const hmoe_lora_t* p, int64_t n, const void* X_sorted, const int32_t* offsets,
                       const int32_t* perm, const void* U, const void* dY, void* dX, float* dA, float* dB, void* ws,
                       size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* HMOE_LM_H_ */
