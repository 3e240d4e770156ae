/*
 * hmoe_lm.h -- C ABI of the operators around the hard mixture that answer with its model and adapt
 * it: log-probabilities of given tokens, the whole mixture layer for a few samples, low-rank
 * adapters beside a shared projection.  A "token" is an entry of the decoder's vocabulary, a tag.
 *
 * The conventions are hmoe.h's: device pointers, the caller's workspace, one stream, no
 * allocation, no state and no host synchronisation, argument errors before any launch
 * (hmoe_last_error), HMOE_F32 or HMOE_BF16 data with sums in fp32 or wider, calls that can be
 * captured into HIP graphs.
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
 *   scale > 0 (an inverse temperature), finite.  token int32[n] or NULL (logp is then not written).
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
 * masked entries and rows of nothing else get 0.
 *   stat and entropy are the forward's.  g_logp, g_entropy float[n], either may be NULL (zeros); entropy
 *   is needed with g_entropy, token with g_logp.
 *   dlogits [n][vocab] in dtype dt, rows ld_out >= vocab elements apart; it may be logits itself (without
 *   anchors, ld_out = ld) and overlap it in no other way.  One pass, no workspace. */
int hmoe_token_logprob_backward(const void* logits, int64_t ld, const float* anchor, hmoe_dtype_t dt, int64_t n,
                                int32_t vocab, float scale, const int32_t* token, const float* stat,
                                const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits,
                                int64_t ld_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* HMOE_LM_H_ */
