/*
 * nm_token_scores.h -- C ABI of what a decoder's class scores say about tokens (gfx950): log-probabilities of given tokens, entropies, the
 * likeliest alternatives, and the gradient with respect to the scores.
 *
 * The paper's recipes train a decoder on the log-probabilities of its targets and decode by the likeliest classes (Section 4.1.1).
 *
 *   lse[b,u]     = log sum_v exp(scores[b,v,u]);   logq[v] = scores[b,v,u] - lse[b,u];   q = exp(logq)
 *   logp[b,u]    = logq[targets[b,u]];   0 where the target is outside [0,V) (no token is asked for)
 *   entropy[b,u] = -sum_v q[v] * logq[v]      (a class at -infinity adds nothing)
 *   top_ids[b,i,u], top_logp[b,i,u]: the class of the i-th largest score and its logq, i < top; of equal scores the lower class first; a NaN
 *     counts as -infinity there
 *   dscores[b,v,u] = dlogp[b,u] * ([v = targets[b,u]] - q[v]) - dentropy[b,u] * q[v] * (logq[v] + entropy[b,u])
 *     (without a target as if dlogp were 0)
 *   at u >= lengths[b]: logp, entropy, lse, top_logp 0, top_ids -1, dscores 0
 *   a place where all classes are at -infinity: lse and the logp of a target -infinity, entropy 0, top_logp -infinity, dscores 0
 *
 * Conventions are those of nm_conv1d.h (device pointers the caller owns, one stream, enqueue only, argument errors before
 * any device call, deterministic results), with these additions:
 *  - dtype (NM_BF16 or NM_F32) is the storage type of scores; that of dscores is grad_dtype.  Everything else is float, sums too.  Scores are
 *    sums of anything, of any finite size: logits, or log-probabilities as nm_decoder_logsoftmax_fwd gives them.  +infinity gives NaN.  A
 *    log-probability below float's range is -infinity.
 *  - targets [B][U]: int32 (target_bytes 4) or int64 (8).  lengths [B] int32, optional (NULL); any values are taken, clipped to [0,U].
 *    scores are not used at u >= lengths[b], whatever they hold.
 *  - top is at most 16 and at most V.
 *  - workspace: nm_token_scores_workspace_bytes bytes, 256-byte aligned (NULL where that is 0).
 *  - B * V * U must be below 2^31, V at most 2^31 - 2^16 - 1, U at most 2^29.
 */
#ifndef NM_TOKEN_SCORES_H
#define NM_TOKEN_SCORES_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { NM_MOST_ALTERNATIVES = 16 };

/* Bytes of workspace of nm_token_scores_fwd; 0 for invalid arguments too.  Host only. */
size_t nm_token_scores_workspace_bytes(int B, int V, int U, int top, int dtype);

/* Forward.  scores [B][V][U] in;  logp (with targets, else NULL), entropy, lse [B][U] out, each may be NULL but one of them or top;
 * top_ids [B][top][U] int32 and top_logp [B][top][U] out (NULL where top is 0). */
int nm_token_scores_fwd(int B, int V, int U, const void *scores, const void *targets, int target_bytes, const int *lengths, int top,
                        float *logp, float *entropy, float *lse, int *top_ids, float *top_logp, int dtype, void *workspace,
                        size_t workspace_bytes, void *hip_stream);

/* Backward.  lse and entropy as the forward pass gave them (entropy is read only with dentropy; up to a magnitude of 4096 q has lse's rounding,
 * beyond that the call sums over the classes again, once for each workgroup that has such a place); dlogp with targets, dentropy: one of
 * them at least.  dscores [B][V][U] out, written whole. */
int nm_token_scores_bwd(int B, int V, int U, const void *scores, const void *targets, int target_bytes, const int *lengths,
                        const float *lse, const float *entropy, const float *dlogp, const float *dentropy, void *dscores, int dtype,
                        int grad_dtype, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_TOKEN_SCORES_H */
