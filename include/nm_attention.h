/*
 * nm_attention.h -- C ABI of cross attention from a decoder's tokens to an encoder's states (gfx950), forward and backward.
 *
 * The acoustic encoder (paper Section 4.1.1) turns an utterance into a sequence of T states; an attention decoder writes
 * the transcript token by token and looks at all states for every token.  Both sequences have lengths of their own.
 * Activations are channel-major like the encoder's ([batch][channels][time]), so that the projections in front of and
 * behind this operator are its 1x1 convolutions; the heads of a tensor lie side by side in its channels.
 *
 *   G      = heads / kv_heads;  head h reads the keys and values of kv head h / G
 *   s[u,t] = scale * sum_d q[h*D+d, u] * k[(h/G)*D+d, t]
 *   frames that token u may look at: lo <= t < hi, with lo = 0, hi = T; with lengths hi = min(hi, lengths[b]);
 *     with windows lo = max(lo, windows[b,u,0]) and hi = min(hi, windows[b,u,1]); none where u >= q_lengths[b]
 *   lse[h,u] = log sum_t exp(s[u,t]);   p = exp(s - lse);   o[h*D+d, u] = sum_t p[u,t] * v[(h/G)*D+d, t]
 *   a token without frames: o = 0, lse = -infinity
 * and for the gradient do of o
 *   dv = sum over the heads of a kv head and their tokens of p * do;   dp = sum_d do * v;   delta[u] = sum_d do * o
 *   ds = p * (dp - delta);   dq = scale * sum_t ds * k;   dk = scale * sum over those heads and tokens of ds * q
 *   (a token without frames has dq = 0 and adds nothing to dk and dv; tokens at u >= q_lengths[b] are not read)
 *
 * Conventions are those of nm_conv1d.h (device pointers the caller owns, one stream, enqueue only, argument errors before
 * any device call, deterministic results), with these additions:
 *  - dtype (NM_BF16 or NM_F32) is the storage type of q, k, v, o and their gradients; lse is float.  Sums, maxima and
 *    probabilities are float32; in NM_BF16 mode p is rounded to bfloat16 as an operand of the second product, ds to two such terms
 *    (outputs and gradients differ from 64 bits by 1.1 to 1.4 times what rounding the results alone would make; NM_F32 has no such rounding).
 *  - a tensor is [batch][channels][positions] with dense rows; *_stride is the distance of its batch items in elements
 *    (at least channels * positions, so that keys and values may be the halves of one projection's output).
 *  - D is at most 128; kv_heads divides heads; a tensor spans fewer than 2^40 elements, an item of it fewer than 2^31.  Larger batches
 *    than a launch can have work items for (from B * kv_heads = 2^23, B * heads * ceil(U/32) or B * kv_heads * ceil(T/32) = 2^24 on) are
 *    unsupported.
 *  - lengths, q_lengths [B] int32 and windows [B][U][2] int32 are optional (NULL); any values are taken, clipped to the
 *    sequence.  Keys and values at t >= lengths[b] are not used, whatever they hold (NaN included); dk and dv are 0 there.
 *    Those below it that are outside a token's window count for other tokens: they have to be finite.  So have q and dout at
 *    u < q_lengths[b], also of tokens whose window leaves them nothing.
 *  - U = 1 is the form for single tokens; hypotheses of a beam search that share an utterance are its U tokens.
 *  - workspace: nm_cross_attn_workspace_bytes bytes, 256-byte aligned (NULL where that is 0).
 */
#ifndef NM_ATTENTION_H
#define NM_ATTENTION_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { NM_OP_ATTN_FWD = 16, NM_OP_ATTN_BWD = 17 };

/* Bytes of workspace of nm_cross_attn_fwd / nm_cross_attn_bwd; 0 for invalid arguments.  Host only. */
size_t nm_cross_attn_workspace_bytes(int op, int B, int heads, int kv_heads, int D, int U, int T, int dtype);

/* Forward.  q [B][heads*D][U], k, v [B][kv_heads*D][T] in;  o [B][heads*D][U] out;  lse [B][heads][U] float out, or NULL. */
int nm_cross_attn_fwd(int B, int heads, int kv_heads, int D, int U, int T, const void *q, long long q_stride,
                      const void *k, long long k_stride, const void *v, long long v_stride, const int *lengths,
                      const int *q_lengths, const int *windows, float scale, void *o, long long o_stride, float *lse,
                      int dtype, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Backward.  dout = the gradient of o; o and lse as the forward pass gave them; lengths, q_lengths, windows and scale as there.
 * dq [B][heads*D][U], dk, dv [B][kv_heads*D][T] out, written whole. */
int nm_cross_attn_bwd(int B, int heads, int kv_heads, int D, int U, int T, const void *dout, long long dout_stride,
                      const void *q, long long q_stride, const void *k, long long k_stride, const void *v,
                      long long v_stride, const void *o, long long o_stride, const float *lse, const int *lengths,
                      const int *q_lengths, const int *windows, float scale, void *dq, long long dq_stride, void *dk,
                      long long dk_stride, void *dv, long long dv_stride, int dtype, void *workspace,
                      size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_ATTENTION_H */
