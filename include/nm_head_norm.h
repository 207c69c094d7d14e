/*
 * nm_head_norm.h -- C ABI of the norms of queries and keys, head by head, with their rotation by position in the same pass
 * (gfx950): forward and backward for training, and a form for serving that writes keys and values into a paged cache.
 *
 * x holds the heads' channels of a projection's output, [batch][channels][tokens]: first `heads` query heads, then `kv_heads` key heads, of
 * D channels each.  For every head and token, with w = q_weight or k_weight:
 *
 *   n[d] = x[d] * r * w[d],  r = 1/sqrt(mean_d x[d]^2 + eps)     with NM_HEADS_NORM (w NULL: 1), else n = x
 *   out: the first `rot` channels are turned in pairs by position * freqs[i], i < rot/2, the others are n:
 *     out[a] = n[a] * cos - n[b] * sin;   out[b] = n[b] * cos + n[a] * sin
 *     (a, b) = (i, i + rot/2), or (2i, 2i + 1) with NM_HEADS_PAIRS
 *   position: positions[b,u], or u
 *
 * Backward, from dout:  dn = dout turned back;  dw[d] = sum over tokens, items and heads of dn[d] * x[d] * r;
 *   dx[d] = r * (w[d] * dn[d] - x[d] * r * mean_e(w[e] * dn[e] * x[e] * r)), or dn without a norm.
 *
 * The cache consists of `pages` pages of page_size tokens: k_cache [pages][kv_heads][page_size][D], v_cache [pages][kv_heads][D][page_size].
 * A sequence's p-th token lies on page page_table[b][p / page_size], in row p % page_size.  lengths[b] is the number of tokens that
 * sequence b has with the new ones, q_lengths[b] (NULL: U) of which are new: the u-th of them is token lengths[b] - q_lengths[b] + u, and that
 * is its position too.
 *
 * Conventions are those of nm_conv1d.h (device pointers the caller owns, one stream, enqueue only, argument errors before
 * any device call, deterministic results), with these additions:
 *  - dtype (NM_BF16 or NM_F32) is the storage type of x, out, their gradients and the cache.  Weights and their gradients are float, sums
 *    and norms float32; freqs is double, and angles are made in double: positions of any size keep their digits.
 *  - a tensor is [batch][channels][tokens] with dense rows; *_stride is the distance of its batch items in elements, so that x may be
 *    the first part of a projection's output.
 *  - lengths, q_lengths and positions are int32; any values are taken (lengths clipped to [0,U], q_lengths too, lengths of
 *    a cache at 0).  x and dout are not used at tokens behind an item's end, whatever they hold; out, dx and the returned queries are 0 there.
 *  - a token whose place in the cache does not exist (before 0, behind max_pages * page_size, on a page outside [0, pages)) is not
 *    written.  No two tokens of a call may have the same place.  Everything else in the cache stays as it was.
 *  - D is even and at most 128; rot is even and at most D.  A tensor spans fewer than 2^40 elements, an item of it fewer than 2^31, a
 *    head of an item less than 4 GiB.
 *  - without an eps the norm of a head of zeros is NaN.
 */
#ifndef NM_HEAD_NORM_H
#define NM_HEAD_NORM_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* flags */
enum { NM_HEADS_NORM = 1u, NM_HEADS_PAIRS = 2u };

/* Forward.  x [B][(heads+kv_heads)*D][U] in, q_weight, k_weight [D] in or NULL, freqs [rot/2] in (NULL where rot is 0), positions [B][U]
 * and lengths [B] in or NULL;  out like x, elsewhere. */
int nm_head_norm_fwd(int B, int heads, int kv_heads, int D, int U, const void *x, long long x_stride, const float *q_weight,
                     const float *k_weight, float eps, const double *freqs, int rot, const int *positions, const int *lengths, void *out,
                     long long out_stride, unsigned flags, int dtype, void *hip_stream);

/* Bytes of workspace of nm_head_norm_bwd; 0 for invalid arguments.  Host only. */
size_t nm_head_norm_bwd_workspace_bytes(int B, int heads, int kv_heads, int D, int U, int dtype);

/* Backward.  dout and x in (x as of the forward call);  dx out, written whole;  dq_weight, dk_weight [D] out or NULL (each needs its weight).
 * workspace: 256-byte aligned; only where a weight's gradient is wanted, else NULL will do. */
int nm_head_norm_bwd(int B, int heads, int kv_heads, int D, int U, const void *dout, long long dout_stride, const void *x,
                     long long x_stride, const float *q_weight, const float *k_weight, float eps, const double *freqs, int rot,
                     const int *positions, const int *lengths, void *dx, long long dx_stride, float *dq_weight, float *dk_weight,
                     unsigned flags, int dtype, void *workspace, size_t workspace_bytes, void *hip_stream);

/* The serving form.  x [B][(heads+2*kv_heads)*D][U] in (queries, keys, values), page_table [B][max_pages], lengths [B], q_lengths [B] or NULL
 * in;  q_out [B][heads*D][U] out;  k_cache, v_cache in and out.  page_size: 16, 32, 64, 128 or 256. */
int nm_head_norm_cache(int B, int heads, int kv_heads, int D, int U, const void *x, long long x_stride, const float *q_weight,
                       const float *k_weight, float eps, const double *freqs, int rot, int pages, int page_size, const int *page_table,
                       int max_pages, const int *lengths, const int *q_lengths, void *k_cache, void *v_cache, void *q_out,
                       long long q_stride, unsigned flags, int dtype, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_HEAD_NORM_H */
