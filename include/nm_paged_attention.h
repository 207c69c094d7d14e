/*
 * nm_paged_attention.h -- C ABI of attention of new tokens over a paged cache of keys and values (gfx950): a decoding step (one token a
 * sequence), a few tokens that are checked at once, or a chunk of a prompt behind what is cached already.
 *
 * The cache is that of nm_head_norm.h: k_cache [pages][kv_heads][page_size][D], v_cache [pages][kv_heads][D][page_size], the p-th token of sequence
 * b in row p % page_size of page page_table[b][p / page_size].  It holds the new tokens' keys and values already.  lengths[b] tokens
 * has the sequence with the new ones, q_lengths[b] (NULL: U) of which are new.
 *
 *   G = heads / kv_heads;  head h reads the keys and values of kv head h / G
 *   at = lengths[b] - q_lengths[b] + u: the place of new token u, which looks at the places p with p <= at, p > at - window where window is
 *     not 0, and whose page exists (p < max_pages * page_size, page number in [0, pages))
 *   s[u,p] = scale * sum_d q[h*D+d, u] * k[p,d];   lse[h,u] = log sum_p exp(s[u,p]);   o[h*D+d, u] = sum_p exp(s[u,p] - lse) * v[p,d]
 *   a token without places, and those at u >= q_lengths[b]: o = 0, lse = -infinity
 *
 * Conventions are those of nm_conv1d.h (device pointers the caller owns, one stream, enqueue only, argument errors before
 * any device call, deterministic results), with these additions:
 *  - dtype (NM_BF16 or NM_F32) is the storage type of q, o and the cache; lse is float.  Sums, maxima and probabilities are float32; in
 *    NM_BF16 mode probabilities enter the second product as two bfloat16 terms, off by 2^-16 of themselves.
 *  - q and o are [B][heads*D][U] with dense rows; *_stride is the distance of their batch items in elements.
 *  - lengths, q_lengths and page_table are int32; any values are taken: lengths below 0 are 0, q_lengths are clipped to [0,U].  Rows of the
 *    cache that no token of the call looks at are not used, whatever they hold (NaN included); the others have to be finite, and so has q at
 *    u < q_lengths[b].  Sequences may share pages.
 *  - D is a multiple of 16, at most 128; kv_heads divides heads; page_size is 16, 32, 64, 128 or 256; max_pages * page_size is below
 *    2^31 - 512.  The cache may be of any size: offsets in it are of 64 bits.
 *  - workspace: nm_paged_attn_workspace_bytes bytes, 256-byte aligned (NULL where that is 0).
 */
#ifndef NM_PAGED_ATTENTION_H
#define NM_PAGED_ATTENTION_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of workspace of nm_paged_attn_fwd; 0 for invalid arguments too.  Host only. */
size_t nm_paged_attn_workspace_bytes(int B, int heads, int kv_heads, int D, int U, int page_size, int max_pages, int dtype);

/* q [B][heads*D][U], k_cache, v_cache, page_table [B][max_pages], lengths [B], q_lengths [B] or NULL in;  o [B][heads*D][U] out,
 * lse [B][heads][U] out or NULL. */
int nm_paged_attn_fwd(int B, int heads, int kv_heads, int D, int U, const void *q, long long q_stride, const void *k_cache,
                      const void *v_cache, int pages, int page_size, const int *page_table, int max_pages, const int *lengths,
                      const int *q_lengths, int window, float scale, void *o, long long o_stride, float *lse, int dtype, void *workspace,
                      size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_PAGED_ATTENTION_H */
