/*
 * nm_embedding.h -- C ABI of the lookup of tokens' embeddings and of its gradient (gfx950).
 *
 * A decoder over the acoustic encoder's states (paper Section 4.1.1) begins with the tokens written so far: each is a row of a
 * table, and the rows are laid out as the other calls of this library take activations, [batch][channels][tokens].
 *
 *   out[b,c,u]   = scale * table[ids[b,u]][c];   0 where ids[b,u] is outside [0,V) or u >= lengths[b]
 *   dtable[v][c] = scale * sum of dout[b,c,u] over the places with ids[b,u] = v and u < lengths[b]
 *
 * Conventions are those of nm_conv1d.h (device pointers the caller owns, one stream, enqueue only, argument errors before
 * any device call, deterministic results), with these additions:
 *  - dtype (NM_BF16 or NM_F32) is the storage type of table, out and dout; dtable is float.  Sums are float32, in the order of the
 *    places, in groups that depend on how often a token occurs.
 *  - ids [B][U]: int32 (id_bytes 4) or int64 (id_bytes 8).  lengths [B] int32, optional (NULL); any values are taken, clipped to
 *    [0,U].  dout is not used at u >= lengths[b] or where the id is outside [0,V), whatever it holds.
 *  - workspace: nm_embedding_bwd_workspace_bytes bytes, 256-byte aligned.
 *  - V * C and B * C * U must be below 2^31, B * U at most 2^31 - 2^14 - 1, B at most 65535; tiles of 64 tokens and 64 channels, the items'
 *    last ones counted whole, below 2^23.
 */
#ifndef NM_EMBEDDING_H
#define NM_EMBEDDING_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Forward.  ids [B][U], table [V][C] in;  out [B][C][U] out. */
int nm_embedding_fwd(int B, int V, int C, int U, const void *ids, int id_bytes, const void *table, float scale, const int *lengths,
                     void *out, int dtype, void *hip_stream);

/* Bytes of workspace of nm_embedding_bwd; 0 for invalid arguments.  Host only. */
size_t nm_embedding_bwd_workspace_bytes(int B, int V, int C, int U, int dtype);

/* Gradient of the table.  dout [B][C][U], ids [B][U] in;  dtable [V][C] out, written whole (in and out with NM_ACCUM_DW in flags: the
 * gradient is added to what it holds, and rows without a token keep their bits). */
int nm_embedding_bwd(int B, int V, int C, int U, const void *dout, const void *ids, int id_bytes, float scale, const int *lengths,
                     float *dtable, unsigned flags, int dtype, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_EMBEDDING_H */
