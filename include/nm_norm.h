/*
 * nm_norm.h -- C ABI of the norms around a block, fused with its gate and residual scale (gfx950), forward and backward.
 *
 * What lies between the last product of one block and the first of the next, in one pass over channel-major activations
 * [batch][channels][time]:
 *
 *   h = f, or Norm(f; post_weight, post_bias) with NM_NORM_POST          f: the block's output
 *   y = x + rscale[c] * gate * h                                         x: the residual stream; y in storage type
 *   n = Norm(y; next_weight, next_bias) with NM_NORM_NEXT                of the stored y: the next block's input
 *   Norm over the C channels of a position:  z * rstd * weight[c] + bias[c],  rstd = 1/sqrt(mean(z^2) + eps), and with
 *   NM_NORM_LAYER of z - mean(z) instead of z.
 * Without f, y = x is not written and n = Norm(x): the norm in front of the first block.
 *   gate: none, one value per item and channel (NM_GATE_ITEM, [B][C] float) or per element (NM_GATE_ELEMENT, [B][C][T], dtype).
 *
 * Backward, from dy (the gradient of y, NULL: none) and dn (that of n):
 *   g = dy + NormBackward(dn; y);   dx = g
 *   dh = rscale[c] * gate * g;   df = dh, or NormBackward(dh; f)
 *   dgate = rscale[c] * g * h (summed over time for NM_GATE_ITEM);   drscale[c] = sum over b, t of g * gate * h
 *   dpost_weight = sum dh * fhat, dpost_bias = sum dh;   dnext_weight = sum dn * yhat, dnext_bias = sum dn
 * Norms are made again from f and y: nothing but them is kept between the passes.
 *
 * Conventions are those of nm_conv1d.h.  dtype is the storage type of x, f, y, n, an element gate and their gradients;
 * rscale, weights, biases, an item gate and their gradients are float; all arithmetic is float32.  lengths [B] int32 (NULL:
 * none): positions at or beyond an item's length are not read; y, n, dx, df and an element gate's gradient are zero there,
 * and they add nothing to the sums.  Up to 1024 channels (rows of 16 bytes or more) are held in registers, wider rows are read again for
 * every sum, many times as long.  Without an eps the norm of a position of zeros is NaN.  C is at most 8192, B at most 65000, and
 * B*C*T below 2^31; the forward pass takes no more than some 2^28 positions in bfloat16, 2^27 in float (which calls of 16 channels
 * or fewer can reach).
 */
#ifndef NM_NORM_H
#define NM_NORM_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { NM_NORM_POST = 1u, NM_NORM_NEXT = 2u, NM_NORM_LAYER = 4u };
enum { NM_GATE_NONE = 0, NM_GATE_ITEM = 1, NM_GATE_ELEMENT = 2 };

/* Forward.  Vectors that are NULL: 1 for rscale and weights, 0 for biases.  y is required iff f is given, n iff NM_NORM_NEXT
 * is.  NM_NORM_POST needs f; biases need NM_NORM_LAYER; at least one of f and NM_NORM_NEXT.  Needs no workspace. */
int nm_residual_norm_fwd(int B, int C, int T, const void *x, const void *f, const void *gate, int gate_kind,
                         const float *rscale, const float *post_weight, const float *post_bias, const float *next_weight,
                         const float *next_bias, float eps, const int *lengths, void *y, void *n, unsigned flags, int dtype,
                         void *hip_stream);

/* Bytes of workspace of nm_residual_norm_bwd; 0 for invalid arguments.  Host only. */
size_t nm_residual_norm_bwd_workspace_bytes(int B, int C, int T, int dtype);

/* Backward.  y as the forward pass stored it (x without f; needed iff NM_NORM_NEXT).  dx required; df required iff f is given.
 * The other gradients are optional (NULL), and NULL where what they belong to is not there. */
int nm_residual_norm_bwd(int B, int C, int T, const void *dy, const void *dn, const void *y, const void *f, const void *gate,
                         int gate_kind, const float *rscale, const float *post_weight, const float *post_bias,
                         const float *next_weight, float eps, const int *lengths, void *dx, void *df, void *dgate,
                         float *drscale, float *dpost_weight, float *dpost_bias, float *dnext_weight, float *dnext_bias,
                         unsigned flags, int dtype, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_NORM_H */
