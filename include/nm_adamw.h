/*
 * nm_adamw.h -- C ABI of an AdamW step over many tensors in one launch (gfx950), states in 32 or in 8 bits.
 *
 * The weight gradients of the other calls are float32 and, as the paper's mixed-precision contract has it (Section 3.3),
 * so is the state of training; the low-precision weights that those calls read are a rounded copy.  For every element
 *
 *   g = grad * grad_scale[0];   m = beta1*m + (1-beta1)*g;   v = beta2*v + (1-beta2)*g^2
 *   param = param*(1 - lr*weight_decay) - lr/(1-beta1^step) * m / (sqrt(v/(1-beta2^step)) + eps);   copy = bf16(param)
 *
 * 32 state bits: m and v are float.  8 state bits: a tensor is cut into blocks of 256 elements (the last one shorter); m and
 * r = sqrt(v) are held as E4M3 codes with a float scale per block and moment,
 *   scale = max |value of the block| / 448, at least 2^-126 (1 where that maximum is 0);   value = decode(code) * scale
 * The update takes m and r as they are before they are rounded.  Rounding is stochastic: with ulp the distance of the E4M3
 * values around z = |value|/scale, the code is that of floor(z/ulp + i/65536)*ulp, at most 448, where i is the low (m) or
 * the high (r) half of 32 bits mixed from `seed` and the element's number (below).  Rounded to nearest, a moment that
 * changes by less than half a step per call, as v with its beta2 always does, would never move.  It is r whose mean is kept:
 * that of v = r^2 lies 4 to 6 % above (beta2 from 0.98 to 0.999), its root 2 to 3 %.  An r above zero does not
 * become zero (it becomes 2^-9 of the scale: m/r stays bounded).  All of this is decided in 64-bit arithmetic.  Moments
 * that are infinite, NaN or larger than 448 times the largest float are stored as NaN and left out of the block's maximum.
 *   bits of element e: 256*(blocks of the plan in front of its tensor) + (its index in the tensor), mod 2^32;
 *   h = e*0x9E3779B9 ^ seed;  h = (h ^ h>>16)*0x6A09E667;  h = (h ^ h>>13)*0xBB67AE85;  h ^ h>>16        (mod 2^32)
 *
 * Conventions are those of nm_conv1d.h.  The tensors of a step are described once, in a plan: nm_adamw_plan writes it into
 * host memory, the caller copies those bytes to the device and hands both copies to every step.  A plan holds addresses: the
 * tensors stay where they are while it is in use.  No tensor of a plan overlaps another, and together
 * they have less than 2^24 runs of 4096 elements (a tensor's last run may be shorter).
 */
#ifndef NM_ADAMW_H
#define NM_ADAMW_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    float *param;         /* [n] in/out */
    const float *grad;    /* [n] in */
    void *m, *v;          /* [n] in/out: float, or E4M3 codes of m and of sqrt(v) */
    float *m_scale, *v_scale; /* [ceil(n/256)] in/out with 8 state bits, else NULL */
    void *copy;           /* [n] bfloat16 out, or NULL */
    long long n;          /* at least 1, below 2^31 */
    float weight_decay;   /* finite, not negative */
} nm_adamw_tensor;

/* Bytes of the plan of these tensors (0: invalid arguments).  Host only. */
size_t nm_adamw_plan_bytes(const nm_adamw_tensor *tensors, int count, int state_bits);
/* Writes the plan into `plan` (host memory, plan_bytes as above).  Host only. */
int nm_adamw_plan(const nm_adamw_tensor *tensors, int count, int state_bits, void *plan, size_t plan_bytes);

/* One step.  plan: the host copy; plan_device: the same bytes in device memory (256-byte aligned).  step counts from 1.
 * 0 <= beta < 1, eps at least 2^-126, lr finite.  grad_scale [1] float, device, or NULL (1).  seed: another one each step; unused with
 * 32 state bits. */
int nm_adamw_step(const void *plan, const void *plan_device, size_t plan_bytes, double lr, double beta1, double beta2,
                  double eps, long long step, const float *grad_scale, unsigned seed, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NM_ADAMW_H */
