// One AdamW update of one element, in fp32:
//   m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2,
//   p <- p (1 - lr decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
#pragma once
#include "operators.h"

namespace tensair {

// Square root and quotient go into the update alone, where the approximate instructions' errors (2^-23 and 2 units in the
// last place) are those of a rounding or two; the exact ones are ten instructions each.
__device__ __forceinline__ float approximate_root(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float adamw_update(float p, float g, float& m, float& v, const AdamwConsts& c, float step_size,
                                              float keep) {
    m = fmaf(c.beta1, m, c.rest1 * g);
    v = fmaf(c.beta2, v, c.rest2 * g * g);
    return fmaf(p, keep, -step_size * __fdividef(m, fmaf(approximate_root(v), c.inv_root2, c.eps)));
}

// The factor on the gradients, read on the device.  false: it is not finite and the step is left out.
__device__ __forceinline__ bool adamw_grad_scale(const AdamwConsts& c, float* scale) {
    *scale = c.grad_scale ? __ldg(c.grad_scale) : 1.0f;
    return isfinite(*scale);
}

}  // namespace tensair
