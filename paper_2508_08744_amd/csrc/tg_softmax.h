// Exponentials of logits, and (maximum, sum) pairs: shared by the cross entropy and the log probabilities.
#pragma once
#include <hip/hip_runtime.h>

#define XENT_LOG2E 1.4426950408889634f

__device__ inline float xent_exp(float x) { return __builtin_amdgcn_exp2f(x * XENT_LOG2E); }

// Up to here exp(z - m) is 2 to the power of one multiply-add, z log2(e) - m log2(e), whose rounding is that of its terms: 2^-7 at this size, and beyond it
// more and more, up to results that overflow.  (For the sums it is no larger than that of the logits and of lse themselves; the gradients, which have lse as a number, give it back: xent_p_kernel.)  Logits (or a scale) beyond it take the difference first: in the place of the products it makes the
// exponents, to be taken with a factor of 1 and nothing subtracted, so that what follows is the same for both.
#define XENT_NEAR 65536.0f
__device__ inline bool xent_near(float m, float base) { return fabsf(m) < XENT_NEAR && fabsf(base) <= 3.4028234e38f; }
// LARGEST: m is the largest logit, and one that is infinite is taken in by its equals alone.  Else it is lse, and the difference what it is.
template <bool LARGEST>
__device__ inline float xent_far(float product, float scale, float m)
{
    // (the logit is rounded before the difference, as m was: one multiply-add of both would leave m's rounding, which is large here)
#pragma clang fp contract(off)
    asm volatile("" : "+v"(product));        // (nothing of this is made out where it is not needed)
    const float z = product * scale;
    return LARGEST && z == m ? (m == -__builtin_inff() ? m : 0.0f) : (z - m) * XENT_LOG2E;
}

// (maximum, sum) pairs: one that stands for nothing is (-infinity, 0)
__device__ inline void xent_join(float& m, float& l, float m2, float l2)
{
    const float top = fmaxf(m, m2);
    l = (m == top ? l : l * xent_exp(m - top)) + (m2 == top ? l2 : l2 * xent_exp(m2 - top));
    m = top;
}
