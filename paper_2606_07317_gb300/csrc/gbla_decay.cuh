// Powers of a head's decay, shared by the kernels of decayed linear attention.
#pragma once

#include <math.h>

namespace gbla {

// gamma^n for n >= 0 with l2 = log2 gamma; gamma^0 is 1 also for gamma = 0.  A power
// that fp32 cannot hold is the least positive float, not 0: it weighs a state, and an
// infinite state stays infinite however far it fades (0 times it would be NaN).
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float decay_pow(float l2, float n) {
  if (n == 0.f) return 1.f;
  const float w = exp2f(n * l2);
  return w == 0.f && l2 > -INFINITY ? kLeast : w;
}
// scale * gamma^n, in the same way.
__device__ __forceinline__ float scaled_pow(float scale, float l2, float n) {
  const float w = scale * decay_pow(l2, n);
  return w == 0.f && l2 > -INFINITY ? copysignf(kLeast, scale) : w;
}
__device__ __forceinline__ float log2_decay(const float *log_decay, int h) {
  return __ldg(log_decay + h) * 1.4426950408889634f;
}

// e^x as the sum of two floats: the factor by which a state decays again and
// again.  Rounded to one float, its error of up to 2^-25 would grow with the
// number of factors that a contribution meets before it fades, 1 / |x| (2e-6 of a
// state that decays over 4096 tokens in chunks of 64, 1e-4 token by token).
// Near 1 it is 1 + expm1(x), whose error is 2^-24 of the small part and of lo (below
// 2^-47); where it is not, contributions fade after a few factors.  Both parts are
// positive for every gamma > 0 (so hi is rounded down), so that an infinite state gives
// infinities of one sign; the least lo changes no rounding of a finite one.
struct DecayFactor {
  float hi, lo;
};
__device__ __forceinline__ DecayFactor one_factor(float f) {
  return {f, f > 0.f ? fmaxf(f * 0x1p-40f, kLeast) : 0.f};
}
__device__ __forceinline__ DecayFactor decay_factor(float x) {
  if (fabsf(x) > 0.35f) {
    const float f = expf(x);
    return one_factor(f == 0.f && x > -INFINITY ? kLeast : f);
  }
  const float e = expm1f(x), hi = __fadd_rd(1.f, e);
  return {hi, fmaxf(e - (hi - 1.f), 0x1p-60f)};
}

}  // namespace gbla
