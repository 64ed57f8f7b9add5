// Powers of a head's decay, shared by the kernels of decayed linear attention.
#pragma once

namespace gbla {

// gamma^n for n >= 0 with l2 = log2 gamma; gamma^0 is 1 also for gamma = 0.
__device__ __forceinline__ float decay_pow(float l2, float n) {
  return n == 0.f ? 1.f : exp2f(n * l2);
}
__device__ __forceinline__ float log2_decay(const float *log_decay, int h) {
  return __ldg(log_decay + h) * 1.4426950408889634f;
}

// e^x as the sum of two floats: the factor by which a state decays again and
// again.  Rounded to one float, its error of up to 2^-25 would grow with the
// number of factors that a contribution meets before it fades, 1 / |x| (2e-6 of a
// state that decays over 4096 tokens in chunks of 64, 1e-4 token by token).
// Near 1 it is 1 + expm1(x), whose error is 2^-24 of the small part alone; where
// it is not, contributions fade after a few factors.
struct DecayFactor {
  float hi, lo;
};
__device__ __forceinline__ DecayFactor decay_factor(float x) {
  if (fabsf(x) > 0.35f) return {expf(x), 0.f};
  const float e = expm1f(x), hi = 1.f + e;
  return {hi, e - (hi - 1.f)};
}

}  // namespace gbla
