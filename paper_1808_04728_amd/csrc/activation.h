// activation.h -- the activations that epilogues and normalisations apply, and their
// derivatives, in fp32.
#pragma once

#include <type_traits>

#include "cf_common.h"

namespace cf {

enum : int { ACT_NONE = 0, ACT_LRELU = 1, ACT_SILU = 2, ACT_GELU = 3 };

// e^x to about an ulp: infinite from 88.73 on, 0 far below (a NaN counts as -120: callers
// multiply by x itself).  x log2 e is rounded to t; what that left out, r, comes back as a
// factor e^(r ln 2) = 1 + r ln 2.  (A factor, not a sum of e and e r ln 2: where e is infinite
// and r is below zero that has no value.  x is clamped so that r is finite.)
__device__ __forceinline__ float fast_exp(float x) {
  constexpr float L = 1.44269504f, L_LO = 1.92596303e-8f;  // log2 e = L + L_LO
  x = fminf(fmaxf(x, -120.f), 120.f);
  const float t = x * L;
  const float r = __builtin_fmaf(x, L_LO, __builtin_fmaf(x, L, -t));
  return __builtin_amdgcn_exp2f(t) * __builtin_fmaf(r, 0.693147181f, 1.f);
}

__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + fast_exp(-u)); }

// Phi(-t) e^(t^2 / 2) for t >= 0, Phi the normal distribution function: a polynomial in
// 1 / (1 + t / 4), fitted to the function so that u Phi(u) is within 2^-21.9 |u| and Phi(u)
// + u phi(u) within 2^-21.9.  (erff costs three times as much: the epilogue of 32768 x 1024 x
// 4096 took 113 us with it.)
__device__ __forceinline__ float normal_tail(float t) {
  const float s = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, t, 1.f));
  float q = -0.0978302136f;
  q = __builtin_fmaf(q, s, 0.371543974f);
  q = __builtin_fmaf(q, s, -0.327021211f);
  q = __builtin_fmaf(q, s, 0.346005082f);
  q = __builtin_fmaf(q, s, -0.0157256275f);
  q = __builtin_fmaf(q, s, 0.126760602f);
  q = __builtin_fmaf(q, s, 0.0960564613f);
  return __builtin_fmaf(q, s, 0.000210965038f);
}
// e^(-u^2 / 2)
__device__ __forceinline__ float bell(float u) { return __builtin_amdgcn_exp2f(u * u * -0.721347520f); }

// act(u)
template <int ACT> __device__ __forceinline__ float act(float u, float alpha) {
  if constexpr (ACT == ACT_LRELU) return u > 0.f ? u : alpha * u;
  if constexpr (ACT == ACT_SILU) return u * sigmoid(u);
  if constexpr (ACT == ACT_GELU) {
    const float q = bell(u) * normal_tail(fabsf(u));
    return u * (u >= 0.f ? 1.f - q : q);
  }
  return u;
}

// act'(u); the leaky ReLU's is alpha at 0
template <int ACT> __device__ __forceinline__ float act_slope(float u, float alpha) {
  if constexpr (ACT == ACT_LRELU) return u > 0.f ? 1.f : alpha;
  if constexpr (ACT == ACT_SILU) {
    const float s = sigmoid(u);
    return s * (1.f + u * (1.f - s));
  }
  if constexpr (ACT == ACT_GELU) {
    const float e = bell(u), q = e * normal_tail(fabsf(u));
    return (u >= 0.f ? 1.f - q : q) + u * (e * 0.398942280f);
  }
  return 1.f;
}

// f(std::integral_constant<int, ACT>) for an activation that is known on the host
template <class F> auto with_act(int a, F f) {
  switch (a) {
    case ACT_LRELU: return f(std::integral_constant<int, ACT_LRELU>{});
    case ACT_SILU: return f(std::integral_constant<int, ACT_SILU>{});
    case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>{});
    default: return f(std::integral_constant<int, ACT_NONE>{});
  }
}

}  // namespace cf
