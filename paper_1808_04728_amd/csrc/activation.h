// activation.h -- the activations that epilogues and normalisations apply, and their
// derivatives, in fp32.
#pragma once

#include <type_traits>

#include "cf_common.h"

namespace cf {

enum : int { ACT_NONE = 0, ACT_LRELU = 1, ACT_SILU = 2, ACT_GELU = 3 };

// e^x to about an ulp, x clamped to where it neither over- nor underflows before infinity
// and zero (a NaN counts as the lower bound: callers multiply by x itself).  x log2 e is
// rounded to t; what that left out, r, comes back as a factor e^(r ln 2) = 1 + r ln 2.
__device__ __forceinline__ float fast_exp(float x) {
  constexpr float L = 1.44269504f, L_LO = 1.92596303e-8f;  // log2 e = L + L_LO
  x = fminf(fmaxf(x, -120.f), 120.f);
  const float t = x * L;
  const float r = __builtin_fmaf(x, L_LO, __builtin_fmaf(x, L, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_fmaf(e, r * 0.693147181f, e);
}

__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + fast_exp(-u)); }

// act(u)
template <int ACT> __device__ __forceinline__ float act(float u, float alpha) {
  if constexpr (ACT == ACT_LRELU) return u > 0.f ? u : alpha * u;
  if constexpr (ACT == ACT_SILU) return u * sigmoid(u);
  if constexpr (ACT == ACT_GELU) return 0.5f * u * (1.f + erff(u * 0.707106781f));
  return u;
}

// act'(u); the leaky ReLU's is alpha at 0
template <int ACT> __device__ __forceinline__ float act_slope(float u, float alpha) {
  if constexpr (ACT == ACT_LRELU) return u > 0.f ? 1.f : alpha;
  if constexpr (ACT == ACT_SILU) {
    const float s = sigmoid(u);
    return s * (1.f + u * (1.f - s));
  }
  if constexpr (ACT == ACT_GELU)
    return 0.5f * (1.f + erff(u * 0.707106781f)) + u * (fast_exp(-0.5f * u * u) * 0.398942280f);
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
