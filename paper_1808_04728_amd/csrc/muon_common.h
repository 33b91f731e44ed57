// muon_common.h -- device helpers shared by the Newton-Schulz kernels (gfx950).
#pragma once

#include "cf_common.h"
#include "cf_kernels.h"

namespace cf {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));

// the matrix of workgroup b of a launch (matrices without workgroups share their
// first with the next)
__device__ __forceinline__ int ns_find(const NsTable &T, int b) {
  int l = 0;
  while (l + 1 < T.count && T.first[l + 1] <= b) ++l;
  return l;
}

// Sum of a double over 256 threads in a fixed order.
__device__ __forceinline__ double ns_block_sum(double a, double *red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) a += __shfl_xor(a, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// 1 / (||u|| + eps) from the chunks' sums, by every workgroup in the same order
__device__ __forceinline__ double ns_inv_norm(const NsMat &M, const char *ws, double eps, double *red) {
  const double *p = (const double *)(ws + M.ws_norm);
  double s = 0.0;
  for (int i = threadIdx.x; i < M.chunks; i += 256) s += p[i];
  return 1.0 / (sqrt(ns_block_sum(s, red)) + eps);
}

struct Half2 {
  _Float16 hi, lo;
};
// x = hi + lo to 2^-23 of x
__device__ __forceinline__ Half2 ns_split(float x) {
  Half2 r;
  r.hi = (_Float16)x;
  r.lo = (_Float16)(x - (float)r.hi);
  return r;
}

// The same of eight values at two instructions a value: hi by pairs, the remainder
// x - hi as a mixed-precision fma, which reads hi's halves in place.
__device__ __forceinline__ void ns_split8(const float (&x)[8], f16x8_t &hi, f16x8_t &lo) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const f16x2_t h = __builtin_convertvector((f32x2_t{x[i], x[i + 1]}), f16x2_t);
    float a, b;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(a) : "v"(h), "v"(x[i]));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(b) : "v"(h), "v"(x[i + 1]));
    const f16x2_t l = __builtin_convertvector((f32x2_t{a, b}), f16x2_t);
    hi[i] = h[0];
    hi[i + 1] = h[1];
    lo[i] = l[0];
    lo[i + 1] = l[1];
  }
}

// one element of the momentum update: new momentum in m, returns the update u
__device__ __forceinline__ float ns_momentum(const NsMomentum &mom, float g, float &m) {
  const float gi = (float)mom.one_mu * g;
  m = (float)mom.mu * m + gi;
  return mom.nesterov ? (float)mom.mu * m + gi : m;
}

}  // namespace cf
