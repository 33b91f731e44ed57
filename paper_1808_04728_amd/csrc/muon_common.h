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

// one element of the momentum update: new momentum in m, returns the update u
__device__ __forceinline__ float ns_momentum(const NsMomentum &mom, float g, float &m) {
  const float gi = (float)mom.one_mu * g;
  m = (float)mom.mu * m + gi;
  return mom.nesterov ? (float)mom.mu * m + gi : m;
}

}  // namespace cf
