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

// Sum of a double over W waves in a fixed order.
template <int W = 4> __device__ __forceinline__ double ns_block_sum(double a, double *red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) a += __shfl_xor(a, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  double s = red[0];
#pragma unroll
  for (int w = 1; w < W; ++w) s += red[w];
  return s;
}

// 1 / (||u|| + eps) from the chunks' sums, by every workgroup in the same order: 256
// threads' shares, whatever the number of threads
template <int W = 4> __device__ __forceinline__ double ns_inv_norm(const NsMat &M, const char *ws, double eps, double *red) {
  const double *p = (const double *)(ws + M.ws_norm);
  double s = 0.0;
  if (W == 4 || threadIdx.x < 256)
    for (int i = threadIdx.x; i < M.chunks; i += 256) s += p[i];
  return 1.0 / (sqrt(ns_block_sum<W>(s, red)) + eps);
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

// The same of N values (N even) at two instructions a value: hi by pairs, the remainder
// x - hi as a mixed-precision fma, which reads hi's halves in place.
template <int N, class V> __device__ __forceinline__ void ns_split_pairs(const float (&x)[N], V &hi, V &lo) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < N; i += 2) {
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
__device__ __forceinline__ void ns_split8(const float (&x)[8], f16x8_t &hi, f16x8_t &lo) { ns_split_pairs<8>(x, hi, lo); }

// one element of the momentum update: new momentum in m, returns the update u
__device__ __forceinline__ float ns_momentum(const NsMomentum &mom, float g, float &m) {
  const float gi = (float)mom.one_mu * g;
  m = (float)mom.mu * m + gi;
  return mom.nesterov ? (float)mom.mu * m + gi : m;
}

template <int VW> __device__ __forceinline__ void load_cols(const float *p, float (&x)[VW]) {
  if constexpr (VW == 4) {
    const float4 a = *reinterpret_cast<const float4 *>(p);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  } else if constexpr (VW == 2) {
    const float2 a = *reinterpret_cast<const float2 *>(p);
    x[0] = a.x; x[1] = a.y;
  } else {
    x[0] = *p;
  }
}

template <int VW> __device__ __forceinline__ void store_cols(float *p, const float (&x)[VW]) {
  if constexpr (VW == 4) *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
  else if constexpr (VW == 2) *reinterpret_cast<float2 *>(p) = make_float2(x[0], x[1]);
  else *p = x[0];
}

// x s1 s2.  s1 is 1 unless 1 / norm is past where fp32's range ends but its product
// with x is not; without `on` x is taken as it is.
struct Scale {
  bool on;
  float s1, s2;
};
__device__ __forceinline__ Scale scale_of(double inv, float sx) {
  int e = 0;
  (void)frexp(inv, &e);
  Scale s;
  s.on = true;
  e = e > 100 || e < -100 ? min(max(e, -126), 126) : 0;
  s.s1 = ldexpf(1.0f, e);
  s.s2 = (float)(inv * (double)sx * ldexp(1.0, -e));
  return s;
}
// the output: the orthogonalised matrix, or the parameters updated with it
struct Out {
  void *o;
  uint16_t *v16;
  int update;
  float eta, decay, gain;
};

__device__ __forceinline__ float update_one(const Out &o, float v, float x) { return v - o.eta * (o.gain * x + o.decay * v); }

// element e
template <int DT> __device__ __forceinline__ void emit1(const Out &o, long long e, float x) {
  if (o.update) {
    float *v = (float *)o.o + e;
    const float a = update_one(o, *v, x);
    *v = a;
    if (o.v16) o.v16[e] = f2bf(a);
  } else {
    ((typename Store<DT>::T *)o.o)[e] = from_f32<DT>(x);
  }
}

// four values at the alignment of one element
typedef uint32_t u32x4f_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2h_t __attribute__((ext_vector_type(2), aligned(2)));

// elements e .. e + 3
template <int DT> __device__ __forceinline__ void emit4(const Out &o, long long e, const float (&x)[4]) {
  if (DT == DT_F32 || o.update) {
    u32x4f_t *p = reinterpret_cast<u32x4f_t *>((float *)o.o + e);
    u32x4f_t a;
    if (o.update) {
      a = *p;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(update_one(o, __uint_as_float(a[i]), x[i]));
      if (o.v16)
        *reinterpret_cast<u32x2h_t *>(o.v16 + e) = u32x2h_t{f2bf2(__uint_as_float(a[0]), __uint_as_float(a[1])),
                                                            f2bf2(__uint_as_float(a[2]), __uint_as_float(a[3]))};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(x[i]);
    }
    *p = a;
  } else {
    *reinterpret_cast<u32x2h_t *>((uint16_t *)o.o + e) = u32x2h_t{f2bf2(x[0], x[1]), f2bf2(x[2], x[3])};
  }
}

// the first k of W consecutive elements from e on
template <int DT, int W> __device__ __forceinline__ void emit(const Out &o, long long e, const float (&x)[W], int k) {
  if constexpr (W == 4) {
    if (k >= 4) {
      emit4<DT>(o, e, x);
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i)
    if (i < k) emit1<DT>(o, e + i, x[i]);
}

}  // namespace cf
