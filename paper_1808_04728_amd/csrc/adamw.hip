// adamw.hip -- AdamW with decoupled weight decay over a list of tensors, moments in fp32
// or in 8 bits:
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2
//   p <- (1 - eta decay) p - eta / (1 - b1^k) m / (sqrt(v / (1 - b2^k)) + eps)
//
// One streaming pass, bound by memory: 28 bytes a value with fp32 moments, 16 with 8-bit
// ones (2 more each with the bf16 copy).  All tensors of a launch share its grid; a
// workgroup finds its tensor in the table of the launch.  Measured: 101 million values in 72
// tensors with 8-bit moments and the bf16 copy 347 us, 5.2 TB/s (a large copy 4.7); 3.4 million
// in 40 tensors of odd sizes, 8-bit moments, 15 us; 1.5 million in 18 tensors, fp32 moments and
// the bf16 copy, 10.3 us.
//
// 8-bit moments.  A block is 256 consecutive values of a tensor, one wave's: four values
// a lane, so the block's largest value is a reduction inside the wave.  It holds m and
// r = sqrt(v) as e4m3 codes of value / scale with a power-of-two scale, so that dividing
// by it is exact.  (The root halves the range that v needs.)  Codes are rounded at random,
// up with the chance of the part left over: with b2 = 0.999 a step moves r by 0.05 % and
// less, where codes are 6 to 12 % apart, and rounded to nearest r would never move.
//
// Every operation is one IEEE fp32 operation in the order written, without contraction:
// the new codes depend on no compiler choice.

#include <type_traits>

#include "cf_common.h"
#include "cf_kernels.h"

namespace cf {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;  // values that share a scale

// 32 bits to 32 bits; the multipliers are the fractions of sqrt 2 and sqrt 3
__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
  h ^= h >> 16;
  h *= 0x6A09E667u;
  h ^= h >> 15;
  h *= 0xBB67AE85u;
  return h ^ (h >> 16);
}
constexpr uint32_t kGolden = 0x9E3779B9u;  // odd, near 2^32 / golden ratio

// the largest over the wave, in every lane
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto step = [&](auto ctrl) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true));
  };
  step(std::integral_constant<int, 0x111>{});  // row_shr:1, 2, 4, 8: lane 15 of a row has the row's
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  step(std::integral_constant<int, 0x118>{});
  step(std::integral_constant<int, 0x142>{});  // row_bcast:15, 31: lane 63 has all
  step(std::integral_constant<int, 0x143>{});
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// exponent field of the smallest power of two s with top / s <= 448 (= 1.75 * 2^8), top
// given by its bits; at least 2^-126
__device__ __forceinline__ uint32_t scale_field(uint32_t top) {
  const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(e, 1);
}

// e4m3 code of x (|x| <= 448, or anything if it is not finite: NaN), 16 random bits
__device__ __forceinline__ uint32_t code_of(float x, uint32_t bits16) {
#pragma clang fp contract(off)
  const uint32_t u = __float_as_uint(x), a = u & 0x7fffffffu;
  // below 2^-6 codes are 2^-9 apart, as they are from 2^-6 to 2^-5
  const bool low = a < 0x3c800000u;
  const uint32_t t = low ? __float_as_uint(__uint_as_float(a) + 0.015625f) : a;
  uint32_t c = ((t + (bits16 << 4)) >> 20) - (low ? 968u : 960u);
  if (a >= 0x7f800000u) c = 0x7f;
  return c | (u >> 31 << 7);
}

template <int B> __device__ __forceinline__ float value_of(uint32_t codes) {  // of byte B
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t f = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, B / 2);
  return f[B % 2];
}

struct Step {
  float b1, c1, b2, c2;  // decays and one less them
  float root;            // 1 / sqrt(1 - b2^k)
  float eps, lr;         // lr: eta / (1 - b1^k)
};

// new m and r = sqrt(v) (v too); p
__device__ __forceinline__ void adamw_one(const Step &s, float keep, float g, float &p, float &m, float &v, float &r) {
#pragma clang fp contract(off)
  m = m * s.b1 + g * s.c1;
  v = v * s.b2 + (g * g) * s.c2;
  r = sqrtf(v);
  const float d = (m / (r * s.root + s.eps)) * s.lr;
  p = p * keep - d;
}

__device__ __forceinline__ int find(const AdamwTable &T, int b) {
  // last l with first[l] <= b (every tensor of a table has a workgroup)
  int lo = 0, hi = T.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (T.t[mid].first <= b) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// four values from e on, of which k exist
__device__ __forceinline__ void load4(const float *p, long long e, int k, float (&x)[4]) {
  if (k >= 4) {
    const float4 a = *reinterpret_cast<const float4 *>(p + e);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < k ? p[e + i] : 0.f;
  }
}
__device__ __forceinline__ void load4(const uint16_t *p, long long e, int k, float (&x)[4]) {
  if (k >= 4) {
    const ushort4 a = *reinterpret_cast<const ushort4 *>(p + e);
    x[0] = bf2f(a.x); x[1] = bf2f(a.y); x[2] = bf2f(a.z); x[3] = bf2f(a.w);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i < k ? bf2f(p[e + i]) : 0.f;
  }
}
__device__ __forceinline__ void store4(float *p, long long e, int k, const float (&x)[4]) {
  if (k >= 4) {
    *reinterpret_cast<float4 *>(p + e) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < k) p[e + i] = x[i];
  }
}
__device__ __forceinline__ void store4(uint16_t *p, long long e, int k, const float (&x)[4]) {
  if (k >= 4) {
    *reinterpret_cast<uint2 *>(p + e) = make_uint2(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < k) p[e + i] = f2bf(x[i]);
  }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, long long e, int k) {
  if (k >= 4) return *reinterpret_cast<const uint32_t *>(p + e);
  uint32_t c = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < k) c |= (uint32_t)p[e + i] << (8 * i);
  return c;
}
__device__ __forceinline__ void store_codes(uint8_t *p, long long e, int k, uint32_t c) {
  if (k >= 4) {
    *reinterpret_cast<uint32_t *>(p + e) = c;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < k) p[e + i] = (uint8_t)(c >> (8 * i));
  }
}

// A workgroup takes U turns of 1024 values, the loads of all of them before the first is
// used.
template <int U, bool EIGHT>
__device__ __forceinline__ void run_tensor(const Step &s, const AdamwTensor &A, int chunk) {
  const long long base = (long long)chunk * (U * 4 * kThreads) + 4 * threadIdx.x;
  float p[U][4], g[U][4], m[U][4], v[U][4];
  uint32_t mc[U], rc[U];
  float ms[U], rs[U];
  int k[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long e = base + u * 4 * kThreads;
    k[u] = (int)max(0LL, min(4LL, A.count - e));
    if (A.g16) load4((const uint16_t *)A.g, e, k[u], g[u]);
    else load4((const float *)A.g, e, k[u], g[u]);
    load4(A.p, e, k[u], p[u]);
    if constexpr (EIGHT) {
      mc[u] = load_codes((const uint8_t *)A.m, e, k[u]);
      rc[u] = load_codes((const uint8_t *)A.v, e, k[u]);
      ms[u] = k[u] > 0 ? A.ms[e / kBlock] : 0.f;
      rs[u] = k[u] > 0 ? A.vs[e / kBlock] : 0.f;
    } else {
      load4((const float *)A.m, e, k[u], m[u]);
      load4((const float *)A.v, e, k[u], v[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma clang fp contract(off)
    const long long e = base + u * 4 * kThreads;
    float r[4];
    if constexpr (EIGHT) {
      m[u][0] = value_of<0>(mc[u]) * ms[u]; m[u][1] = value_of<1>(mc[u]) * ms[u];
      m[u][2] = value_of<2>(mc[u]) * ms[u]; m[u][3] = value_of<3>(mc[u]) * ms[u];
      r[0] = value_of<0>(rc[u]) * rs[u]; r[1] = value_of<1>(rc[u]) * rs[u];
      r[2] = value_of<2>(rc[u]) * rs[u]; r[3] = value_of<3>(rc[u]) * rs[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[u][i] = r[i] * r[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) adamw_one(s, A.keep, g[u][i], p[u][i], m[u][i], v[u][i], r[i]);
    store4(A.p, e, k[u], p[u]);
    if (A.p16) store4(A.p16, e, k[u], p[u]);
    if constexpr (EIGHT) {
      // the block's largest finite values (lanes past the tensor's end have zeros)
      uint32_t tm = 0, tr = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t am = __float_as_uint(m[u][i]) & 0x7fffffffu, ar = __float_as_uint(r[i]) & 0x7fffffffu;
        tm = max(tm, am < 0x7f800000u ? am : 0u);
        tr = max(tr, ar < 0x7f800000u ? ar : 0u);
      }
      const uint32_t fm = scale_field(wave_max(tm)), fr = scale_field(wave_max(tr));
      const float im = __uint_as_float((254u - fm) << 23), ir = __uint_as_float((254u - fr) << 23);
      uint32_t cm = 0, cr = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t h = mix(A.key + (uint32_t)(e + i) * kGolden);
        cm |= code_of(m[u][i] * im, h & 0xffffu) << (8 * i);
        uint32_t c = code_of(r[i] * ir, h >> 16);
        if (c == 0 && v[u][i] > 0.f) c = 1;  // a second moment that is not zero is not held as zero
        cr |= c << (8 * i);
      }
      store_codes((uint8_t *)A.m, e, k[u], cm);
      store_codes((uint8_t *)A.v, e, k[u], cr);
      if ((threadIdx.x & 63) == 0 && k[u] > 0) {
        A.ms[e / kBlock] = __uint_as_float(fm << 23);
        A.vs[e / kBlock] = __uint_as_float(fr << 23);
      }
    } else {
      store4((float *)A.m, e, k[u], m[u]);
      store4((float *)A.v, e, k[u], v[u]);
    }
  }
}

template <int U> __global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwTable T, Step s) {
  const int l = find(T, blockIdx.x);
  const AdamwTensor &A = T.t[l];
  const int chunk = blockIdx.x - A.first;
  if (A.ms) run_tensor<U, true>(s, A, chunk);
  else run_tensor<U, false>(s, A, chunk);
}

}  // namespace

uint32_t adamw_key(uint32_t seed, long long t, int tensor) {
  return mix(mix(seed + (uint32_t)t * kGolden) + (uint32_t)tensor * kGolden);
}

hipError_t launch_adamw(AdamwTable &T, const AdamwStep &h, hipStream_t st) {
  const Step s{h.b1, h.c1, h.b2, h.c2, h.root, h.eps, h.lr};
  constexpr int kTurn = 4 * kThreads;
  long long turns = 0;
  for (int l = 0; l < T.count; ++l) turns += (T.t[l].count + kTurn - 1) / kTurn;
  const int U = turns > 8192 ? 4 : 1;
  // (a launch has at most 2^23 workgroups: tensors past that are cut by the caller)
  long long at = 0;
  for (int l = 0; l < T.count; ++l) {
    T.t[l].first = (int)at;
    at += (T.t[l].count + U * kTurn - 1) / (U * kTurn);
  }
  if (at == 0) return hipSuccess;
  if (U == 4) hipLaunchKernelGGL(adamw_kernel<4>, dim3((unsigned)at), dim3(kThreads), 0, st, T, s);
  else hipLaunchKernelGGL(adamw_kernel<1>, dim3((unsigned)at), dim3(kThreads), 0, st, T, s);
  return hipGetLastError();
}

}  // namespace cf
