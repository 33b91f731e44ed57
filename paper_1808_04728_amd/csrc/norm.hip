// norm.hip -- layer normalisation of rows of c values, forward and backward.
//
//   mean = sum x / c,  rstd = (sum (x - mean)^2 / c + eps)^(-1/2)
//   y = (x - mean) rstd gamma + beta
//   g = dy gamma,  xh = (x - mean) rstd
//   dx = rstd (g - sum(g) / c - xh sum(g xh) / c),  dgamma = sum_r dy xh,  dbeta = sum_r dy
//
// Both passes are bound by HBM (7 and 12 operations a value), so a value is
// read once, rows in chunks (below) apart: a team of threads holds its row in
// registers (16-byte vectors as they were loaded) between the sums over the row and
// the stores.  The variance is the second pass over those registers, not a
// difference of moments.
// Statistics, sums and the arithmetic are fp32 for both types; a bf16 output is
// rounded once.
//
// A team is the smallest power of two of lanes that holds a row with one vector
// each (64 / team rows a wave, so a row of 16 channels costs two lanes and one
// exchange), then a wave with more vectors a lane, then a workgroup.  Rows that
// no workgroup holds, and a few long rows that would leave most compute units
// idle, are cut into chunks: a first launch leaves each chunk's statistics, the
// second combines them in a fixed order and reads the chunk again (from HBM in tensors
// larger than the last-level cache: 1024 bf16 rows of 2^18 465 us forward, 4096 of 65536
// 555 us backward, 3.5 and 4.8 TB/s of those that move).
//
// Rows whose length is no multiple of a vector start at any element: their
// vectors are loaded and stored at the elements' own alignment, and the last one is
// the row's last full vector, which repeats some of its neighbour's elements (they
// count once in sums; stored twice they have the same value, and every load of a row
// comes before its first store).  Element by element that vector took up to fourteen
// instructions, more than the rest of a short row: 65536 bf16 rows of 255 went from 20.8
// to 13.6 us.  Rows shorter than a vector, and the ends of chunks (where a
// neighbour may have stored already, in place), do go in smaller pieces.  Nothing
// outside a row is touched.

#include <type_traits>

#include "cf_common.h"
#include "cf_kernels.h"

namespace cf {
namespace {

// 16 bytes at the alignment of one element
typedef uint32_t u32x4f_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4h_t __attribute__((ext_vector_type(4), aligned(2)));
template <int DT> struct Loose;
template <> struct Loose<DT_F32> { using V = u32x4f_t; };
template <> struct Loose<DT_BF16> { using V = u32x4h_t; };

// the product rounded on its own: with one value a row, g - sum(g) / c is exactly 0
__device__ __forceinline__ float mul_rounded(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

template <int DT> __device__ __forceinline__ void unpack(const u32x4_t &v, float (&f)[Store<DT>::VEC]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t w = v[q];
    if constexpr (DT == DT_F32) {
      f[q] = __uint_as_float(w);
    } else {
      f[2 * q] = __uint_as_float(w << 16);
      f[2 * q + 1] = __uint_as_float(w & 0xffff0000u);
    }
  }
}

template <int DT> __device__ __forceinline__ u32x4_t pack(const float (&f)[Store<DT>::VEC]) {
  if constexpr (DT == DT_F32) {
    return u32x4_t{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  } else {
    return pack_bf16x8(f);
  }
}

// How rows lie: FULL a multiple of a vector, STREAM the same in tensors that the
// last-level cache does not hold and that pass it by, RAGGED longer than a vector, SHORT
// below one.
enum : int { FULL = 0, RAGGED = 1, SHORT = 2, STREAM = 3 };

// A lane's vector j of a row: its first element, and how many of its elements belong to
// the vector before (all of them for a vector past the row's end).
template <int DT, int ROW> struct Place {
  int e, skip;
  __device__ __forceinline__ Place(int j, int c) {
    constexpr int V = Store<DT>::VEC;
    e = j * V;
    if constexpr (ROW == RAGGED) e = min(e, c - V);
    skip = j * V < c ? j * V - e : V;
  }
  __device__ __forceinline__ bool any() const { return skip < Store<DT>::VEC; }
  // whether element i counts (c: the row's length)
  __device__ __forceinline__ bool has(int i, int c) const {
    if constexpr (ROW == SHORT) return i < c;
    else if constexpr (ROW == RAGGED) return i >= skip;
    else return any();
  }
};

// the first c < V elements at p in pieces of 4, 2 and 1
template <int DT> __device__ __forceinline__ u32x4_t load_short(const typename Store<DT>::T *p, int c) {
  u32x4_t v = {0u, 0u, 0u, 0u};
  if constexpr (DT == DT_F32) {
    if (c & 2) {
      v[0] = __float_as_uint(p[0]);
      v[1] = __float_as_uint(p[1]);
    }
    if (c & 1) v[c & 2] = __float_as_uint(p[c & 2]);
  } else {
    typedef uint32_t u32x2h_t __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t u32h_t __attribute__((aligned(2)));
    if (c & 4) {
      const u32x2h_t a = *reinterpret_cast<const u32x2h_t *>(p);
      v[0] = a[0];
      v[1] = a[1];
    }
    const int at = c & 4;
    uint32_t w = 0;
    if (c & 2) w = *reinterpret_cast<const u32h_t *>(p + at);
    uint32_t z = 0;
    if (c & 1) z = p[c & 6];
    const uint32_t lo = c & 2 ? w : z, hi = c & 2 ? z : 0u;
    if (at) {
      v[2] = lo;
      v[3] = hi;
    } else {
      v[0] = lo;
      v[1] = hi;
    }
  }
  return v;
}

template <int DT> __device__ __forceinline__ void store_short(typename Store<DT>::T *p, int c, const u32x4_t &v) {
  if constexpr (DT == DT_F32) {
    if (c & 2) {
      p[0] = __uint_as_float(v[0]);
      p[1] = __uint_as_float(v[1]);
    }
    if (c & 1) p[c & 2] = __uint_as_float(c & 2 ? v[2] : v[0]);
  } else {
    typedef uint32_t u32x2h_t __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t u32h_t __attribute__((aligned(2)));
    if (c & 4) *reinterpret_cast<u32x2h_t *>(p) = u32x2h_t{v[0], v[1]};
    const uint32_t lo = c & 4 ? v[2] : v[0], hi = c & 4 ? v[3] : v[1];
    if (c & 2) *reinterpret_cast<u32h_t *>(p + (c & 4)) = lo;
    if (c & 1) p[c & 6] = (uint16_t)(c & 2 ? hi : lo);
  }
}

// A lane's vector of a row, zero unless `in` and where the lane has none.  ALWAYS: the load
// itself does not depend on that (row is one that exists); under a condition each load of
// a team's waits for the one before.  A workgroup's row has its ends in few waves and
// needs the registers instead.
template <int DT, int ROW, bool ALWAYS>
__device__ __forceinline__ u32x4_t load_vec(const typename Store<DT>::T *row, const Place<DT, ROW> &at, int c, bool in = true) {
  in = in && at.any();
  if (!ALWAYS && !in) return u32x4_t{0u, 0u, 0u, 0u};
  const int e = ALWAYS ? min(at.e, c - Store<DT>::VEC) : at.e;
  u32x4_t v;
  if constexpr (ROW == FULL) v = *reinterpret_cast<const u32x4_t *>(row + e);
  else if constexpr (ROW == STREAM) v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(row + e));
  else if constexpr (ROW == RAGGED) v = *reinterpret_cast<const typename Loose<DT>::V *>(row + e);
  else v = load_short<DT>(row, c);
  if (ALWAYS) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = in ? v[q] : 0u;
  }
  return v;
}

template <int DT, int ROW>
__device__ __forceinline__ void store_vec(typename Store<DT>::T *row, const Place<DT, ROW> &at, int c, const u32x4_t &v) {
  if (!at.any()) return;
  if constexpr (ROW == FULL) *reinterpret_cast<u32x4_t *>(row + at.e) = v;
  else if constexpr (ROW == STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t *>(row + at.e));
  else if constexpr (ROW == RAGGED) *reinterpret_cast<typename Loose<DT>::V *>(row + at.e) = v;
  else store_short<DT>(row, c, v);
}

// vector at element e of a chunk of n values (zero past its end), the last one in pieces
template <int DT, bool RAG> __device__ __forceinline__ u32x4_t load_part(const typename Store<DT>::T *p, int e, int n) {
  constexpr int V = Store<DT>::VEC;
  if (e >= n) return u32x4_t{0u, 0u, 0u, 0u};
  if constexpr (!RAG) {
    return *reinterpret_cast<const u32x4_t *>(p + e);
  } else {
    if (e + V <= n) return *reinterpret_cast<const typename Loose<DT>::V *>(p + e);
    return load_short<DT>(p + e, n - e);
  }
}

template <int DT, bool RAG>
__device__ __forceinline__ void store_part(typename Store<DT>::T *p, int e, int n, const u32x4_t &v) {
  constexpr int V = Store<DT>::VEC;
  if (e >= n) return;
  if constexpr (!RAG) {
    *reinterpret_cast<u32x4_t *>(p + e) = v;
  } else {
    if (e + V <= n) *reinterpret_cast<typename Loose<DT>::V *>(p + e) = v;
    else store_short<DT>(p + e, n - e, v);
  }
}

// a lane's V values of an fp32 vector of c (gamma, beta), zero where it has none
template <int DT, int ROW, bool ALWAYS>
__device__ __forceinline__ void load_f32(const float *p, const Place<DT, ROW> &at, int c, float (&f)[Store<DT>::VEC]) {
  constexpr int V = Store<DT>::VEC;
  if constexpr (ROW == SHORT) {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i < c && at.any() ? p[i] : 0.f;
  } else {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      u32x4f_t a = {0u, 0u, 0u, 0u};
      if (ALWAYS || at.any()) a = *reinterpret_cast<const u32x4f_t *>(p + (ALWAYS ? min(at.e, c - V) : at.e) + q);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[q + i] = at.any() ? __uint_as_float(a[i]) : 0.f;
    }
  }
}

// the lane's own of V column sums, into a row of c
template <int DT, int ROW>
__device__ __forceinline__ void store_f32(float *p, const Place<DT, ROW> &at, int c, const float (&f)[Store<DT>::VEC]) {
  constexpr int V = Store<DT>::VEC;
  if (ROW != SHORT && at.skip == 0) {
#pragma unroll
    for (int q = 0; q < V; q += 4)
      *reinterpret_cast<u32x4f_t *>(p + at.e + q) = u32x4f_t{__float_as_uint(f[q]), __float_as_uint(f[q + 1]),
                                                             __float_as_uint(f[q + 2]), __float_as_uint(f[q + 3])};
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (at.any() && at.has(i, c)) p[at.e + i] = f[i];
  }
}

// the same from element e of a chunk of n on
template <int V> __device__ __forceinline__ void load_f32_part(const float *p, int e, int n, float (&f)[V]) {
#pragma unroll
  for (int q = 0; q < V; q += 4) {
    if (e + q + 4 <= n) {
      const float4 a = *reinterpret_cast<const float4 *>(p + e + q);
      f[q] = a.x; f[q + 1] = a.y; f[q + 2] = a.z; f[q + 3] = a.w;
    } else {
#pragma unroll
      for (int i = q; i < q + 4; ++i) f[i] = e + i < n ? p[e + i] : 0.f;
    }
  }
}

template <int V> __device__ __forceinline__ void store_f32_part(float *p, int e, int n, const float (&f)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (e + i < n) p[e + i] = f[i];
}

template <int T> __device__ __forceinline__ float team_sum(float s) {
#pragma unroll
  for (int o = T / 2; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  return s;
}

// sum over a workgroup of W waves in wave order; `slot` alternates between two
// halves of red so that one barrier a sum is enough
template <int W> __device__ __forceinline__ float block_sum(float s, float *red, int slot) {
  s = team_sum<64>(s);
  if ((threadIdx.x & 63) == 0) red[slot * W + (threadIdx.x >> 6)] = s;
  __syncthreads();
  float t = red[slot * W];
#pragma unroll
  for (int w = 1; w < W; ++w) t += red[slot * W + w];
  return t;
}

// ---- forward ------------------------------------------------------------------

struct FwdArgs {
  long long rows;
  int c;
  float eps, inv_c;
  const void *x;
  const float *gamma, *beta;
  void *y;
  float *mean, *rstd;
};

// sum of f over the elements that count
template <int DT, int ROW> __device__ __forceinline__ float vec_sum(const u32x4_t &v, const Place<DT, ROW> &at, int c) {
  constexpr int V = Store<DT>::VEC;
  float f[V];
  unpack<DT>(v, f);
  // (past a short row's end, and in vectors past the end, the elements are zero)
  if constexpr (ROW == RAGGED) {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = at.has(i, c) ? f[i] : 0.f;
  }
#pragma unroll
  for (int w = V / 2; w >= 1; w >>= 1)
#pragma unroll
    for (int i = 0; i < w; ++i) f[i] += f[i + w];
  return f[0];
}

// their squared distance from the mean
template <int DT, int ROW>
__device__ __forceinline__ float sq_dist(const u32x4_t &v, const Place<DT, ROW> &at, int c, float mean) {
  constexpr int V = Store<DT>::VEC;
  float f[V], q = 0.f;
  unpack<DT>(v, f);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float d = f[i] - mean;
    q += at.has(i, c) ? d * d : 0.f;
  }
  return q;
}

// the same of the vector at element e of a chunk of n
template <int DT> __device__ __forceinline__ float sum_part(const u32x4_t &v) {
  return vec_sum<DT, FULL>(v, Place<DT, FULL>(0, Store<DT>::VEC), Store<DT>::VEC);
}
template <int DT> __device__ __forceinline__ float sq_dist_part(const u32x4_t &v, int e, int n, float mean) {
  constexpr int V = Store<DT>::VEC;
  float f[V], q = 0.f;
  unpack<DT>(v, f);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float d = f[i] - mean;
    q += e + i < n ? d * d : 0.f;
  }
  return q;
}

template <int DT>
__device__ __forceinline__ u32x4_t normalised(const u32x4_t &v, float mean, float rstd,
                                              const float (&ga)[Store<DT>::VEC], const float (&be)[Store<DT>::VEC]) {
  constexpr int V = Store<DT>::VEC;
  float f[V];
  unpack<DT>(v, f);
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = (f[i] - mean) * rstd * ga[i] + be[i];
  return pack<DT>(f);
}

// Teams of T lanes, NV vectors a lane, U rows a team, their loads all in flight.  Memory
// bounds it: 2^24 bf16 rows of 16 175 to 202 us on several cards, 6.0 to 6.9 TB/s; 65536 fp32
// rows of 1024 90 us, 5.9.
template <int DT, int T, int NV, int U, int ROW>
__global__ __launch_bounds__(256) void norm_fwd_wave(FwdArgs a) {
  constexpr int V = Store<DT>::VEC;
  using S = typename Store<DT>::T;
  const int t = threadIdx.x % T;
  // rows of a wave's teams follow each other, so that each of its instructions covers them
  // in one piece (with U rows of its own a team: 306 us for the 2^24 of 16 instead of 210,
  // before they passed the cache by)
  const long long r0 = (long long)blockIdx.x * (256 / T * U) + threadIdx.x / T;
  auto row = [&](int u) { return r0 + u * (256 / T); };
  u32x4_t v[U][NV];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const S *x = (const S *)a.x + min(row(u), a.rows - 1) * a.c;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[u][i] = load_vec<DT, ROW, true>(x, Place<DT, ROW>(t + T * i, a.c), a.c);
  }
  float mean[U], rstd[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s += vec_sum<DT, ROW>(v[u][i], Place<DT, ROW>(t + T * i, a.c), a.c);
    mean[u] = team_sum<T>(s) * a.inv_c;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) q += sq_dist<DT, ROW>(v[u][i], Place<DT, ROW>(t + T * i, a.c), a.c, mean[u]);
    rstd[u] = 1.0f / sqrtf(team_sum<T>(q) * a.inv_c + a.eps);
    if (t == 0 && row(u) < a.rows) {
      a.mean[row(u)] = mean[u];
      a.rstd[row(u)] = rstd[u];
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place<DT, ROW> at(t + T * i, a.c);
    float ga[V], be[V];
    load_f32<DT, ROW, true>(a.gamma, at, a.c, ga);
    load_f32<DT, ROW, true>(a.beta, at, a.c, be);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (row(u) < a.rows)
        store_vec<DT, ROW>((S *)a.y + row(u) * a.c, at, a.c, normalised<DT>(v[u][i], mean[u], rstd[u], ga, be));
  }
}

// a workgroup a row
template <int DT, int TH, int NV, int ROW> __global__ __launch_bounds__(TH) void norm_fwd_block(FwdArgs a) {
  constexpr int V = Store<DT>::VEC, W = TH / 64;
  using S = typename Store<DT>::T;
  __shared__ float red[2 * W];
  const long long r = blockIdx.x;
  const int t = threadIdx.x;
  const S *row = (const S *)a.x + r * a.c;
  u32x4_t v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = load_vec<DT, ROW, false>(row, Place<DT, ROW>(t + TH * i, a.c), a.c);
  float s = 0.f, q = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) s += vec_sum<DT, ROW>(v[i], Place<DT, ROW>(t + TH * i, a.c), a.c);
  const float mean = block_sum<W>(s, red, 0) * a.inv_c;
#pragma unroll
  for (int i = 0; i < NV; ++i) q += sq_dist<DT, ROW>(v[i], Place<DT, ROW>(t + TH * i, a.c), a.c, mean);
  const float rstd = 1.0f / sqrtf(block_sum<W>(q, red, 1) * a.inv_c + a.eps);
  if (t == 0) {
    a.mean[r] = mean;
    a.rstd[r] = rstd;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place<DT, ROW> at(t + TH * i, a.c);
    if (at.any()) {
      float ga[V], be[V];
      load_f32<DT, ROW, false>(a.gamma, at, a.c, ga);
      load_f32<DT, ROW, false>(a.beta, at, a.c, be);
      store_vec<DT, ROW>((S *)a.y + r * a.c, at, a.c, normalised<DT>(v[i], mean, rstd, ga, be));
    }
  }
}

// rows in chunks: grid (chunk, row).  part[row][chunk] = (mean, sum of squares about it)
template <int DT, int NV, bool RAG>
__global__ __launch_bounds__(256) void norm_fwd_chunk_stats(FwdArgs a, int chunk, float2 *part) {
  constexpr int V = Store<DT>::VEC;
  using S = typename Store<DT>::T;
  __shared__ float red[8];
  const long long r = blockIdx.y + (long long)gridDim.y * blockIdx.z;
  if (r >= a.rows) return;
  const int beg = blockIdx.x * chunk, n = min(chunk, a.c - beg);
  const S *row = (const S *)a.x + r * a.c + beg;
  float mean = 0.f, m2 = 0.f;
  int have = 0;
  for (int o = 0; o < n; o += 256 * V * NV) {  // pieces that the registers hold, combined one after the other
    const int k = min(n - o, 256 * V * NV);
    u32x4_t v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = load_part<DT, RAG>(row + o, ((int)threadIdx.x + 256 * i) * V, k);
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s += sum_part<DT>(v[i]);
    const float pm = block_sum<4>(s, red, 0) / (float)k;
#pragma unroll
    for (int i = 0; i < NV; ++i) q += sq_dist_part<DT>(v[i], ((int)threadIdx.x + 256 * i) * V, k, pm);
    const float pq = block_sum<4>(q, red, 1);
    const float d = pm - mean, w = (float)k / (float)(have + k);
    m2 += pq + (have > 0 ? d * d * (float)have * w : 0.f);  // (the first d is the mean itself: its square may be infinite)
    mean += d * w;
    have += k;
  }
  if (threadIdx.x == 0) part[r * gridDim.x + blockIdx.x] = make_float2(mean, m2);
}

template <int DT, bool RAG>
__global__ __launch_bounds__(256) void norm_fwd_chunk_apply(FwdArgs a, int chunk, const float2 *part) {
  constexpr int V = Store<DT>::VEC;
  using S = typename Store<DT>::T;
  __shared__ float red[8];
  const long long r = blockIdx.y + (long long)gridDim.y * blockIdx.z;
  if (r >= a.rows) return;
  const int beg = blockIdx.x * chunk, n = min(chunk, a.c - beg), nch = gridDim.x;
  const float2 *pr = part + r * nch;
  float s = 0.f, q = 0.f;
  for (int i = threadIdx.x; i < nch; i += 256) s += pr[i].x * (float)min(chunk, a.c - i * chunk);
  const float mean = block_sum<4>(s, red, 0) * a.inv_c;
  for (int i = threadIdx.x; i < nch; i += 256) {
    const float2 p = pr[i];
    const float d = p.x - mean;
    q += p.y + d * d * (float)min(chunk, a.c - i * chunk);
  }
  const float rstd = 1.0f / sqrtf(block_sum<4>(q, red, 1) * a.inv_c + a.eps);
  if (beg == 0 && threadIdx.x == 0) {
    a.mean[r] = mean;
    a.rstd[r] = rstd;
  }
  const S *row = (const S *)a.x + r * a.c + beg;
  S *out = (S *)a.y + r * a.c + beg;
  for (int e = threadIdx.x * V; e < n; e += 256 * V) {
    float ga[V], be[V];
    const u32x4_t v = load_part<DT, RAG>(row, e, n);
    load_f32_part<V>(a.gamma + beg, e, n, ga);
    load_f32_part<V>(a.beta + beg, e, n, be);
    store_part<DT, RAG>(out, e, n, normalised<DT>(v, mean, rstd, ga, be));
  }
}

// ---- backward -----------------------------------------------------------------

struct BwdArgs {
  long long rows;
  int c;
  float inv_c;
  const void *dy, *x;
  const float *gamma, *mean, *rstd;
  void *dx;
  float *pg, *pb;  // [workgroup][c] partial sums of dgamma and dbeta
};

// adds a vector's share of the two sums over the row (of the elements that count; dy is
// zero past the end, and so has to be xh, where mean rstd may be infinite though no value's
// xh is: mean and rstd are zero for FULL vectors past the end) and of dgamma, dbeta
template <int DT, int ROW>
__device__ __forceinline__ void bwd_sums(const u32x4_t &xv, const u32x4_t &dv, const Place<DT, ROW> &at, int c, float mean,
                                         float rstd, const float (&ga)[Store<DT>::VEC], float &sg, float &sgx,
                                         float (&dg)[Store<DT>::VEC], float (&db)[Store<DT>::VEC]) {
  constexpr int V = Store<DT>::VEC;
  float x[V], d[V];
  unpack<DT>(xv, x);
  unpack<DT>(dv, d);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float xh = (x[i] - mean) * rstd;
    if constexpr (ROW == SHORT) xh = at.has(i, c) ? xh : 0.f;
    const float g = mul_rounded(d[i], ga[i]);
    dg[i] += d[i] * xh;
    db[i] += d[i];
    if constexpr (ROW == RAGGED) {
      sg += at.has(i, c) ? g : 0.f;
      sgx += at.has(i, c) ? g * xh : 0.f;
    } else {
      sg += g;
      sgx += g * xh;
    }
  }
}

template <int DT>
__device__ __forceinline__ u32x4_t bwd_dx(const u32x4_t &xv, const u32x4_t &dv, float mean, float rstd,
                                          const float (&ga)[Store<DT>::VEC], float mg, float mgx) {
  constexpr int V = Store<DT>::VEC;
  float x[V], d[V];
  unpack<DT>(xv, x);
  unpack<DT>(dv, d);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float xh = (x[i] - mean) * rstd, g = mul_rounded(d[i], ga[i]);
    x[i] = rstd * ((g - mg) - xh * mgx);
  }
  return pack<DT>(x);
}

// Teams of T lanes; every team walks rows and keeps its columns' sums.  2^24 bf16 rows of 16
// 295 to 318 us on several cards, 5.5 to 5.9 TB/s; 65536 fp32 rows of 1024 139 to 150 us, 5.4 to
// 5.8.
template <int DT, int T, int NV, int U, int ROW>
__global__ __launch_bounds__(256) void norm_bwd_wave(BwdArgs a) {
  constexpr int V = Store<DT>::VEC;
  using S = typename Store<DT>::T;
  __shared__ float red[4][T * V];
  const int t = threadIdx.x % T;
  float ga[NV][V], dg[NV][V], db[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    load_f32<DT, ROW, true>(a.gamma, Place<DT, ROW>(t + T * i, a.c), a.c, ga[i]);
#pragma unroll
    for (int j = 0; j < V; ++j) dg[i][j] = db[i][j] = 0.f;
  }
  constexpr int RB = 256 / T * U;  // rows a workgroup takes at a time
  for (long long rb = (long long)blockIdx.x * RB; rb < a.rows; rb += (long long)gridDim.x * RB) {
    u32x4_t xv[U][NV], dv[U][NV];
    float mean[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long r = rb + u * (256 / T) + threadIdx.x / T;
      const bool in = r < a.rows;
      const long long have = in ? r : a.rows - 1;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Place<DT, ROW> at(t + T * i, a.c);
        xv[u][i] = load_vec<DT, ROW, ROW != RAGGED>((const S *)a.x + have * a.c, at, a.c, in);
        dv[u][i] = load_vec<DT, ROW, ROW != RAGGED>((const S *)a.dy + have * a.c, at, a.c, in);
      }
      const bool use = in && (NV > 1 || Place<DT, ROW>(t, a.c).any());
      mean[u] = use ? a.mean[have] : 0.f;
      rstd[u] = use ? a.rstd[have] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long r = rb + u * (256 / T) + threadIdx.x / T;
      float sg = 0.f, sgx = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Place<DT, ROW> at(t + T * i, a.c);
        const bool use = NV == 1 || ROW == RAGGED || at.any();
        bwd_sums<DT, ROW>(xv[u][i], dv[u][i], at, a.c, use ? mean[u] : 0.f, use ? rstd[u] : 0.f, ga[i], sg, sgx, dg[i], db[i]);
      }
      const float mg = team_sum<T>(sg) * a.inv_c, mgx = team_sum<T>(sgx) * a.inv_c;
      if (r < a.rows) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          store_vec<DT, ROW>((S *)a.dx + r * a.c, Place<DT, ROW>(t + T * i, a.c), a.c,
                             bwd_dx<DT>(xv[u][i], dv[u][i], mean[u], rstd[u], ga[i], mg, mgx));
      }
    }
  }
  // the workgroup's teams: those of a wave by exchanges, the four waves in order
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float *s = k ? db[i] : dg[i];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        float z = s[j];
#pragma unroll
        for (int o = T; o < 64; o <<= 1) z += __shfl_xor(z, o, 64);
        if (lane < T) red[wave][lane * V + j] = z;
      }
      __syncthreads();
      for (int j = threadIdx.x; j < T * V; j += 256) {
        const Place<DT, ROW> at(j / V + T * i, a.c);
        if (at.any() && at.has(j % V, a.c))
          (k ? a.pb : a.pg)[(long long)blockIdx.x * a.c + at.e + j % V] = (red[0][j] + red[1][j]) + (red[2][j] + red[3][j]);
      }
      __syncthreads();
    }
  }
}

// a workgroup a row at a time; 1024 threads, of 128 registers each, read gamma again for
// every row where it would not fit beside the sums (2000 fp32 rows of 12345 105 us with
// it kept, 78 so)
template <int DT, int TH, int NV, int ROW> __global__ __launch_bounds__(TH) void norm_bwd_block(BwdArgs a) {
  constexpr int V = Store<DT>::VEC, W = TH / 64;
  constexpr bool kKeep = TH < 1024 || NV * V <= 12;
  using S = typename Store<DT>::T;
  __shared__ float red[4 * W];
  const int t = threadIdx.x;
  float ga[kKeep ? NV : 1][V], dg[NV][V], db[NV][V];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if constexpr (kKeep) load_f32<DT, ROW, false>(a.gamma, Place<DT, ROW>(t + TH * i, a.c), a.c, ga[i]);
#pragma unroll
    for (int j = 0; j < V; ++j) dg[i][j] = db[i][j] = 0.f;
  }
  int half = 0;
  for (long long r = blockIdx.x; r < a.rows; r += gridDim.x, half ^= 1) {
    u32x4_t xv[NV], dv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place<DT, ROW> at(t + TH * i, a.c);
      xv[i] = load_vec<DT, ROW, false>((const S *)a.x + r * a.c, at, a.c);
      dv[i] = load_vec<DT, ROW, false>((const S *)a.dy + r * a.c, at, a.c);
    }
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place<DT, ROW> at(t + TH * i, a.c);
      if constexpr (!kKeep) load_f32<DT, ROW, false>(a.gamma, at, a.c, ga[0]);
      const bool use = ROW == RAGGED || at.any();
      bwd_sums<DT, ROW>(xv[i], dv[i], at, a.c, use ? mean : 0.f, use ? rstd : 0.f, ga[kKeep ? i : 0], sg, sgx, dg[i], db[i]);
    }
    sg = team_sum<64>(sg);
    sgx = team_sum<64>(sgx);
    // the halves of red alternate: one barrier a row
    if ((t & 63) == 0) {
      red[half * 2 * W + (t >> 6)] = sg;
      red[half * 2 * W + W + (t >> 6)] = sgx;
    }
    __syncthreads();
    float mg = 0.f, mgx = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      mg += red[half * 2 * W + w];
      mgx += red[half * 2 * W + W + w];
    }
    mg *= a.inv_c;
    mgx *= a.inv_c;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place<DT, ROW> at(t + TH * i, a.c);
      if constexpr (!kKeep) load_f32<DT, ROW, false>(a.gamma, at, a.c, ga[0]);
      store_vec<DT, ROW>((S *)a.dx + r * a.c, at, a.c, bwd_dx<DT>(xv[i], dv[i], mean, rstd, ga[kKeep ? i : 0], mg, mgx));
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place<DT, ROW> at(t + TH * i, a.c);
    if (at.any()) {
      store_f32<DT, ROW>(a.pg + (long long)blockIdx.x * a.c, at, a.c, dg[i]);
      store_f32<DT, ROW>(a.pb + (long long)blockIdx.x * a.c, at, a.c, db[i]);
    }
  }
}

// rows in chunks: part[row][chunk] = (sum g, sum g xh)
template <int DT, bool RAG>
__global__ __launch_bounds__(256) void norm_bwd_chunk_sums(BwdArgs a, int chunk, float2 *part) {
  constexpr int V = Store<DT>::VEC;
  using S = typename Store<DT>::T;
  __shared__ float red[8];
  const long long r = blockIdx.y + (long long)gridDim.y * blockIdx.z;
  if (r >= a.rows) return;
  const int beg = blockIdx.x * chunk, n = min(chunk, a.c - beg);
  const S *x = (const S *)a.x + r * a.c + beg, *dy = (const S *)a.dy + r * a.c + beg;
  const float mean = a.mean[r], rstd = a.rstd[r];
  float sg = 0.f, sgx = 0.f, unused0[V] = {}, unused1[V] = {};
  for (int e = threadIdx.x * V; e < n; e += 256 * V) {
    float ga[V];
    const u32x4_t xv = load_part<DT, RAG>(x, e, n), dv = load_part<DT, RAG>(dy, e, n);
    load_f32_part<V>(a.gamma + beg, e, n, ga);
    constexpr int PART = RAG ? SHORT : FULL;  // the last vector may end early
    bwd_sums<DT, PART>(xv, dv, Place<DT, PART>(0, V), n - e, mean, rstd, ga, sg, sgx, unused0, unused1);
  }
  sg = block_sum<4>(sg, red, 0);
  sgx = block_sum<4>(sgx, red, 1);
  if (threadIdx.x == 0) part[r * gridDim.x + blockIdx.x] = make_float2(sg, sgx);
}

// One vector column a thread over a block of `per` rows: dx, and the block's share of
// dgamma and dbeta.  grid (64-vector column strip, row block); nch chunks a row in part.
// (A wave a workgroup: 8 rows of 65536 leave three quarters of the compute units idle with
// strips of 256 vectors: the pass 8.6 us instead of 7.4, in bf16 10.8 instead of 8.7.)
constexpr int kColRows = 16;  // rows whose sums are combined at a time
template <int DT, bool RAG>
__global__ __launch_bounds__(64) void norm_bwd_columns(BwdArgs a, int per, int nch, const float2 *part) {
  constexpr int V = Store<DT>::VEC;
  using S = typename Store<DT>::T;
  __shared__ float2 rs[kColRows];
  const long long e = ((long long)blockIdx.x * 64 + threadIdx.x) * V;
  float ga[V] = {}, dg[V] = {}, db[V] = {};
  if (e < a.c) load_f32_part<V>(a.gamma, (int)e, a.c, ga);
  const long long rend = min(((long long)blockIdx.y + 1) * per, a.rows);
  for (long long r0 = (long long)blockIdx.y * per; r0 < rend; r0 += kColRows) {
    const int nr = (int)min((long long)kColRows, rend - r0);
    {  // 64 lanes for one row to four a row for kColRows
      int lanes = 64;
      while (lanes * nr > 64) lanes >>= 1;
      const int i = threadIdx.x / lanes;
      float sg = 0.f, sgx = 0.f;
      if (i < nr) {
#pragma unroll 8
        for (int k = threadIdx.x & (lanes - 1); k < nch; k += lanes) {
          const float2 p = part[(r0 + i) * nch + k];
          sg += p.x;
          sgx += p.y;
        }
      }
      for (int o = lanes / 2; o >= 1; o >>= 1) {
        sg += __shfl_xor(sg, o, 64);
        sgx += __shfl_xor(sgx, o, 64);
      }
      if (i < nr && (threadIdx.x & (lanes - 1)) == 0) rs[i] = make_float2(sg * a.inv_c, sgx * a.inv_c);
    }
    __syncthreads();
    if (e < a.c) {
      for (int i = 0; i < nr; ++i) {
        const long long at = (r0 + i) * a.c;
        const u32x4_t xv = load_part<DT, RAG>((const S *)a.x + at, (int)e, a.c);
        const u32x4_t dv = load_part<DT, RAG>((const S *)a.dy + at, (int)e, a.c);
        const float mean = a.mean[r0 + i], rstd = a.rstd[r0 + i];
        float s0 = 0.f, s1 = 0.f;
        bwd_sums<DT, FULL>(xv, dv, Place<DT, FULL>(0, V), V, mean, rstd, ga, s0, s1, dg, db);
        store_part<DT, RAG>((S *)a.dx + at, (int)e, a.c, bwd_dx<DT>(xv, dv, mean, rstd, ga, rs[i].x, rs[i].y));
      }
    }
    __syncthreads();
  }
  if (e < a.c) {
    store_f32_part<V>(a.pg + (long long)blockIdx.y * a.c, (int)e, a.c, dg);
    store_f32_part<V>(a.pb + (long long)blockIdx.y * a.c, (int)e, a.c, db);
  }
}

// ---- plans --------------------------------------------------------------------

int vec_of(int dtype) { return dtype == DT_BF16 ? Store<DT_BF16>::VEC : Store<DT_F32>::VEC; }

// Lanes of a team and vectors a lane for rows of nv <= 512 vectors: the fewest lanes of
// those with one, two or three vectors that waste least (33 vectors: 16 lanes with
// three rather than 64 with one; two lanes' three vectors are too short a piece of memory:
// 2^20 fp32 rows of 17 58.7 us forward, 32.8 with eight lanes).
struct Team {
  int lanes, vecs;
};
Team team_of(long long nv) {
  if (nv > 256) return {64, 8};
  if (nv > 192) return {64, 4};
  if (nv > 128) return {64, 3};
  if (nv > 96) return {64, 2};
  for (int t = 1; t < 64; t *= 2) {
    if (nv <= t) return {t, 1};
    if (t >= 4 && nv > t * 2 && nv <= t * 3) return {t, 3};
  }
  return {64, 1};
}

// elements of a chunk (a multiple of the 256 vectors of one load round) and chunks
// a row, for rows cut over workgroups: about four workgroups a compute unit and
// at most 1024 chunks
void plan_chunks(long long rows, int c, int V, int *chunk, int *nch) {
  const long long unit = 256LL * V, units = (c + unit - 1) / unit;
  const long long want = (4LL * kNumCUs + rows - 1) / rows;
  long long per = (units + want - 1) / want;
  while ((units + per - 1) / per > 1024) ++per;
  *chunk = (int)(per * unit < (1LL << 31) - unit ? per * unit : c);
  *nch = (int)((c + (long long)*chunk - 1) / *chunk);
}

// Whether the forward pass cuts rows into chunks: past the 2^16 values that a workgroup of
// 1024 threads holds in registers, and from 2^14 on when there are fewer rows than compute
// units (8 rows of 65536 fp32 values 11.3 us with a workgroup a row).
bool fwd_chunked(long long rows, int c) { return c > 65536 || (c > 16384 && rows < kNumCUs); }

// Backward: past what 1024 threads hold of x, dy and the column sums.
bool bwd_chunked(int c) { return c > 16384; }

// Rows of a block of the column pass: a multiple of kColRows that leaves about four blocks a
// compute unit over 256 vectors each.  (The launch's strips are of 64, a wave each: sixteen
// workgroups a compute unit.)
int column_rows(long long rows, int c, int V) {
  const long long strips = (c + 256LL * V - 1) / (256LL * V), want = (4LL * kNumCUs + strips - 1) / strips;
  const long long per = (rows + want - 1) / want;
  return (int)((per + kColRows - 1) / kColRows * kColRows);
}

// workgroups of the backward pass that keep column sums (rows of partials)
int bwd_groups(long long rows, int c, int dtype) {
  const int V = vec_of(dtype);
  const long long nv = ((long long)c + V - 1) / V;
  if (bwd_chunked(c)) {
    const int per = column_rows(rows, c, V);
    return (int)((rows + per - 1) / per);
  }
  // rows a workgroup takes at a time; a workgroup of at least twice that keeps the
  // partial sums (8 bytes a column and workgroup) small beside the rows, but every
  // compute unit should have one
  long long per = 1, cap = kNumCUs;
  if (c <= 1024) {
    const Team t = team_of(nv);
    per = 256 / t.lanes * (t.vecs == 1 ? 2 : 1);
    cap = 8 * kNumCUs;
  } else if (c <= 4096) {
    cap = 4 * kNumCUs;
  }
  const long long need = (rows + per - 1) / per;
  long long groups = need / 2 > kNumCUs ? need / 2 : kNumCUs;
  if (groups > cap) groups = cap;
  return (int)(need < groups ? need : groups);
}

template <int DT, int ROW> hipError_t fwd(const FwdArgs &a, void *ws, hipStream_t st) {
  constexpr int V = Store<DT>::VEC;
  const long long nv = ((long long)a.c + V - 1) / V;
  if (fwd_chunked(a.rows, a.c)) {
    constexpr bool RAG = ROW == RAGGED;
    int chunk, nch;
    plan_chunks(a.rows, a.c, V, &chunk, &nch);
    const unsigned gy = (unsigned)(a.rows < 32768 ? a.rows : 32768), gz = (unsigned)((a.rows + gy - 1) / gy);
    hipLaunchKernelGGL((norm_fwd_chunk_stats<DT, 4, RAG>), dim3(nch, gy, gz), dim3(256), 0, st, a, chunk, (float2 *)ws);
    hipLaunchKernelGGL((norm_fwd_chunk_apply<DT, RAG>), dim3(nch, gy, gz), dim3(256), 0, st, a, chunk, (const float2 *)ws);
    return hipGetLastError();
  }
#define CF_FWD_WAVE(T, NV, U)                                                                                       \
  {                                                                                                                 \
    const long long per = 256 / (T) * (U);                                                                          \
    hipLaunchKernelGGL((norm_fwd_wave<DT, T, NV, U, ROW>), dim3((unsigned)((a.rows + per - 1) / per)), dim3(256), 0, \
                       st, a);                                                                                      \
    return hipGetLastError();                                                                                       \
  }
#define CF_FWD_BLOCK(TH, NV)                                                                                    \
  {                                                                                                             \
    hipLaunchKernelGGL((norm_fwd_block<DT, TH, NV, ROW>), dim3((unsigned)a.rows), dim3(TH), 0, st, a);          \
    return hipGetLastError();                                                                                   \
  }
  if constexpr (ROW == SHORT) CF_FWD_WAVE(1, 1, 4)
  else {
    if (nv <= 512) {
      const Team t = team_of(nv);
      switch (t.lanes * 16 + t.vecs) {
        case 1 * 16 + 1: CF_FWD_WAVE(1, 1, 4)
        case 2 * 16 + 1: CF_FWD_WAVE(2, 1, 4)
        case 4 * 16 + 1: CF_FWD_WAVE(4, 1, 4)
        case 4 * 16 + 3: CF_FWD_WAVE(4, 3, 2)
        case 8 * 16 + 1: CF_FWD_WAVE(8, 1, 4)
        case 8 * 16 + 3: CF_FWD_WAVE(8, 3, 2)
        case 16 * 16 + 1: CF_FWD_WAVE(16, 1, 4)
        case 16 * 16 + 3: CF_FWD_WAVE(16, 3, 2)
        case 32 * 16 + 1: CF_FWD_WAVE(32, 1, 4)
        case 32 * 16 + 3: CF_FWD_WAVE(32, 3, 2)
        case 64 * 16 + 1: CF_FWD_WAVE(64, 1, 4)
        case 64 * 16 + 2: CF_FWD_WAVE(64, 2, 2)
        case 64 * 16 + 3: CF_FWD_WAVE(64, 3, 1)
        case 64 * 16 + 4: CF_FWD_WAVE(64, 4, 1)
        default: CF_FWD_WAVE(64, 8, 1)
      }
    }
    if (nv <= 768) CF_FWD_BLOCK(256, 3)
    if (nv <= 1024) CF_FWD_BLOCK(256, 4)
    if (nv <= 1536) CF_FWD_BLOCK(256, 6)
    if (nv <= 2048) CF_FWD_BLOCK(256, 8)
    if (nv <= 3 * 1024) CF_FWD_BLOCK(1024, 3)
    if (nv <= 4096) CF_FWD_BLOCK(1024, 4)
    if constexpr (DT == DT_F32) {
      if (nv <= 8192) CF_FWD_BLOCK(1024, 8)
      CF_FWD_BLOCK(1024, 16)
    } else {
      CF_FWD_BLOCK(1024, 8)
    }
  }
#undef CF_FWD_WAVE
#undef CF_FWD_BLOCK
}

template <int DT, int ROW> hipError_t bwd(const BwdArgs &a, int groups, void *rowpart, hipStream_t st) {
  constexpr int V = Store<DT>::VEC;
  const long long nv = ((long long)a.c + V - 1) / V;
  if (bwd_chunked(a.c)) {
    constexpr bool RAG = ROW == RAGGED;
    int chunk, nch;
    plan_chunks(a.rows, a.c, V, &chunk, &nch);
    const unsigned gy = (unsigned)(a.rows < 32768 ? a.rows : 32768), gz = (unsigned)((a.rows + gy - 1) / gy);
    hipLaunchKernelGGL((norm_bwd_chunk_sums<DT, RAG>), dim3(nch, gy, gz), dim3(256), 0, st, a, chunk, (float2 *)rowpart);
    hipLaunchKernelGGL((norm_bwd_columns<DT, RAG>), dim3((unsigned)((nv + 63) / 64), groups), dim3(64), 0, st, a,
                       column_rows(a.rows, a.c, V), nch, (const float2 *)rowpart);
    return hipGetLastError();
  }
#define CF_BWD_WAVE(T, NV, U)                                                                        \
  {                                                                                                  \
    hipLaunchKernelGGL((norm_bwd_wave<DT, T, NV, U, ROW>), dim3(groups), dim3(256), 0, st, a);       \
    return hipGetLastError();                                                                        \
  }
#define CF_BWD_BLOCK(TH, NV)                                                                         \
  {                                                                                                  \
    hipLaunchKernelGGL((norm_bwd_block<DT, TH, NV, ROW>), dim3(groups), dim3(TH), 0, st, a);         \
    return hipGetLastError();                                                                        \
  }
  if constexpr (ROW == SHORT) CF_BWD_WAVE(1, 1, 2)
  else {
    if (a.c <= 1024) {
      const Team t = team_of(nv);
      switch (t.lanes * 16 + t.vecs) {
        case 1 * 16 + 1: CF_BWD_WAVE(1, 1, 2)
        case 2 * 16 + 1: CF_BWD_WAVE(2, 1, 2)
        case 4 * 16 + 1: CF_BWD_WAVE(4, 1, 2)
        case 4 * 16 + 3: CF_BWD_WAVE(4, 3, 1)
        case 8 * 16 + 1: CF_BWD_WAVE(8, 1, 2)
        case 8 * 16 + 3: CF_BWD_WAVE(8, 3, 1)
        case 16 * 16 + 1: CF_BWD_WAVE(16, 1, 2)
        case 16 * 16 + 3: CF_BWD_WAVE(16, 3, 1)
        case 32 * 16 + 1: CF_BWD_WAVE(32, 1, 2)
        case 32 * 16 + 3: CF_BWD_WAVE(32, 3, 1)
        case 64 * 16 + 1: CF_BWD_WAVE(64, 1, 2)
        case 64 * 16 + 2: CF_BWD_WAVE(64, 2, 1)
        case 64 * 16 + 3: CF_BWD_WAVE(64, 3, 1)
        default: CF_BWD_WAVE(64, 4, 1)
      }
    }
    // (up to 16384 values: four vectors of fp32, two of bf16 for each of 1024 threads)
    if constexpr (DT == DT_F32) {
      if (nv <= 512) CF_BWD_BLOCK(256, 2)
      if (nv <= 768) CF_BWD_BLOCK(256, 3)
      if (nv <= 1024) CF_BWD_BLOCK(256, 4)
      if (nv <= 2048) CF_BWD_BLOCK(1024, 2)
      if (nv <= 3 * 1024) CF_BWD_BLOCK(1024, 3)
      CF_BWD_BLOCK(1024, 4)
    } else {
      if (nv <= 256) CF_BWD_BLOCK(256, 1)
      if (nv <= 512) CF_BWD_BLOCK(256, 2)
      if (nv <= 1024) CF_BWD_BLOCK(1024, 1)
      CF_BWD_BLOCK(1024, 2)
    }
  }
#undef CF_BWD_WAVE
#undef CF_BWD_BLOCK
}

// How the rows lie picks the kernels.  `bytes` of all tensors past what the last-level cache
// holds pass it by: 2^24 bf16 rows of 16 176 us forward instead of 210 and 295 backward
// instead of 349, 65536 fp32 rows of 1024 89 / 150 instead of 95 / 169; but at 256 MiB, 2^21
// fp32 rows of 16, 44.6 instead of 43.4 forward.
template <int DT, class F> hipError_t by_row(int c, long long bytes, F f) {
  constexpr int V = Store<DT>::VEC;
  if (c % V == 0 && bytes > kStreamBytes) return f(std::integral_constant<int, STREAM>{});
  if (c % V == 0) return f(std::integral_constant<int, FULL>{});
  if (c > V) return f(std::integral_constant<int, RAGGED>{});
  return f(std::integral_constant<int, SHORT>{});
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

size_t layernorm_fwd_workspace(long long rows, int c, int dtype) {
  if (!fwd_chunked(rows, c)) return 0;
  int chunk, nch;
  plan_chunks(rows, c, vec_of(dtype), &chunk, &nch);
  return up16((size_t)rows * nch * sizeof(float2));
}

size_t layernorm_bwd_workspace(long long rows, int c, int dtype) {
  const size_t part = up16((size_t)bwd_groups(rows, c, dtype) * c * sizeof(float));
  size_t n = 2 * part;
  if (bwd_chunked(c)) {
    int chunk, nch;
    plan_chunks(rows, c, vec_of(dtype), &chunk, &nch);
    n += up16((size_t)rows * nch * sizeof(float2));
  }
  return n;
}

hipError_t launch_layernorm_fwd(long long rows, int c, int dtype, const void *x, const float *gamma, const float *beta,
                                float eps, void *y, float *mean, float *rstd, void *ws, hipStream_t st) {
  const long long es = dtype == DT_BF16 ? 2 : 4, bytes = 2 * rows * c * es;
  // a launch has fewer than 2^32 threads: rows of 2^32 values at a time, a thread for at
  // least two (the chunks of longer rows lie along several grid dimensions)
  const long long pieces = fwd_chunked(rows, c) ? 1 : (rows * c + (1LL << 32) - 1) >> 32, per = (rows + pieces - 1) / pieces;
  for (long long r = 0; r < rows; r += per) {
    const FwdArgs a{min(per, rows - r), c, eps, 1.0f / (float)c, (const char *)x + r * c * es, gamma, beta, (char *)y + r * c * es,
                    mean + r, rstd + r};
    const hipError_t e =
        dtype == DT_BF16
            ? by_row<DT_BF16>(c, bytes, [&](auto row) { return fwd<DT_BF16, decltype(row)::value>(a, ws, st); })
            : by_row<DT_F32>(c, bytes, [&](auto row) { return fwd<DT_F32, decltype(row)::value>(a, ws, st); });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_layernorm_bwd(long long rows, int c, int dtype, const void *dy, const void *x, const float *gamma,
                                const float *mean, const float *rstd, void *dx, float *dgamma, float *dbeta, void *ws,
                                hipStream_t st) {
  const long long bytes = 3 * rows * c * (dtype == DT_BF16 ? 2 : 4);
  const int groups = bwd_groups(rows, c, dtype);
  const size_t part = up16((size_t)groups * c * sizeof(float));
  // one row of partials is the result itself
  float *pg = groups == 1 ? dgamma : (float *)ws, *pb = groups == 1 ? dbeta : (float *)((char *)ws + part);
  const BwdArgs a{rows, c, 1.0f / (float)c, dy, x, gamma, mean, rstd, dx, pg, pb};
  void *rowpart = (char *)ws + 2 * part;
  const hipError_t e =
      dtype == DT_BF16
          ? by_row<DT_BF16>(c, bytes, [&](auto row) { return bwd<DT_BF16, decltype(row)::value>(a, groups, rowpart, st); })
          : by_row<DT_F32>(c, bytes, [&](auto row) { return bwd<DT_F32, decltype(row)::value>(a, groups, rowpart, st); });
  if (e != hipSuccess || groups == 1) return e;
  const SumJob jobs[2] = {{pg, dgamma, groups, c}, {pb, dbeta, groups, c}};
  return launch_sum_batch(jobs, 2, st);
}

}  // namespace cf
