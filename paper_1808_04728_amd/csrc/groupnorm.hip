// groupnorm.hip -- group normalisation of NDHWC tensors with the activation behind it,
// forward and backward.
//
//   u = (x - mean) rstd gamma + beta,  y = act(u)            mean, rstd of a sample's group
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du xh,   xh = (x - mean) rstd
//   dx = rstd (gamma du - mean_g(gamma du) - xh mean_g(gamma du xh))
//
// Channels are innermost, so a sample is one run of vox * c values.  A workgroup's threads
// walk it a whole number of voxels a turn: T threads of V consecutive values each (16
// bytes), T V a multiple of c, so that a thread's V values have the same channels in every
// turn, whatever c is, and per-channel constants and sums stay in its registers.  (Vectors
// need no alignment.)  A sample is cut into slices; each leaves per-channel partial results,
// rows of a small matrix, which a second launch joins in a fixed order, and a third reads
// the data again and writes.  Groups of a few thousand values are one workgroup's, held in
// registers between the sums and the stores, in one launch.

#include <math.h>

#include <algorithm>
#include <numeric>

#include "activation.h"
#include "cf_common.h"
#include "cf_kernels.h"

namespace cf {
namespace {

constexpr int kThreads = 256;

// 16 bytes that start at any element
typedef uint32_t u32x4e2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4e4_t __attribute__((ext_vector_type(4), aligned(4)));

template <int DT> struct Run;
template <> struct Run<DT_F32> {
  static constexpr int V = 4;
  typedef u32x4e4_t Vec;
};
template <> struct Run<DT_BF16> {
  static constexpr int V = 8;
  typedef u32x4e2_t Vec;
};

template <int DT> __device__ __forceinline__ u32x4_t load_raw(const typename Store<DT>::T *p) {
  return *reinterpret_cast<const typename Run<DT>::Vec *>(p);
}
template <int DT> __device__ __forceinline__ void unpack(const u32x4_t &a, float (&f)[Run<DT>::V]) {
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(a[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(a[i] << 16);
      f[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
}
template <int DT> __device__ __forceinline__ void store_run(typename Store<DT>::T *p, const float (&f)[Run<DT>::V]) {
  u32x4_t a;
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = f2bf2(f[2 * i], f[2 * i + 1]);
  }
  *reinterpret_cast<typename Run<DT>::Vec *>(p) = a;
}

// How a sample is walked.  A turn is `width` = T V values = `rows` voxels; a slice is `turns`
// turns.  T threads are `parts` workgroups side by side.  The partial results of a slice are
// `prows` rows of c values: one, or (voxels of more values than a workgroup's turn) one for
// every voxel of a turn.
struct Walk {
  int c, groups, per;  // channels, groups, channels a group
  long long vox, count;  // voxels and values of a sample
  int threads, parts, rows, width;
  int turns, slices, prows;
};

// values of channel ch that slice s has in partial row r
__device__ __forceinline__ int row_count(const Walk &w, int s, int r, int ch) {
  const long long beg = (long long)s * w.turns * w.width;
  const long long len = min((long long)w.turns * w.width, w.count - beg);
  if (w.prows == 1) return (int)(len / w.c);
  return (int)max(0LL, (len - (r * w.c + ch) + w.width - 1) / w.width);
}

// mean and sum of squared distances of na and nb values joined
template <class T> __device__ __forceinline__ void join(T &mean, T &m2, T &na, T mb, T m2b, T nb) {
  const T n = na + nb;
  if (nb == (T)0) return;
  const T d = mb - mean, f = nb / n;
  mean += d * f;
  m2 += m2b + d * d * (na * f);
  na = n;
}

// ---- sums over a slice --------------------------------------------------------------

// Rows of `width` values in LDS joined to one row of c values a tree; f(dst, src) joins two
// entries.  n: rows.
template <class F> __device__ __forceinline__ void join_rows(int n, int c, F f) {
  while (n > 1) {
    const int h = (n + 1) >> 1, todo = (n - h) * c;
    for (int i = threadIdx.x; i < todo; i += kThreads) f(i, i + h * c);
    n = h;
    __syncthreads();
  }
}

constexpr int kUnroll = 4;

// part[(sample, slice, row)][c] = (mean, sum of squared distances to it) of each channel
template <int DT>
__global__ __launch_bounds__(kThreads) void gn_stats_kernel(Walk w, const void *x_, float2 *part) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  __shared__ float2 red[kThreads * V];
  __shared__ float cnt[kThreads * V];
  const int pb = blockIdx.x % w.parts, s = blockIdx.x / w.parts % w.slices;
  const long long n = blockIdx.x / w.parts / w.slices;
  const T *x = (const T *)x_ + n * w.count;
  const int tau = pb * kThreads + threadIdx.x;
  const bool live = tau < w.threads;
  const long long beg = (long long)s * w.turns * w.width;
  const long long end = min(beg + (long long)w.turns * w.width, w.count);
  const int f0 = tau * V;
  float mean[V], m2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) mean[j] = m2[j] = 0.f;
  float na = 0.f;
  long long e = beg + f0;
  if (live) {
    for (; e + (long long)(kUnroll - 1) * w.width + V <= end; e += (long long)kUnroll * w.width) {
      u32x4_t raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = load_raw<DT>(x + e + (long long)u * w.width);
      float v[kUnroll][V];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) unpack<DT>(raw[u], v[u]);
      const float nb = na + kUnroll, f = kUnroll / nb, g = na * f;
      na = nb;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        // the batch's own mean and distances, then joined to what there was
        const float mb = 0.25f * ((v[0][j] + v[1][j]) + (v[2][j] + v[3][j]));
        float q = 0.f;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) q += (v[u][j] - mb) * (v[u][j] - mb);
        const float d = mb - mean[j];
        mean[j] += d * f;
        m2[j] += q + d * d * g;
      }
    }
    for (; e + V <= end; e += w.width) {
      float v[V];
      unpack<DT>(load_raw<DT>(x + e), v);
      na += 1.f;
      const float f = 1.f / na;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = v[j] - mean[j];
        mean[j] += d * f;
        m2[j] += d * (v[j] - mean[j]);
      }
    }
  }
  // the sample's last values, fewer than a vector, end one thread's walk
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float nj = na;
    if (live && e < end && e + j < end) {
      const float v = to_f32<DT>(x[e + j]);
      nj += 1.f;
      const float d = v - mean[j];
      mean[j] += d / nj;
      m2[j] += d * (v - mean[j]);
    }
    red[threadIdx.x * V + j] = make_float2(mean[j], m2[j]);
    cnt[threadIdx.x * V + j] = nj;
  }
  __syncthreads();
  float2 *out = part + ((n * w.slices + s) * w.prows) * w.c;
  if (w.prows > 1 || w.parts > 1) {
    for (int i = threadIdx.x; i < kThreads * V; i += kThreads) {
      const int f = pb * kThreads * V + i;
      if (f < w.width) out[f] = red[i];
    }
    return;
  }
  join_rows(w.rows, w.c, [&](int a, int b) {
    float2 p = red[a];
    const float2 q = red[b];
    float na = cnt[a];
    join<float>(p.x, p.y, na, q.x, q.y, cnt[b]);
    red[a] = p;
    cnt[a] = na;
  });
  for (int i = threadIdx.x; i < w.c; i += kThreads) out[i] = red[i];
}

// mean and rstd of each sample's group from its partial rows
__global__ __launch_bounds__(kThreads) void gn_finish_stats_kernel(Walk w, float eps, const float2 *part, float *mean_,
                                                                   float *rstd_) {
  __shared__ double red[3][kThreads];
  const int g = blockIdx.x % w.groups;
  const long long n = blockIdx.x / w.groups;
  const int rows = w.slices * w.prows;
  double mean = 0.0, m2 = 0.0, na = 0.0;
  for (long long i = threadIdx.x; i < (long long)rows * w.per; i += kThreads) {
    const int r = (int)(i / w.per), ch = g * w.per + (int)(i % w.per);
    const float2 p = part[(n * rows + r) * w.c + ch];
    join<double>(mean, m2, na, p.x, p.y, row_count(w, r / w.prows, r % w.prows, ch));
  }
  red[0][threadIdx.x] = mean;
  red[1][threadIdx.x] = m2;
  red[2][threadIdx.x] = na;
  __syncthreads();
  for (int h = kThreads / 2; h > 0; h >>= 1) {
    if ((int)threadIdx.x < h) {
      const int a = threadIdx.x, b = a + h;
      join<double>(red[0][a], red[1][a], red[2][a], red[0][b], red[1][b], red[2][b]);
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    mean_[blockIdx.x] = (float)red[0][0];
    rstd_[blockIdx.x] = (float)(1.0 / sqrt(red[1][0] / red[2][0] + (double)eps));
  }
}

// ---- the second pass, forward -------------------------------------------------------

template <int DT, int ACT>
__global__ __launch_bounds__(kThreads) void gn_apply_kernel(Walk w, const void *x_, const float *gamma, const float *beta,
                                                            const float *mean_, const float *rstd_, float alpha, void *y_) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  const int pb = blockIdx.x % w.parts, s = blockIdx.x / w.parts % w.slices;
  const long long n = blockIdx.x / w.parts / w.slices;
  const T *x = (const T *)x_ + n * w.count;
  T *y = (T *)y_ + n * w.count;
  const int tau = pb * kThreads + threadIdx.x;
  if (tau >= w.threads) return;
  float mean[V], a[V], b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (tau * V + j) % w.c;
    const long long g = n * w.groups + ch / w.per;
    mean[j] = mean_[g];
    a[j] = rstd_[g] * gamma[ch];
    b[j] = beta[ch];
  }
  const long long beg = (long long)s * w.turns * w.width;
  const long long end = min(beg + (long long)w.turns * w.width, w.count);
  long long e = beg + tau * V;
  for (; e + (long long)(kUnroll - 1) * w.width + V <= end; e += (long long)kUnroll * w.width) {
    u32x4_t raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u] = load_raw<DT>(x + e + (long long)u * w.width);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float v[V];
      unpack<DT>(raw[u], v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = act<ACT>((v[j] - mean[j]) * a[j] + b[j], alpha);
      store_run<DT>(y + e + (long long)u * w.width, v);
    }
  }
  for (; e + V <= end; e += w.width) {
    float v[V];
    unpack<DT>(load_raw<DT>(x + e), v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = act<ACT>((v[j] - mean[j]) * a[j] + b[j], alpha);
    store_run<DT>(y + e, v);
  }
  if (e < end) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e + j < end) y[e + j] = from_f32<DT>(act<ACT>((to_f32<DT>(x[e + j]) - mean[j]) * a[j] + b[j], alpha));
  }
}

// ---- backward -----------------------------------------------------------------------

// du = dy act'(u) of one channel.  The leaky ReLU's slope changes where u crosses zero, and
// a u whose rounding has the wrong sign would be a whole slope off: so x is compared with
// the place of the crossing, mean - beta / (rstd gamma), computed in fp64 and rounded to
// the fp32 value below it (or the largest one below it, where u falls with x), after which
// a comparison of fp32 values decides exactly.
template <int ACT> struct Slope {
  float mean, a, b;
  __device__ __forceinline__ void set(float m, float rstd, float gamma, float beta, float) {
    mean = m;
    a = rstd * gamma;
    b = beta;
  }
  __device__ __forceinline__ float at(float x, float alpha) const { return act_slope<ACT>((x - mean) * a + b, alpha); }
};
template <> struct Slope<ACT_NONE> {
  __device__ __forceinline__ void set(float, float, float, float, float) {}
  __device__ __forceinline__ float at(float, float) const { return 1.f; }
};
template <> struct Slope<ACT_LRELU> {
  float edge, above, below;
  __device__ __forceinline__ void set(float m, float rstd, float gamma, float beta, float alpha) {
    const double a = (double)rstd * (double)gamma;
    if (a == 0.0 || !isfinite(a) || !isfinite(beta) || !isfinite(m)) {
      // u is beta, or NaN (which is not above zero) wherever x is finite
      edge = 0.f;
      above = below = (beta > 0.f && isfinite(a) && isfinite(m)) ? 1.f : alpha;
      return;
    }
    const double t = (double)m - (double)beta / a;
    float f = (float)t;  // to nearest
    const bool falls = a < 0.0;
    // u > 0 is x > t, or (falling) x < t
    if (falls ? (double)f >= t : (double)f > t) f = nextafterf(f, -INFINITY);
    edge = f;
    above = falls ? alpha : 1.f;
    below = falls ? 1.f : alpha;
  }
  __device__ __forceinline__ float at(float x, float) const { return x > edge ? above : below; }
};

// part[(sample, slice, row)][c] = (sum du, sum du (x - mean)) of each channel
template <int DT, int ACT>
__global__ __launch_bounds__(kThreads) void gn_bwd_sums_kernel(Walk w, const void *dy_, const void *x_, const float *gamma,
                                                               const float *beta, const float *mean_, const float *rstd_,
                                                               float alpha, float2 *part) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  __shared__ float2 red[kThreads * V];
  const int pb = blockIdx.x % w.parts, s = blockIdx.x / w.parts % w.slices;
  const long long n = blockIdx.x / w.parts / w.slices;
  const T *x = (const T *)x_ + n * w.count, *dy = (const T *)dy_ + n * w.count;
  const int tau = pb * kThreads + threadIdx.x;
  const bool live = tau < w.threads;
  float mean[V], s1[V], s2[V];
  Slope<ACT> slope[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (tau * V + j) % w.c;
    const long long g = n * w.groups + ch / w.per;
    mean[j] = mean_[g];
    slope[j].set(mean[j], rstd_[g], gamma[ch], beta[ch], alpha);
    s1[j] = s2[j] = 0.f;
  }
  const long long beg = (long long)s * w.turns * w.width;
  const long long end = min(beg + (long long)w.turns * w.width, w.count);
  long long e = beg + tau * V;
  auto add = [&](const u32x4_t &rx, const u32x4_t &rd) {
    float v[V], d[V];
    unpack<DT>(rx, v);
    unpack<DT>(rd, d);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float du = d[j] * slope[j].at(v[j], alpha);
      s1[j] += du;
      s2[j] += du * (v[j] - mean[j]);
    }
  };
  if (live) {
    for (; e + (long long)(kUnroll - 1) * w.width + V <= end; e += (long long)kUnroll * w.width) {
      u32x4_t rx[kUnroll], rd[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        rx[u] = load_raw<DT>(x + e + (long long)u * w.width);
        rd[u] = load_raw<DT>(dy + e + (long long)u * w.width);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) add(rx[u], rd[u]);
    }
    for (; e + V <= end; e += w.width) add(load_raw<DT>(x + e), load_raw<DT>(dy + e));
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (live && e + j < end) {
      const float v = to_f32<DT>(x[e + j]), du = to_f32<DT>(dy[e + j]) * slope[j].at(v, alpha);
      s1[j] += du;
      s2[j] += du * (v - mean[j]);
    }
    red[threadIdx.x * V + j] = make_float2(s1[j], s2[j]);
  }
  __syncthreads();
  float2 *out = part + ((n * w.slices + s) * w.prows) * w.c;
  if (w.prows > 1 || w.parts > 1) {
    for (int i = threadIdx.x; i < kThreads * V; i += kThreads) {
      const int f = pb * kThreads * V + i;
      if (f < w.width) out[f] = red[i];
    }
    return;
  }
  join_rows(w.rows, w.c, [&](int a, int b) {
    const float2 p = red[a], q = red[b];
    red[a] = make_float2(p.x + q.x, p.y + q.y);
  });
  for (int i = threadIdx.x; i < w.c; i += kThreads) out[i] = red[i];
}

// sums[n][c] = (sum du, sum du xh) of the partial rows; 16 channels a workgroup, 16 rows at
// a time
__global__ __launch_bounds__(kThreads) void gn_bwd_join_kernel(Walk w, const float2 *part, const float *rstd_, float2 *sums) {
  __shared__ float2 red[kThreads];
  const int tiles = (w.c + 15) / 16;
  const long long n = blockIdx.x / tiles;
  const int ch = blockIdx.x % tiles * 16 + (threadIdx.x & 15), ph = threadIdx.x >> 4;
  const int rows = w.slices * w.prows;
  float a = 0.f, b = 0.f;
  if (ch < w.c) {
    for (int r = ph; r < rows; r += 16) {
      const float2 p = part[(n * rows + r) * w.c + ch];
      a += p.x;
      b += p.y;
    }
  }
  red[threadIdx.x] = make_float2(a, b);
  __syncthreads();
  for (int h = 8; h > 0; h >>= 1) {
    if (ph < h) {
      const float2 p = red[threadIdx.x], q = red[threadIdx.x + 16 * h];
      red[threadIdx.x] = make_float2(p.x + q.x, p.y + q.y);
    }
    __syncthreads();
  }
  if (ph == 0 && ch < w.c) {
    const float2 p = red[threadIdx.x];
    sums[n * w.c + ch] = make_float2(p.x, p.y * rstd_[n * w.groups + ch / w.per]);
  }
}

// means over each group of gamma du and gamma du xh, [n][groups]; and dgamma, dbeta
__global__ __launch_bounds__(kThreads) void gn_bwd_groups_kernel(Walk w, int n, const float2 *sums, const float *gamma,
                                                                 float2 *means, float *dgamma, float *dbeta) {
  const long long groups = (long long)n * w.groups;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long gb = (groups + 3) / 4;  // workgroups of groups, a wave each
  if (blockIdx.x < gb) {
    const long long q = (long long)blockIdx.x * 4 + wave;
    if (q >= groups) return;
    const int g = (int)(q % w.groups);
    float a = 0.f, b = 0.f;
    for (int i = lane; i < w.per; i += 64) {
      const int ch = g * w.per + i;
      const float2 p = sums[q / w.groups * w.c + ch];
      a += p.x * gamma[ch];
      b += p.y * gamma[ch];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      a += __shfl_xor(a, o, 64);
      b += __shfl_xor(b, o, 64);
    }
    const float inv = 1.f / ((float)w.vox * (float)w.per);
    if (lane == 0) means[q] = make_float2(a * inv, b * inv);
    return;
  }
  const long long ch = (blockIdx.x - gb) * kThreads + threadIdx.x;
  if (ch >= w.c) return;
  float a = 0.f, b = 0.f;
  for (int i = 0; i < n; ++i) {
    const float2 p = sums[(long long)i * w.c + ch];
    a += p.x;
    b += p.y;
  }
  dbeta[ch] = a;
  dgamma[ch] = b;
}

template <int DT, int ACT>
__global__ __launch_bounds__(kThreads) void gn_bwd_apply_kernel(Walk w, const void *dy_, const void *x_, const float *gamma,
                                                                const float *beta, const float *mean_, const float *rstd_,
                                                                const float2 *means, float alpha, void *dx_) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  const int pb = blockIdx.x % w.parts, s = blockIdx.x / w.parts % w.slices;
  const long long n = blockIdx.x / w.parts / w.slices;
  const T *x = (const T *)x_ + n * w.count, *dy = (const T *)dy_ + n * w.count;
  T *dx = (T *)dx_ + n * w.count;
  const int tau = pb * kThreads + threadIdx.x;
  if (tau >= w.threads) return;
  // dx = (rstd gamma) du - rstd m1 - (x - mean) (rstd^2 m2)
  float mean[V], a[V], b[V], k[V];
  Slope<ACT> slope[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (tau * V + j) % w.c;
    const long long g = n * w.groups + ch / w.per;
    const float rstd = rstd_[g];
    const float2 m = means[g];
    mean[j] = mean_[g];
    slope[j].set(mean[j], rstd, gamma[ch], beta[ch], alpha);
    a[j] = rstd * gamma[ch];
    b[j] = rstd * m.x;
    k[j] = rstd * rstd * m.y;
  }
  const long long beg = (long long)s * w.turns * w.width;
  const long long end = min(beg + (long long)w.turns * w.width, w.count);
  long long e = beg + tau * V;
  auto one = [&](float v, float d, int j) {
    return a[j] * (d * slope[j].at(v, alpha)) - b[j] - (v - mean[j]) * k[j];
  };
  auto put = [&](const u32x4_t &rx, const u32x4_t &rd, T *o) {
    float v[V], d[V];
    unpack<DT>(rx, v);
    unpack<DT>(rd, d);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = one(v[j], d[j], j);
    store_run<DT>(o, v);
  };
  for (; e + (long long)(kUnroll - 1) * w.width + V <= end; e += (long long)kUnroll * w.width) {
    u32x4_t rx[kUnroll], rd[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      rx[u] = load_raw<DT>(x + e + (long long)u * w.width);
      rd[u] = load_raw<DT>(dy + e + (long long)u * w.width);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) put(rx[u], rd[u], dx + e + (long long)u * w.width);
  }
  for (; e + V <= end; e += w.width) put(load_raw<DT>(x + e), load_raw<DT>(dy + e), dx + e);
  if (e < end) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e + j < end) dx[e + j] = from_f32<DT>(one(to_f32<DT>(x[e + j]), to_f32<DT>(dy[e + j]), j));
  }
}

// ---- plan ---------------------------------------------------------------------------

constexpr int kTargetBlocks = 2048;  // eight workgroups of four waves a compute unit
constexpr int kMinTurns = 4;

Walk make_walk(int n, long long vox, int c, int groups, int dtype) {
  const int V = dtype == DT_BF16 ? 8 : 4;
  Walk w{};
  w.c = c;
  w.groups = groups;
  w.per = c / groups;
  w.vox = vox;
  w.count = vox * c;
  const int period = c / std::gcd(c, V);  // threads after which the channels repeat
  w.threads = period <= kThreads ? kThreads / period * period : period;
  w.parts = (w.threads + kThreads - 1) / kThreads;
  w.width = w.threads * V;
  w.rows = w.width / c;
  w.prows = w.parts > 1 ? w.rows : 1;
  const long long turns = (w.count + w.width - 1) / w.width;
  const long long want = std::max(1LL, kTargetBlocks / ((long long)n * w.parts));
  w.turns = (int)std::max<long long>(kMinTurns, (turns + want - 1) / want);
  w.slices = (int)((turns + w.turns - 1) / w.turns);
  return w;
}
long long rows_of(const Walk &w, int n) { return (long long)n * w.slices * w.prows; }
}  // namespace

size_t groupnorm_fwd_workspace(int n, long long vox, int c, int groups, int dtype) {
  const Walk w = make_walk(n, vox, c, groups, dtype);
  return (size_t)(rows_of(w, n) * c * 8 + 15) / 16 * 16;
}
size_t groupnorm_bwd_workspace(int n, long long vox, int c, int groups, int dtype) {
  const Walk w = make_walk(n, vox, c, groups, dtype);
  return (size_t)(((rows_of(w, n) + n) * c + (long long)n * groups) * 8 + 15) / 16 * 16;
}

hipError_t launch_groupnorm_fwd(int n, long long vox, int c, int groups, int dtype, const void *x, const float *gamma,
                                const float *beta, float eps, int act, float alpha, void *y, float *mean, float *rstd,
                                void *ws, hipStream_t st) {
  const Walk w = make_walk(n, vox, c, groups, dtype);
  const dim3 grid((unsigned)((long long)n * w.slices * w.parts)), block(kThreads);
  float2 *part = (float2 *)ws;
  auto run = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    hipLaunchKernelGGL((gn_stats_kernel<DT>), grid, block, 0, st, w, x, part);
    hipLaunchKernelGGL(gn_finish_stats_kernel, dim3((unsigned)(n * groups)), block, 0, st, w, eps, (const float2 *)part,
                       mean, rstd);
    with_act(act, [&](auto a) {
      hipLaunchKernelGGL((gn_apply_kernel<DT, decltype(a)::value>), grid, block, 0, st, w, x, gamma, beta,
                         (const float *)mean, (const float *)rstd, alpha, y);
    });
  };
  if (dtype == DT_BF16) run(std::integral_constant<int, DT_BF16>{});
  else run(std::integral_constant<int, DT_F32>{});
  return hipGetLastError();
}

hipError_t launch_groupnorm_bwd(int n, long long vox, int c, int groups, int dtype, const void *dy, const void *x,
                                const float *gamma, const float *beta, const float *mean, const float *rstd, int act,
                                float alpha, void *dx, float *dgamma, float *dbeta, void *ws, hipStream_t st) {
  const Walk w = make_walk(n, vox, c, groups, dtype);
  const dim3 grid((unsigned)((long long)n * w.slices * w.parts)), block(kThreads);
  float2 *part = (float2 *)ws, *sums = part + rows_of(w, n) * c, *means = sums + (long long)n * c;
  auto run = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    with_act(act, [&](auto a) {
      constexpr int ACT = decltype(a)::value;
      hipLaunchKernelGGL((gn_bwd_sums_kernel<DT, ACT>), grid, block, 0, st, w, dy, x, gamma, beta, mean, rstd, alpha, part);
      hipLaunchKernelGGL(gn_bwd_join_kernel, dim3((unsigned)((long long)n * ((c + 15) / 16))), block, 0, st, w,
                         (const float2 *)part, rstd, sums);
      hipLaunchKernelGGL(gn_bwd_groups_kernel, dim3((unsigned)(((long long)n * groups + 3) / 4 + (c + kThreads - 1) / kThreads)),
                         block, 0, st, w, n, (const float2 *)sums, gamma, means, dgamma, dbeta);
      hipLaunchKernelGGL((gn_bwd_apply_kernel<DT, ACT>), grid, block, 0, st, w, dy, x, gamma, beta, mean, rstd,
                         (const float2 *)means, alpha, dx);
    });
  };
  if (dtype == DT_BF16) run(std::integral_constant<int, DT_BF16>{});
  else run(std::integral_constant<int, DT_F32>{});
  return hipGetLastError();
}

}  // namespace cf
