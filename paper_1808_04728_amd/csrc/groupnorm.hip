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
// need no alignment.)  A sample is cut into slices; each leaves partial results, rows of a
// small matrix, which the workgroups of the second pass join in a fixed order before they
// read the data again and write.
//
// Bound by memory: the second pass reads again what the first one read.  It goes through the
// slices from the last to the first, so that it begins with what the last-level cache still
// has, and its own loads and stores pass that by.  (Taking some samples at a time, a launch
// with the second pass of some beside the first pass of the next, took longer: 128^3 batch
// 8 of 16 bf16 channels 350 us a sample at a time, and 328 in two launches then, where a launch's
// ends cost more than the cache gave.)  Groups of a few thousand values are one workgroup's,
// held in registers between the sums and the stores, in one launch.
//
// Measured: 128^3 batch 8 of 16 bf16 channels forward 268 us (1.61 GB at 6.0 TB/s: the sums 89,
// the second pass 178) and backward 475 (2.68 GB at 5.6 TB/s: 190 and 274), where a copy of
// 4 GiB makes 4.7 TB/s; 3 x 31^3 of 48 fp32 channels backward 22 (two launches of 11; 26
// with one more of 4 for dgamma and dbeta); 4^3 of 128 fp32 channels forward 6, 4 of them on the GPU.

#include <math.h>

#include <algorithm>
#include <numeric>

#include "activation.h"
#include "cf_common.h"
#include "cf_kernels.h"

namespace cf {
namespace {

constexpr int kThreads = 256;   // of a workgroup, where a voxel's channels repeat within them,
constexpr int kThreadsL = 1024;  // or else

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

// NT: past the last-level cache (see kStreamBytes)
template <int DT, bool NT = false> __device__ __forceinline__ u32x4_t load_raw(const typename Store<DT>::T *p) {
  const auto *q = reinterpret_cast<const typename Run<DT>::Vec *>(p);
  if constexpr (NT) return __builtin_nontemporal_load(q);
  else return *q;
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
template <int DT, bool NT> __device__ __forceinline__ void store_run(typename Store<DT>::T *p, const float (&f)[Run<DT>::V]) {
  u32x4_t a;
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = f2bf2(f[2 * i], f[2 * i + 1]);
  }
  auto *q = reinterpret_cast<typename Run<DT>::Vec *>(p);
  if constexpr (NT) __builtin_nontemporal_store((typename Run<DT>::Vec)a, q);
  else *q = a;
}

// How a sample is walked.  A turn is `width` = T V values = `rows` voxels; a slice is `turns`
// turns.  T threads are `parts` workgroups side by side.  The partial results of a slice are
// `prows` rows of `cols` values: one row of a value a group; or (`wide`: voxels of more values
// than a workgroup's turn) rows of a value a channel, one for every voxel of a turn.
struct Walk {
  int c, groups, per;  // channels, groups, channels a group
  long long vox, count;  // voxels and values of a sample
  int threads, parts, rows, width;
  int turns, slices, prows, cols;
  int wide, bt;  // bt: threads of a workgroup
  int join;      // the second pass's workgroups join the rows themselves
};

// values of channel ch that slice s has in partial row r
__device__ __forceinline__ int row_count(const Walk &w, int s, int r, int ch) {
  const long long beg = (long long)s * w.turns * w.width;
  const long long len = min((long long)w.turns * w.width, w.count - beg);
  if (w.prows == 1) return (int)(len / w.c);
  return (int)max(0LL, (len - (r * w.c + ch) + w.width - 1) / w.width);
}

// mean and sum of squared distances of na and nb values joined (d is multiplied by the weight
// first: joined to no values it is the mean itself, whose square may be infinite)
template <class T> __device__ __forceinline__ void join(T &mean, T &m2, T &na, T mb, T m2b, T nb) {
  const T n = na + nb;
  if (nb == (T)0) return;
  const T d = mb - mean, f = nb / n;
  mean += d * f;
  m2 += m2b + d * (d * (na * f));
  na = n;
}

// ---- sums over a slice --------------------------------------------------------------

// Rows of `width` values in LDS joined to one row of c values a tree; f(dst, src) joins two
// entries.  n: rows.
template <int BT, class F> __device__ __forceinline__ void join_rows(int n, int c, F f) {
  while (n > 1) {
    const int h = (n + 1) >> 1, todo = (n - h) * c;
    for (int i = threadIdx.x; i < todo; i += BT) f(i, i + h * c);
    n = h;
    __syncthreads();
  }
}

constexpr int kUnroll = 4;

// part[(sample, slice, row)][c] = (mean, sum of squared distances to it) of each channel
// (or, joined, of each group)
template <int DT, int BT>
__global__ __launch_bounds__(BT) void gn_stats_kernel(Walk w, const void *x_, float2 *part) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  __shared__ float2 red[BT * V];
  __shared__ float cnt[BT * V];
  const int pb = blockIdx.x % w.parts, s = blockIdx.x / w.parts % w.slices;
  const long long n = blockIdx.x / w.parts / w.slices;
  const T *x = (const T *)x_ + n * w.count;
  const int tau = pb * BT + threadIdx.x;
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
        m2[j] += q + d * (d * g);
      }
    }
    u32x4_t raw[kUnroll - 1];
#pragma unroll
    for (int u = 0; u < kUnroll - 1; ++u)
      if (e + (long long)u * w.width + V <= end) raw[u] = load_raw<DT>(x + e + (long long)u * w.width);
#pragma unroll
    for (int u = 0; u < kUnroll - 1; ++u) {
      if (e + V > end) break;
      float v[V];
      unpack<DT>(raw[u], v);
      na += 1.f;
      const float f = 1.f / na;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = v[j] - mean[j];
        mean[j] += d * f;
        m2[j] += d * (v[j] - mean[j]);
      }
      e += w.width;
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
  float2 *out = part + ((n * w.slices + s) * w.prows) * w.cols;
  if (w.wide) {
    for (int i = threadIdx.x; i < BT * V; i += BT) {
      const int f = pb * BT * V + i;
      if (f < w.width) out[f] = red[i];
    }
    return;
  }
  auto join2 = [&](int a, int b) {
    float2 p = red[a];
    const float2 q = red[b];
    float na = cnt[a];
    join<float>(p.x, p.y, na, q.x, q.y, cnt[b]);
    red[a] = p;
    cnt[a] = na;
  };
  join_rows<BT>(w.rows, w.c, join2);
  // the channels of each group, halving them
  for (int n = w.per; n > 1;) {
    const int h = (n + 1) >> 1, todo = (n - h) * w.groups;
    for (int i = threadIdx.x; i < todo; i += BT) {
      const int at = i / (n - h) * w.per + i % (n - h);
      join2(at, at + h);
    }
    n = h;
    __syncthreads();
  }
  for (int i = threadIdx.x; i < w.groups; i += BT) out[i] = red[i * w.per];
}

// wide: joined[n][c] of the partial rows; 16 channels a workgroup, 16 rows at a time
__global__ __launch_bounds__(kThreads) void gn_stats_join_kernel(Walk w, const float2 *part, float2 *joined) {
  __shared__ float red[3][kThreads];
  const int tiles = (w.c + 15) / 16;
  const long long n = blockIdx.x / tiles;
  const int ch = blockIdx.x % tiles * 16 + (threadIdx.x & 15), ph = threadIdx.x >> 4;
  const int rows = w.slices * w.prows;
  float mean = 0.f, m2 = 0.f, na = 0.f;
  if (ch < w.c) {
    for (int r = ph; r < rows; r += 16) {
      const float2 p = part[(n * rows + r) * w.c + ch];
      join<float>(mean, m2, na, p.x, p.y, (float)row_count(w, r / w.prows, r % w.prows, ch));
    }
  }
  red[0][threadIdx.x] = mean;
  red[1][threadIdx.x] = m2;
  red[2][threadIdx.x] = na;
  __syncthreads();
  for (int h = 8; h > 0; h >>= 1) {
    if (ph < h) {
      const int a = threadIdx.x, b = a + 16 * h;
      join<float>(red[0][a], red[1][a], red[2][a], red[0][b], red[1][b], red[2][b]);
    }
    __syncthreads();
  }
  if (ph == 0 && ch < w.c) joined[n * w.c + ch] = make_float2(red[0][threadIdx.x], red[1][threadIdx.x]);
}

// mean and rstd of each sample's group, a workgroup a group: from its slices' rows, or (wide)
// from its channels
__global__ __launch_bounds__(kThreads) void gn_finish_stats_kernel(Walk w, float eps, const float2 *part, float *mean_,
                                                                   float *rstd_) {
  __shared__ double red[3][kThreads];
  const int g = blockIdx.x % w.groups;
  const long long n = blockIdx.x / w.groups;
  double mean = 0.0, m2 = 0.0, na = 0.0;
  for (int i = threadIdx.x; i < (w.wide ? w.per : w.slices); i += kThreads) {
    const float2 p = w.wide ? part[n * w.c + g * w.per + i] : part[(n * w.slices + i) * w.groups + g];
    join<double>(mean, m2, na, p.x, p.y, w.wide ? (double)w.vox : (double)row_count(w, i, 0, 0) * w.per);
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

template <int BT> struct GroupLds {
  float a[BT], b[BT], n[BT];
};
// Rows that a workgroup of the second pass joins itself (sixteen a thread at most): lds.a[g],
// lds.b[g] = the result for each group, every group's rows by BT / groups threads,
// each its every so many-th row, which are joined in a tree
template <int BT, class Init, class Add, class Join>
__device__ __forceinline__ void join_groups(const Walk &w, GroupLds<BT> &lds, Init init, Add add, Join join2) {
  int phases = 1;
  while (2 * phases * w.groups <= BT) phases *= 2;
  const int g = threadIdx.x % w.groups, ph = threadIdx.x / w.groups;
  float a, b, n;
  init(a, b, n);
  if (ph < phases)
    for (int s = ph; s < w.slices; s += phases) add(a, b, n, s, g);
  lds.a[threadIdx.x] = a;
  lds.b[threadIdx.x] = b;
  lds.n[threadIdx.x] = n;
  __syncthreads();
  for (int h = phases / 2; h > 0; h >>= 1) {
    if (ph < h) join2(threadIdx.x, threadIdx.x + h * w.groups);
    __syncthreads();
  }
}

// ---- the second pass, forward -------------------------------------------------------

template <int DT, int BT, int ACT, bool NT>
__global__ __launch_bounds__(BT) void gn_apply_kernel(Walk w, const void *x_, const float *gamma, const float *beta,
                                                            float eps, const float2 *part, float *mean_, float *rstd_,
                                                            float alpha, void *y_) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  __shared__ GroupLds<BT> lds;
  const unsigned block = gridDim.x - 1 - blockIdx.x;
  const int pb = block % w.parts, s = block / w.parts % w.slices;
  const long long n = block / w.parts / w.slices;
  if (w.join) {
    join_groups(
        w, lds, [](float &a, float &b, float &k) { a = b = k = 0.f; },
        [&](float &a, float &b, float &k, int r, int g) {
          const float2 p = part[(n * w.slices + r) * w.cols + g];
          join<float>(a, b, k, p.x, p.y, (float)row_count(w, r, 0, 0) * w.per);
        },
        [&](int i, int j) { join<float>(lds.a[i], lds.b[i], lds.n[i], lds.a[j], lds.b[j], lds.n[j]); });
    if ((int)threadIdx.x < w.groups) {
      const float rstd = 1.f / sqrtf(lds.b[threadIdx.x] / lds.n[threadIdx.x] + eps);
      lds.b[threadIdx.x] = rstd;
      if (s == 0) {
        mean_[n * w.groups + threadIdx.x] = lds.a[threadIdx.x];
        rstd_[n * w.groups + threadIdx.x] = rstd;
      }
    }
    __syncthreads();
  }
  const T *x = (const T *)x_ + n * w.count;
  T *y = (T *)y_ + n * w.count;
  const int tau = pb * BT + threadIdx.x;
  if (tau >= w.threads) return;
  float mean[V], a[V], b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (tau * V + j) % w.c, q = ch / w.per;
    const long long g = n * w.groups + q;
    mean[j] = w.join ? lds.a[q] : mean_[g];
    a[j] = (w.join ? lds.b[q] : rstd_[g]) * gamma[ch];
    b[j] = beta[ch];
  }
  const long long beg = (long long)s * w.turns * w.width;
  const long long end = min(beg + (long long)w.turns * w.width, w.count);
  long long e = beg + tau * V;
  for (; e + (long long)(kUnroll - 1) * w.width + V <= end; e += (long long)kUnroll * w.width) {
    u32x4_t raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u] = load_raw<DT, NT>(x + e + (long long)u * w.width);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float v[V];
      unpack<DT>(raw[u], v);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = act<ACT>((v[j] - mean[j]) * a[j] + b[j], alpha);
      store_run<DT, NT>(y + e + (long long)u * w.width, v);
    }
  }
  u32x4_t raw[kUnroll - 1];
#pragma unroll
  for (int u = 0; u < kUnroll - 1; ++u)
    if (e + (long long)u * w.width + V <= end) raw[u] = load_raw<DT, NT>(x + e + (long long)u * w.width);
#pragma unroll
  for (int u = 0; u < kUnroll - 1; ++u) {
    if (e + V > end) break;
    float v[V];
    unpack<DT>(raw[u], v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = act<ACT>((v[j] - mean[j]) * a[j] + b[j], alpha);
    store_run<DT, NT>(y + e, v);
    e += w.width;
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

// wide: part[(sample, slice, row)][c] = (sum du, sum du (x - mean)) of each channel.  Otherwise
// db and dg [(sample, slice)][c] = sum du and sum du xh, and part[(sample, slice)][groups] = the
// sums of gamma du and gamma du xh.
template <int DT, int BT, int ACT>
__global__ __launch_bounds__(BT) void gn_bwd_sums_kernel(Walk w, const void *dy_, const void *x_, const float *gamma,
                                                               const float *beta, const float *mean_, const float *rstd_,
                                                               float alpha, float2 *part, float *db, float *dg) {
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  __shared__ float2 red[BT * V];
  const int pb = blockIdx.x % w.parts, s = blockIdx.x / w.parts % w.slices;
  const long long n = blockIdx.x / w.parts / w.slices;
  const T *x = (const T *)x_ + n * w.count, *dy = (const T *)dy_ + n * w.count;
  const int tau = pb * BT + threadIdx.x;
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
    u32x4_t rx[kUnroll - 1], rd[kUnroll - 1];
#pragma unroll
    for (int u = 0; u < kUnroll - 1; ++u)
      if (e + (long long)u * w.width + V <= end) {
        rx[u] = load_raw<DT>(x + e + (long long)u * w.width);
        rd[u] = load_raw<DT>(dy + e + (long long)u * w.width);
      }
#pragma unroll
    for (int u = 0; u < kUnroll - 1; ++u) {
      if (e + V > end) break;
      add(rx[u], rd[u]);
      e += w.width;
    }
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
  float2 *out = part + ((n * w.slices + s) * w.prows) * w.cols;
  if (w.wide) {
    for (int i = threadIdx.x; i < BT * V; i += BT) {
      const int f = pb * BT * V + i;
      if (f < w.width) out[f] = red[i];
    }
    return;
  }
  join_rows<BT>(w.rows, w.c, [&](int a, int b) {
    const float2 p = red[a], q = red[b];
    red[a] = make_float2(p.x + q.x, p.y + q.y);
  });
  const long long row = (n * w.slices + s) * w.c;
  for (int i = threadIdx.x; i < w.c; i += BT) {
    const float2 p = red[i];
    const float b = p.x, g = p.y * rstd_[n * w.groups + i / w.per];
    db[row + i] = b;
    dg[row + i] = g;
    red[i] = make_float2(b * gamma[i], g * gamma[i]);
  }
  __syncthreads();
  for (int n = w.per; n > 1;) {  // the channels of each group, halving them
    const int h = (n + 1) >> 1, todo = (n - h) * w.groups;
    for (int i = threadIdx.x; i < todo; i += BT) {
      const int at = i / (n - h) * w.per + i % (n - h);
      const float2 p = red[at], q = red[at + h];
      red[at] = make_float2(p.x + q.x, p.y + q.y);
    }
    n = h;
    __syncthreads();
  }
  for (int i = threadIdx.x; i < w.groups; i += BT) out[i] = red[i * w.per];
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

// means[n][groups] of the slices' sums part[(sample, slice)][groups], a wave a group
__global__ __launch_bounds__(kThreads) void gn_bwd_means_kernel(Walk w, long long groups, const float2 *part, float2 *means) {
  const long long q = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (q >= groups) return;
  const long long n = q / w.groups;
  float a = 0.f, b = 0.f;
  for (int s = lane; s < w.slices; s += 64) {
    const float2 p = part[(n * w.slices + s) * w.cols + q % w.groups];
    a += p.x;
    b += p.y;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    a += __shfl_xor(a, o, 64);
    b += __shfl_xor(b, o, 64);
  }
  const float inv = 1.f / ((float)w.vox * (float)w.per);
  if (lane == 0) means[q] = make_float2(a * inv, b * inv);
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

// dbeta and dgamma from rows [rows][c] of partial sums: workgroups in front of a launch of the
// second pass, each of 16 columns of one of the two.
struct Columns {
  int count;  // workgroups
  int rows;
  const float *db, *dg;
  float *dbeta, *dgamma;
};
constexpr int kColumnRows = 1024;  // (more take a launch of their own, of more workgroups)
template <int BT> __device__ __forceinline__ void sum_columns(const Columns &q, int c, int block) {
  __shared__ float red[BT];
  const int half = q.count / 2, ch = block % half * 16 + threadIdx.x % 16, lane = threadIdx.x / 16;
  constexpr int LANES = BT / 16, U = 8;
  const float *part = block < half ? q.db : q.dg;
  float s = 0.f;
  if (ch < c) {
    for (int r = lane; r < q.rows; r += LANES * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = r + u * LANES < q.rows ? part[(long long)(r + u * LANES) * c + ch] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];
    }
  }
  red[threadIdx.x] = s;
  __syncthreads();
  for (int k = LANES / 2; k > 0; k /= 2) {
    if (lane < k) red[threadIdx.x] += red[threadIdx.x + k * 16];
    __syncthreads();
  }
  if (lane == 0 && ch < c) (block < half ? q.dbeta : q.dgamma)[ch] = red[threadIdx.x];
}

// means: of every group, or (w.join) the slices' sums that the workgroup joins itself
template <int DT, int BT, int ACT, bool NT>
__global__ __launch_bounds__(BT) void gn_bwd_apply_kernel(Walk w, const void *dy_, const void *x_, const float *gamma,
                                                                const float *beta, const float *mean_, const float *rstd_,
                                                                const float2 *means, float alpha, void *dx_, Columns columns) {
  if ((int)blockIdx.x < columns.count) return sum_columns<BT>(columns, w.c, blockIdx.x);
  constexpr int V = Run<DT>::V;
  typedef typename Store<DT>::T T;
  __shared__ GroupLds<BT> lds;
  const unsigned block = gridDim.x - 1 - blockIdx.x;
  const int pb = block % w.parts, s = block / w.parts % w.slices;
  const long long n = block / w.parts / w.slices;
  if (w.join) {
    join_groups(
        w, lds, [](float &a, float &b, float &) { a = b = 0.f; },
        [&](float &a, float &b, float &, int r, int g) {
          const float2 p = means[(n * w.slices + r) * w.cols + g];
          a += p.x;
          b += p.y;
        },
        [&](int i, int j) {
          lds.a[i] += lds.a[j];
          lds.b[i] += lds.b[j];
        });
  }
  const float inv = w.join ? 1.f / ((float)w.vox * (float)w.per) : 1.f;
  const T *x = (const T *)x_ + n * w.count, *dy = (const T *)dy_ + n * w.count;
  T *dx = (T *)dx_ + n * w.count;
  const int tau = pb * BT + threadIdx.x;
  if (tau >= w.threads) return;
  // dx = (rstd gamma) du - rstd m1 - (x - mean) (rstd^2 m2)
  float mean[V], a[V], b[V], k[V];
  Slope<ACT> slope[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int ch = (tau * V + j) % w.c, q = ch / w.per;
    const long long g = n * w.groups + q;
    const float rstd = rstd_[g];
    const float2 m = w.join ? make_float2(lds.a[q] * inv, lds.b[q] * inv) : means[g];
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
    store_run<DT, NT>(o, v);
  };
  for (; e + (long long)(kUnroll - 1) * w.width + V <= end; e += (long long)kUnroll * w.width) {
    u32x4_t rx[kUnroll], rd[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      rx[u] = load_raw<DT, NT>(x + e + (long long)u * w.width);
      rd[u] = load_raw<DT, NT>(dy + e + (long long)u * w.width);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) put(rx[u], rd[u], dx + e + (long long)u * w.width);
  }
  u32x4_t rx[kUnroll - 1], rd[kUnroll - 1];
#pragma unroll
  for (int u = 0; u < kUnroll - 1; ++u)
    if (e + (long long)u * w.width + V <= end) {
      rx[u] = load_raw<DT, NT>(x + e + (long long)u * w.width);
      rd[u] = load_raw<DT, NT>(dy + e + (long long)u * w.width);
    }
#pragma unroll
  for (int u = 0; u < kUnroll - 1; ++u) {
    if (e + V > end) break;
    put(rx[u], rd[u], dx + e);
    e += w.width;
  }
  if (e < end) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (e + j < end) dx[e + j] = from_f32<DT>(one(to_f32<DT>(x[e + j]), to_f32<DT>(dy[e + j]), j));
  }
}

// ---- a group a workgroup --------------------------------------------------------------

// A group's `vox` rows of `per` values, `line` pieces of V values each; T threads, a multiple of
// line, so that a thread's pieces have the same channels; a thread's piece in turn u is of row
// tid / line + u T / line.  At most kPieces turns.
template <int BT> constexpr int kPieces = BT == kThreads ? 8 : 4;  // (1024 threads have 128 registers)
struct Small {
  int c, groups, per, vox;
  int line, threads, step;  // step: T / line
};

// one value or 16 bytes
template <int DT, int V> struct Piece {
  typedef u32x4_t Raw;
  static __device__ __forceinline__ Raw load(const typename Store<DT>::T *p) { return load_raw<DT>(p); }
  static __device__ __forceinline__ void get(const Raw &r, float (&f)[V]) { unpack<DT>(r, f); }
  static __device__ __forceinline__ void put(typename Store<DT>::T *p, const float (&f)[V]) { store_run<DT, false>(p, f); }
};
template <int DT> struct Piece<DT, 1> {
  typedef typename Store<DT>::T Raw;
  static __device__ __forceinline__ Raw load(const Raw *p) { return *p; }
  static __device__ __forceinline__ void get(const Raw &r, float (&f)[1]) { f[0] = to_f32<DT>(r); }
  static __device__ __forceinline__ void put(Raw *p, const float (&f)[1]) { *p = from_f32<DT>(f[0]); }
};

// the sum over the workgroup, in every thread (red: a value a wave, free again at the next barrier)
template <int BT> __device__ __forceinline__ float block_sum(float x, float *red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = red[0];
#pragma unroll
  for (int i = 1; i < BT / 64; ++i) s += red[i];
  return s;
}

template <int DT, int V, int BT, int ACT>
__global__ __launch_bounds__(BT) void gn_small_fwd_kernel(Small q, const void *x_, const float *gamma, const float *beta,
                                                          float eps, float alpha, void *y_, float *mean_, float *rstd_) {
  typedef Piece<DT, V> P;
  typedef typename Store<DT>::T T;
  __shared__ float red[2][BT / 64];
  const int g = blockIdx.x % q.groups, row = threadIdx.x / q.line, ch = g * q.per + threadIdx.x % q.line * V;
  const long long at = (long long)(blockIdx.x / q.groups) * q.vox * q.c + ch;
  const T *x = (const T *)x_ + at;
  T *y = (T *)y_ + at;
  const bool live = (int)threadIdx.x < q.threads;
  auto has = [&](int u) { return live && row + u * q.step < q.vox; };
  auto place = [&](int u) { return (long long)(row + u * q.step) * q.c; };
  typename P::Raw raw[kPieces<BT>];
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u)
    if (has(u)) raw[u] = P::load(x + place(u));
  float ga[V], be[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    ga[j] = live ? gamma[ch + j] : 0.f;
    be[j] = live ? beta[ch + j] : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u) {
    if (!has(u)) continue;
    float v[V];
    P::get(raw[u], v);
#pragma unroll
    for (int j = 0; j < V; ++j) s += v[j];
  }
  const float inv = 1.f / ((float)q.vox * (float)q.per);
  const float mean = block_sum<BT>(s, red[0]) * inv;
  s = 0.f;
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u) {
    if (!has(u)) continue;
    float v[V];
    P::get(raw[u], v);
#pragma unroll
    for (int j = 0; j < V; ++j) s += (v[j] - mean) * (v[j] - mean);
  }
  const float rstd = 1.f / sqrtf(block_sum<BT>(s, red[1]) * inv + eps);
  if (threadIdx.x == 0) {
    mean_[blockIdx.x] = mean;
    rstd_[blockIdx.x] = rstd;
  }
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u) {
    if (!has(u)) continue;
    float v[V];
    P::get(raw[u], v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = act<ACT>((v[j] - mean) * (rstd * ga[j]) + be[j], alpha);
    P::put(y + place(u), v);
  }
}

// db, dg [n][c]: each sample's sums du and du xh
template <int DT, int V, int BT, int ACT>
__global__ __launch_bounds__(BT) void gn_small_bwd_kernel(Small q, const void *dy_, const void *x_, const float *gamma,
                                                          const float *beta, const float *mean_, const float *rstd_, float alpha,
                                                          void *dx_, float *db, float *dg) {
  typedef Piece<DT, V> P;
  typedef typename Store<DT>::T T;
  __shared__ float2 red[BT * V];
  __shared__ float sum[2][BT / 64];
  const int g = blockIdx.x % q.groups, row = threadIdx.x / q.line, ch = g * q.per + threadIdx.x % q.line * V;
  const long long n = blockIdx.x / q.groups, at = n * q.vox * q.c + ch;
  const T *x = (const T *)x_ + at, *dy = (const T *)dy_ + at;
  T *dx = (T *)dx_ + at;
  const bool live = (int)threadIdx.x < q.threads;
  auto has = [&](int u) { return live && row + u * q.step < q.vox; };
  auto place = [&](int u) { return (long long)(row + u * q.step) * q.c; };
  typename P::Raw rx[kPieces<BT>], rd[kPieces<BT>];
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u)
    if (has(u)) {
      rx[u] = P::load(x + place(u));
      rd[u] = P::load(dy + place(u));
    }
  const float mean = mean_[blockIdx.x], rstd = rstd_[blockIdx.x];
  float ga[V], s1[V], s2[V];
  Slope<ACT> slope[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    ga[j] = live ? gamma[ch + j] : 0.f;
    slope[j].set(mean, rstd, ga[j], live ? beta[ch + j] : 0.f, alpha);
    s1[j] = s2[j] = 0.f;
  }
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u) {
    if (!has(u)) continue;
    float v[V], d[V];
    P::get(rx[u], v);
    P::get(rd[u], d);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float du = d[j] * slope[j].at(v[j], alpha);
      s1[j] += du;
      s2[j] += du * (v[j] - mean);
    }
  }
  float m1 = 0.f, m2 = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s2[j] *= rstd;
    if (live) red[threadIdx.x * V + j] = make_float2(s1[j], s2[j]);
    m1 += ga[j] * s1[j];
    m2 += ga[j] * s2[j];
  }
  const float inv = 1.f / ((float)q.vox * (float)q.per);
  m1 = block_sum<BT>(m1, sum[0]) * inv;  // (its barrier is also red's)
  m2 = block_sum<BT>(m2, sum[1]) * inv;
#pragma unroll
  for (int u = 0; u < kPieces<BT>; ++u) {
    if (!has(u)) continue;
    float v[V], d[V];
    P::get(rx[u], v);
    P::get(rd[u], d);
#pragma unroll
    for (int j = 0; j < V; ++j)
      v[j] = rstd * ga[j] * (d[j] * slope[j].at(v[j], alpha)) - rstd * m1 - (v[j] - mean) * (rstd * rstd * m2);
    P::put(dx + place(u), v);
  }
  join_rows<BT>(q.step, q.per, [&](int a, int b) {
    const float2 p = red[a], r = red[b];
    red[a] = make_float2(p.x + r.x, p.y + r.y);
  });
  for (int i = threadIdx.x; i < q.per; i += BT) {
    db[n * q.c + g * q.per + i] = red[i].x;
    dg[n * q.c + g * q.per + i] = red[i].y;
  }
}

// ---- plan ---------------------------------------------------------------------------

// Workgroups of a pass: eight waves a compute unit, which the tensors of 128^3 batch 8 fill the
// memory with as well as sixteen or thirty-two do, and the fewer rows there are to join (3 x
// 31^3 of 48 channels: 18.6, 20.4 and 21.5 us forward).
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
  w.bt = period <= kThreads ? kThreads : kThreadsL;
  w.threads = period <= w.bt ? w.bt / period * period : period;
  w.parts = (w.threads + w.bt - 1) / w.bt;
  w.width = w.threads * V;
  w.rows = w.width / c;
  w.wide = w.parts > 1;
  w.prows = w.wide ? w.rows : 1;
  w.cols = w.wide ? c : groups;
  const long long turns = (w.count + w.width - 1) / w.width;
  const long long want = std::max(1LL, (w.bt == kThreads ? 512 : 256) / ((long long)n * w.parts));
  w.turns = (int)std::max<long long>(kMinTurns, (turns + want - 1) / want);
  w.slices = (int)((turns + w.turns - 1) / w.turns);
  w.join = !w.wide && groups <= w.bt && (long long)w.slices * groups <= 16 * w.bt;
  return w;
}

// A group a workgroup: where its rows are kPieces pieces a thread of 256 threads at most, or of
// 1024 and there are many groups of rows of 64 bytes (the lines of shorter ones would be
// read by several XCDs: 16 x 16^3 x 128 bf16 in groups of 8).  Threads of the workgroup, or 0.
int small_plan(int n, long long vox, int c, int groups, int dtype, Small *q, int *values) {
  const int per = c / groups, vec = dtype == DT_BF16 ? 8 : 4;
  const int V = per % vec == 0 && c % vec == 0 ? vec : 1, line = per / V;
  *values = V;
  for (int bt : {kThreads, kThreadsL}) {
    if (line > bt || (bt > kThreads && ((long long)n * groups < 128 || per * (16 / vec) < 64))) continue;
    const int step = bt / line;
    if (vox > (long long)step * (bt == kThreads ? kPieces<kThreads> : kPieces<kThreadsL>)) continue;
    *q = Small{c, groups, per, (int)vox, line, step * line, step};
    return bt;
  }
  return 0;
}

long long rows_of(const Walk &w, int n) { return (long long)n * w.slices * w.prows; }
size_t up16(long long bytes) { return (size_t)(bytes + 15) / 16 * 16; }

// the backward pass's workspace: rows, the channels' sums, and what they are joined to
struct BwdSpace {
  size_t part, db, dg, sums, means, end;
  BwdSpace(const Walk &w, int n) {
    part = 0;
    db = part + up16(rows_of(w, n) * w.cols * 8);
    dg = db + (w.wide ? 0 : up16(rows_of(w, n) * w.c * 4));
    sums = dg + (w.wide ? 0 : up16(rows_of(w, n) * w.c * 4));
    means = sums + (w.wide ? up16((long long)n * w.c * 8) : 0);
    end = means + (w.join ? 0 : up16((long long)n * w.groups * 8));
  }
};

}  // namespace

size_t groupnorm_fwd_workspace(int n, long long vox, int c, int groups, int dtype) {
  Small q;
  int values;
  if (small_plan(n, vox, c, groups, dtype, &q, &values)) return 0;
  const Walk w = make_walk(n, vox, c, groups, dtype);
  return up16(rows_of(w, n) * w.cols * 8) + (w.wide ? up16((long long)n * c * 8) : 0);
}
size_t groupnorm_bwd_workspace(int n, long long vox, int c, int groups, int dtype) {
  Small q;
  int values;
  if (small_plan(n, vox, c, groups, dtype, &q, &values)) return n > 1 ? 2 * up16((long long)n * c * 4) : 0;
  return BwdSpace(make_walk(n, vox, c, groups, dtype), n).end;
}

namespace {
// f(std::integral_constant of the type, of a piece's values, of a workgroup's threads)
template <class F> void with_small(int dtype, int values, int bt, F f) {
  auto threads = [&](auto dt, auto v) {
    bt == kThreads ? f(dt, v, std::integral_constant<int, kThreads>{}) : f(dt, v, std::integral_constant<int, kThreadsL>{});
  };
  auto piece = [&](auto dt) {
    values == 1 ? threads(dt, std::integral_constant<int, 1>{})
                : threads(dt, std::integral_constant<int, Run<decltype(dt)::value>::V>{});
  };
  dtype == DT_BF16 ? piece(std::integral_constant<int, DT_BF16>{}) : piece(std::integral_constant<int, DT_F32>{});
}

// f(std::integral_constant of the type, of a workgroup's threads)
template <class F> void with_walk(int dtype, const Walk &w, F f) {
  auto type = [&](auto dt) {
    w.bt == kThreads ? f(dt, std::integral_constant<int, kThreads>{}) : f(dt, std::integral_constant<int, kThreadsL>{});
  };
  dtype == DT_BF16 ? type(std::integral_constant<int, DT_BF16>{}) : type(std::integral_constant<int, DT_F32>{});
}
}  // namespace

hipError_t launch_groupnorm_fwd(int n, long long vox, int c, int groups, int dtype, const void *x, const float *gamma,
                                const float *beta, float eps, int act, float alpha, void *y, float *mean, float *rstd,
                                void *ws, hipStream_t st) {
  Small q;
  int values;
  if (const int bt = small_plan(n, vox, c, groups, dtype, &q, &values)) {
    with_small(dtype, values, bt, [&](auto dt, auto v, auto t) {
      with_act(act, [&](auto a) {
        hipLaunchKernelGGL((gn_small_fwd_kernel<decltype(dt)::value, decltype(v)::value, decltype(t)::value, decltype(a)::value>),
                           dim3((unsigned)(n * groups)), dim3(bt), 0, st, q, x, gamma, beta, eps, alpha, y, mean, rstd);
      });
    });
    return hipGetLastError();
  }
  const Walk w = make_walk(n, vox, c, groups, dtype);
  const dim3 grid((unsigned)((long long)n * w.slices * w.parts)), block(w.bt);
  const bool stream = n * w.count * (dtype == DT_BF16 ? 2 : 4) >= kStreamBytes;
  float2 *part = (float2 *)ws, *joined = (float2 *)((char *)ws + up16(rows_of(w, n) * w.cols * 8));
  with_walk(dtype, w, [&](auto dt, auto bt) {
    constexpr int DT = decltype(dt)::value, BT = decltype(bt)::value;
    hipLaunchKernelGGL((gn_stats_kernel<DT, BT>), grid, block, 0, st, w, x, part);
    if (w.wide)
      hipLaunchKernelGGL(gn_stats_join_kernel, dim3((unsigned)((long long)n * ((c + 15) / 16))), dim3(kThreads), 0, st, w,
                         (const float2 *)part, joined);
    if (!w.join)
      hipLaunchKernelGGL(gn_finish_stats_kernel, dim3((unsigned)(n * groups)), dim3(kThreads), 0, st, w, eps,
                         (const float2 *)(w.wide ? joined : part), mean, rstd);
    with_act(act, [&](auto a) {
      constexpr int ACT = decltype(a)::value;
      auto apply = [&](auto nt) {
        hipLaunchKernelGGL((gn_apply_kernel<DT, BT, ACT, decltype(nt)::value>), grid, block, 0, st, w, x, gamma, beta, eps,
                           (const float2 *)part, mean, rstd, alpha, y);
      };
      stream ? apply(std::true_type{}) : apply(std::false_type{});
    });
  });
  return hipGetLastError();
}

hipError_t launch_groupnorm_bwd(int n, long long vox, int c, int groups, int dtype, const void *dy, const void *x,
                                const float *gamma, const float *beta, const float *mean, const float *rstd, int act,
                                float alpha, void *dx, float *dgamma, float *dbeta, void *ws, hipStream_t st) {
  Small q;
  int values;
  if (const int bt = small_plan(n, vox, c, groups, dtype, &q, &values)) {
    float *sb = n > 1 ? (float *)ws : dbeta, *sg = n > 1 ? (float *)((char *)ws + up16((long long)n * c * 4)) : dgamma;
    with_small(dtype, values, bt, [&](auto dt, auto v, auto t) {
      with_act(act, [&](auto a) {
        hipLaunchKernelGGL((gn_small_bwd_kernel<decltype(dt)::value, decltype(v)::value, decltype(t)::value, decltype(a)::value>),
                           dim3((unsigned)(n * groups)), dim3(bt), 0, st, q, dy, x, gamma, beta, mean, rstd, alpha, dx, sb, sg);
      });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == 1) return e;
    const SumJob jobs[2] = {{sb, dbeta, n, c}, {sg, dgamma, n, c}};
    return launch_sum_batch(jobs, 2, st);
  }
  const Walk w = make_walk(n, vox, c, groups, dtype);
  const dim3 grid((unsigned)((long long)n * w.slices * w.parts)), block(w.bt), small(kThreads);
  const bool stream = n * w.count * (dtype == DT_BF16 ? 2 : 4) >= kStreamBytes;
  const BwdSpace at(w, n);
  char *base = (char *)ws;
  float2 *part = (float2 *)(base + at.part), *sums = (float2 *)(base + at.sums), *means = (float2 *)(base + at.means);
  float *db = (float *)(base + at.db), *dg = (float *)(base + at.dg);
  const dim3 waves((unsigned)(((long long)n * groups + 3) / 4));
  const bool here = !w.wide && rows_of(w, n) <= kColumnRows;
  const Columns columns{here ? (c + 15) / 16 * 2 : 0, (int)rows_of(w, n), db, dg, dbeta, dgamma};
  with_walk(dtype, w, [&](auto dt, auto bt) {
    constexpr int DT = decltype(dt)::value, BT = decltype(bt)::value;
    with_act(act, [&](auto a) {
      constexpr int ACT = decltype(a)::value;
      hipLaunchKernelGGL((gn_bwd_sums_kernel<DT, BT, ACT>), grid, block, 0, st, w, dy, x, gamma, beta, mean, rstd, alpha, part,
                         db, dg);
      if (w.wide) {
        hipLaunchKernelGGL(gn_bwd_join_kernel, dim3((unsigned)((long long)n * ((c + 15) / 16))), small, 0, st, w,
                           (const float2 *)part, rstd, sums);
        hipLaunchKernelGGL(gn_bwd_groups_kernel, dim3(waves.x + (c + kThreads - 1) / kThreads), small, 0, st, w, n,
                           (const float2 *)sums, gamma, means, dgamma, dbeta);
      } else if (!w.join) {
        hipLaunchKernelGGL(gn_bwd_means_kernel, waves, small, 0, st, w, (long long)n * groups, (const float2 *)part, means);
      }
      auto apply = [&](auto nt) {
        hipLaunchKernelGGL((gn_bwd_apply_kernel<DT, BT, ACT, decltype(nt)::value>), dim3(grid.x + columns.count), block, 0, st, w,
                           dy, x, gamma, beta, mean, rstd, (const float2 *)(w.join ? part : means), alpha, dx, columns);
      };
      stream ? apply(std::true_type{}) : apply(std::false_type{});
    });
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || w.wide || here) return e;
  const SumJob jobs[2] = {{db, dbeta, (int)rows_of(w, n), c}, {dg, dgamma, (int)rows_of(w, n), c}};
  return launch_sum_batch(jobs, 2, st);
}

}  // namespace cf
