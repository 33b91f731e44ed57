// muon.hip -- orthogonalised updates of weight matrices: Newton-Schulz products
// on the matrix cores, and the momentum step around them.
//
// With X the matrix of a group, its shorter side m first, one step is
//   H = X X',  Q = a I + b H + c H^2,  X <- Q X,
// and since Q commutes with H the next step's H is Q H Q.  Two steps are taken on
// the m x m side before X is touched again (P = Q1 Q0, X <- P X, H from X anew):
// per pair of steps 3 m^2 n + 5 m^3 operations instead of 6 m^2 n + 2 m^3, and as
// exact as stepping X itself; a third step without a new H would square the
// rounding of H into the small singular values.
//
// Products are fp32 to within their last bits on half-precision matrix cores
// (16 times the fp32 rate): each factor is the sum of two fp16 values, x = hi + lo,
// scaled by a power of two so that hi stays in fp16's range (the bounds follow from
// the polynomial, |x_ij| <= ||X||_2) and lo above its smallest step; a product is
// hi hi + hi lo + lo hi in fp32 accumulators, what is left out is 2^-24 of it.
//
// All groups of a call share their launches: a workgroup finds its matrix in the
// table of its launch.

#include <math.h>

#include <type_traits>

#include "muon_common.h"

namespace cf {
namespace {

constexpr int kTile = 64;
constexpr int kStep = 32;  // k of one matrix instruction; both sides are padded to it

// ---- momentum and norm --------------------------------------------------------

// Chunks of kNsChunk << shift elements: with momentum, m <- mu m + (1 - mu) g and the
// update u = (1 - mu) g + mu m (or m) into the group's workspace; the sum of squares
// of u (of g without momentum) in fp64.
template <int DT, bool MOM>
__global__ __launch_bounds__(256) void ns_prep_kernel(NsTable T, NsMomentum mom, const void *g, float *m, char *ws) {
  __shared__ double red[4];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const long long count = (long long)M.m * M.n, span = (long long)kNsChunk << M.shift;
  const int chunk = blockIdx.x - T.first[l];
  const long long beg = chunk * span, end = min(beg + span, count);
  float *u = (float *)(ws + M.ws_u);
  double s = 0.0;
  for (long long e = beg + 4LL * threadIdx.x; e < end; e += 4LL * 256) {
    float x[4];
    const int k = (int)min(4LL, end - e);
    if (DT == DT_F32 && k == 4) {
      const float4 a = *reinterpret_cast<const float4 *>((const float *)g + M.off + e);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = i < k ? to_f32<DT>(((const typename Store<DT>::T *)g)[M.off + e + i]) : 0.f;
    }
    if constexpr (MOM) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < k) {
          x[i] = ns_momentum(mom, x[i], m[M.off + e + i]);
          u[e + i] = x[i];
        }
      }
    }
    s += (double)x[0] * x[0] + (double)x[1] * x[1] + (double)x[2] * x[2] + (double)x[3] * x[3];
  }
  s = ns_block_sum(s, red);
  if (threadIdx.x == 0) ((double *)(ws + M.ws_norm))[chunk] = s;
}

// X = u / (||u|| + eps) in both layouts, xn [mp][np] and xt [np][mp] (hi and lo, zero
// padding), by 64 x 64 tiles of the long side by the short one
template <int DT>
__global__ __launch_bounds__(256) void ns_split_kernel(NsTable T, double eps, float scale, const void *src, char *ws) {
  __shared__ double red[4];
  __shared__ float tile[64][65];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const double inv = ns_inv_norm(M, ws, eps, red);
  const int tm = (M.mp + 63) / 64, b = blockIdx.x - T.first[l];
  const int n0 = b / tm * 64, m0 = b % tm * 64;
  const int c = threadIdx.x & 63, r0 = threadIdx.x >> 6;
  // natural order: tall matrices have the long side as rows
  const int cols = M.tall ? M.m : M.n, rlim = M.tall ? M.n : M.m;
  const int rr = M.tall ? n0 : m0, cc = M.tall ? m0 : n0;
  for (int r = r0; r < 64; r += 4) {
    float x = 0.f;
    if (rr + r < rlim && cc + c < cols) {
      const long long e = (long long)(rr + r) * cols + cc + c;
      const float g = M.ws_u >= 0 ? ((const float *)(ws + M.ws_u))[e]
                                  : to_f32<DT>(((const typename Store<DT>::T *)src)[M.off + e]);
      x = (float)(g * inv) * scale;
    }
    tile[r][c] = x;
  }
  __syncthreads();
  _Float16 *nat = (_Float16 *)(ws + (M.tall ? M.ws_xt : M.ws_xn)), *tr = (_Float16 *)(ws + (M.tall ? M.ws_xn : M.ws_xt));
  const long long plane = (long long)M.mp * M.np;
  const int nrows = M.tall ? M.np : M.mp, ncols = M.tall ? M.mp : M.np;  // natural array, padded
  for (int r = r0; r < 64; r += 4) {
    if (rr + r < nrows && cc + c < ncols) {
      const Half2 h = ns_split(tile[r][c]);
      const long long e = (long long)(rr + r) * ncols + cc + c;
      nat[e] = h.hi;
      nat[plane + e] = h.lo;
    }
    if (cc + r < ncols && rr + c < nrows) {
      const Half2 h = ns_split(tile[c][r]);
      const long long e = (long long)(cc + r) * nrows + rr + c;
      tr[e] = h.hi;
      tr[plane + e] = h.lo;
    }
  }
}

// ---- products -----------------------------------------------------------------

enum : int { NS_GRAM = 0, NS_POLY = 1, NS_PROD = 2, NS_APPLY = 3, NS_FINAL = 4 };

// acc = A B' over k in [k0, k1): 64 x 64 tile at rows i0 of A, j0 of B, a wave 32 x 32
// (2 x 2 instructions).  A, B: [rows][ld] hi, lo one plane apart; rows past the
// arrays read their last row, the results are not stored.
__device__ __forceinline__ void tile_product(const _Float16 *A, long long pa, int ra, const _Float16 *B, long long pb,
                                             int rb, int ld, int i0, int j0, int k0, int k1, f32x4_t (&acc)[2][2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, ko = lane >> 4 << 3;
  const _Float16 *ap[2], *bp[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    ap[t] = A + (long long)min(i0 + (wave >> 1) * 32 + t * 16 + r, ra - 1) * ld + ko;
    bp[t] = B + (long long)min(j0 + (wave & 1) * 32 + t * 16 + r, rb - 1) * ld + ko;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int k = k0; k < k1; k += kStep) {
    f16x8_t ah[2], al[2], bh[2], bl[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      ah[t] = *reinterpret_cast<const f16x8_t *>(ap[t] + k);
      al[t] = *reinterpret_cast<const f16x8_t *>(ap[t] + pa + k);
      bh[t] = *reinterpret_cast<const f16x8_t *>(bp[t] + k);
      bl[t] = *reinterpret_cast<const f16x8_t *>(bp[t] + pb + k);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bl[j], acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[i], bh[j], acc[i][j], 0, 0, 0);
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[i], bh[j], acc[i][j], 0, 0, 0);
      }
  }
}

// One product of every matrix of the launch.  A, B and the output are named by their
// slots in the group's workspace:
//   GRAM   part[slice][mp][mp] = X X' over the slice's columns (fp32)
//   POLY   out = a I + b A + c A A'          (A = B = H)
//   PROD   out = A B'                        (all m x m, symmetric)
//   APPLY  xt' = xt P, xn' its transpose
//   FINAL  the output: o = xt P, or the parameter update with it
template <int MODE, int DT>
__global__ __launch_bounds__(256) void ns_product_kernel(NsTable T, NsProduct p, void *out, uint16_t *v16, char *ws) {
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int b = blockIdx.x - T.first[l];
  const int tm = (M.mp + kTile - 1) / kTile;
  constexpr bool kLong = MODE == NS_APPLY || MODE == NS_FINAL;
  int i0, j0, k0 = 0, k1 = M.mp, ra = M.mp;
  const _Float16 *A, *B;
  long long pa, ld;
  const long long sq = (long long)M.mp * M.mp, plane = (long long)M.mp * M.np;
  int slice = 0;
  if constexpr (MODE == NS_GRAM) {
    slice = b / (tm * tm);
    i0 = b / tm % tm * kTile;
    j0 = b % tm * kTile;
    const int steps = M.np / kStep, per = (steps + M.slices - 1) / M.slices;
    k0 = min(slice * per, steps) * kStep;
    k1 = min((slice + 1) * per, steps) * kStep;
    A = B = (const _Float16 *)(ws + M.ws_xn);
    pa = plane;
    ld = M.np;
  } else if constexpr (kLong) {
    i0 = b / tm * kTile;
    j0 = b % tm * kTile;
    A = (const _Float16 *)(ws + (p.a ? M.ws_xt2 : M.ws_xt));
    B = (const _Float16 *)(ws + M.ws_sq) + 2 * sq * p.b;
    pa = plane;
    ra = M.np;
    ld = M.mp;
  } else {
    i0 = b / tm * kTile;
    j0 = b % tm * kTile;
    A = (const _Float16 *)(ws + M.ws_sq) + 2 * sq * p.a;
    B = (const _Float16 *)(ws + M.ws_sq) + 2 * sq * p.b;
    pa = sq;
    ld = M.mp;
  }
  f32x4_t acc[2][2];
  tile_product(A, pa, ra, B, MODE == NS_GRAM ? plane : sq, M.mp, (int)ld, i0, j0, k0, k1, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int ti = 0; ti < 2; ++ti)
#pragma unroll
    for (int tj = 0; tj < 2; ++tj) {
      const int i = i0 + (wave >> 1) * 32 + ti * 16 + (lane >> 4) * 4;  // rows i .. i + 3
      const int j = j0 + (wave & 1) * 32 + tj * 16 + (lane & 15);
      if (j >= M.mp || i >= (kLong ? M.np : M.mp)) continue;
      if constexpr (MODE == NS_GRAM) {
        float *part = (float *)(ws + M.ws_part) + slice * sq;
#pragma unroll
        for (int q = 0; q < 4; ++q) part[(long long)(i + q) * M.mp + j] = acc[ti][tj][q] * p.unscale;
      } else if constexpr (MODE == NS_POLY || MODE == NS_PROD) {
        _Float16 *o = (_Float16 *)(ws + M.ws_sq) + 2 * sq * p.out;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const long long e = (long long)(i + q) * M.mp + j;
          float x = acc[ti][tj][q] * p.unscale;
          if constexpr (MODE == NS_POLY) {
            const float h = ((float)A[e] + (float)A[sq + e]) * p.unscale_h;
            x = p.cc * x + p.cb * h;
            if (i + q == j && j < M.m) x += p.ca;
          }
          const Half2 s = ns_split(x * p.scale);
          o[e] = s.hi;
          o[sq + e] = s.lo;
        }
      } else if constexpr (MODE == NS_APPLY) {
        _Float16 *xt = (_Float16 *)(ws + (p.a ? M.ws_xt : M.ws_xt2)), *xn = (_Float16 *)(ws + M.ws_xn);
        f16x4_t hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const Half2 s = ns_split(acc[ti][tj][q] * p.unscale * p.scale);
          xt[(long long)(i + q) * M.mp + j] = s.hi;
          xt[plane + (long long)(i + q) * M.mp + j] = s.lo;
          hi[q] = s.hi;
          lo[q] = s.lo;
        }
        *reinterpret_cast<f16x4_t *>(xn + (long long)j * M.np + i) = hi;
        *reinterpret_cast<f16x4_t *>(xn + plane + (long long)j * M.np + i) = lo;
      } else {
        if (j >= M.m) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (i + q >= M.n) continue;
          const long long e = M.off + (M.tall ? (long long)(i + q) * M.m + j : (long long)j * M.n + i + q);
          const float x = acc[ti][tj][q] * p.unscale;
          if (p.update) {
            float *v = (float *)out;
            const float w = v[e] - p.eta * (M.gain * x + p.decay * v[e]);
            v[e] = w;
            if (v16) v16[e] = f2bf(w);
          } else {
            ((typename Store<DT>::T *)out)[e] = from_f32<DT>(x);
          }
        }
      }
    }
}

// H = sum of the slices' Gram matrices, in slice order
__global__ __launch_bounds__(256) void ns_gram_sum_kernel(NsTable T, int slot, float scale, char *ws) {
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const long long sq = (long long)M.mp * M.mp;
  const long long e = (long long)(blockIdx.x - T.first[l]) * 256 + threadIdx.x;
  if (e >= sq) return;
  const float *part = (const float *)(ws + M.ws_part) + e;
  float s = 0.f;
  for (int i = 0; i < M.slices; ++i) s += part[i * sq];
  const Half2 h = ns_split(s * scale);
  _Float16 *o = (_Float16 *)(ws + M.ws_sq) + 2 * sq * slot;
  o[e] = h.hi;
  o[sq + e] = h.lo;
}

}  // namespace

// ---- plan and launches ---------------------------------------------------------

namespace {
long long up(long long n, long long a) { return (n + a - 1) / a * a; }

// first workgroup of every matrix that the general kernels run; returns their number
template <class F> int number(NsTable *T, F blocks) {
  int at = 0;
  for (int l = 0; l < T->count; ++l) {
    T->first[l] = at;
    if (!T->mat[l].mt) at += (int)blocks(T->mat[l]);
  }
  T->first[T->count] = at;
  return at;
}

enum : int { SQ_H = 0, SQ_Q = 1, SQ_T = 2, SQ_Q1 = 3, SQ_P = 4, SQ_COUNT = 5 };
}  // namespace

bool ns_scales(double a, double b, double c, int steps, NsSteps *S) {
  S->a = a;
  S->b = b;
  S->c = c;
  S->stages = (steps + 1) / 2;
  // the largest power of two that keeps values up to `bound` and twice that below 2^16:
  // room for rounding and for what lies between the points at which the bounds are taken
  auto scale = [](double bound) {
    int e = 0;
    (void)frexp(32768.0 / (1.05 * (bound > 0.125 ? bound : 0.125)), &e);
    return (float)ldexp(1.0, e - 1 < 14 ? e - 1 : 14);
  };
  auto most = [](double x, double y) { return x > y ? x : y; };
  constexpr int N = 64;  // (every call pays for them: 8192 points took 100 us)
  double sigma = 1.0;    // bound of the singular values
  for (int s = 0; s < S->stages; ++s) {
    NsStage &G = S->stage[s];
    G = NsStage{};
    G.steps = 2 * s + 1 < steps ? 2 : 1;
    G.sx = scale(sigma);
    double hb[2] = {sigma * sigma, 0.0}, qb[2] = {0.0, 0.0}, tb = 0.0, pb = 0.0, next = 0.0;
    for (int i = 0; i <= N; ++i) {
      const double x = sigma * i / N, h = x * x, q = fabs(a + b * h + c * h * h);
      const double y = x * q, h1 = y * y, q1 = G.steps == 2 ? fabs(a + b * h1 + c * h1 * h1) : 1.0;
      qb[0] = most(q, qb[0]);
      tb = most(q * h, tb);
      hb[1] = most(h1, hb[1]);
      qb[1] = most(q1, qb[1]);
      pb = most(q * q1, pb);
      next = most(y * q1, next);
    }
    if (!(qb[0] < 1024.0 && qb[1] < 1024.0 && pb < 16384.0 && tb < 1024.0 && hb[1] < 1024.0 && next < 32.0)) return false;
    for (int k = 0; k < 2; ++k) {
      G.sh[k] = scale(hb[k]);
      G.sq[k] = scale(qb[k]);
    }
    G.st = scale(tb);
    G.sp = scale(pb);
    sigma = most(next, 0.125);
  }
  return true;
}

size_t ns_plan(int count, const long long *off, const int *rows, const int *cols, int dtype, bool momentum, NsTable *T) {
  long long at = 0;
  auto take = [&](long long bytes) {
    const long long p = at;
    at += up(bytes, 256);
    return p;
  };
  T->count = count;
  for (int l = 0; l < count; ++l) {
    NsMat &M = T->mat[l];
    M.off = off[l];
    M.tall = rows[l] >= cols[l];
    M.m = M.tall ? cols[l] : rows[l];
    M.n = M.tall ? rows[l] : cols[l];
    const long long el = (long long)M.m * M.n;
    M.mt = 0;
    if (M.m <= 128) {
      int mt = 16;
      while (mt < M.m) mt *= 2;
      M.mt = mt;
      // chunks of about 8192 elements, at most 512
      M.prow = (int)up(8192 / mt, 64);
      while (((long long)M.n + M.prow - 1) / M.prow > 512) M.prow *= 2;
      M.chunks = (M.n + M.prow - 1) / M.prow;
      // workgroups of four waves: a wave takes 32 rows at a time
      const long long wgs = ((long long)M.n + 127) / 128;
      M.slices = (int)(wgs < kNumCUs ? wgs : kNumCUs);
      const int tt = mt / 16;
      const bool direct = !momentum && dtype == DT_F32 && M.tall && M.m == mt;
      M.ws_norm = take(8LL * M.chunks);
      const long long x = take(4LL * M.n * mt);
      M.ws_u = direct ? -1 : x;
      M.ws_xn = x;
      M.ws_sq = take((long long)mt * ((tt + 1) / 2) * 128);
      M.ws_part = take(1024LL * (tt * (tt + 1) / 2) * M.slices);
      M.ws_sum = take(1024LL * (tt * (tt + 1) / 2));
      continue;
    }
    M.mp = (int)up(M.m, kStep);
    M.np = (int)up(M.n, kStep);
    M.shift = 0;
    while ((el + ((long long)kNsChunk << M.shift) - 1) / ((long long)kNsChunk << M.shift) > 512) ++M.shift;
    M.chunks = (int)((el + ((long long)kNsChunk << M.shift) - 1) / ((long long)kNsChunk << M.shift));
    const int tm = (M.mp + kTile - 1) / kTile, ksteps = M.np / kStep;
    // slices of the long side: about four workgroups a compute unit, eight k-steps at least
    int slices = (4 * kNumCUs + tm * tm - 1) / (tm * tm);
    if (slices > (ksteps + 7) / 8) slices = (ksteps + 7) / 8;
    M.slices = slices;
    const long long plane = (long long)M.mp * M.np, sq = (long long)M.mp * M.mp;
    M.ws_norm = take(8LL * M.chunks);
    M.ws_u = momentum ? take(4 * el) : -1;
    M.ws_xn = take(4 * plane);
    M.ws_xt = take(4 * plane);
    M.ws_xt2 = take(4 * plane);
    M.ws_sq = take(4 * sq * SQ_COUNT);
    M.ws_part = take(4 * sq * slices);
  }
  return (size_t)at;
}

hipError_t launch_newton_schulz(const NsTable &T0, const NsSteps &S, int dtype, const void *g, const NsMomentum *mom,
                                float *m, const NsUpdate *up_, void *out, uint16_t *v16, void *ws_, hipStream_t st) {
  const hipError_t skinny = launch_ns_skinny(T0, S, dtype, g, mom, m, up_, out, v16, ws_, st);
  if (skinny != hipSuccess) return skinny;
  NsTable T = T0;
  char *ws = (char *)ws_;
  int nb = number(&T, [](const NsMat &M) { return M.chunks; });
  if (nb == 0) return hipSuccess;
  if (mom)
    hipLaunchKernelGGL((ns_prep_kernel<DT_F32, true>), dim3(nb), dim3(256), 0, st, T, *mom, g, m, ws);
  else if (dtype == DT_BF16)
    hipLaunchKernelGGL((ns_prep_kernel<DT_BF16, false>), dim3(nb), dim3(256), 0, st, T, NsMomentum{}, g, m, ws);
  else
    hipLaunchKernelGGL((ns_prep_kernel<DT_F32, false>), dim3(nb), dim3(256), 0, st, T, NsMomentum{}, g, m, ws);
  nb = number(&T, [](const NsMat &M) { return up(M.mp, 64) / 64 * (up(M.np, 64) / 64); });
  const float sx0 = S.stage[0].sx;
  if (dtype == DT_BF16)
    hipLaunchKernelGGL((ns_split_kernel<DT_BF16>), dim3(nb), dim3(256), 0, st, T, S.eps, sx0, g, ws);
  else
    hipLaunchKernelGGL((ns_split_kernel<DT_F32>), dim3(nb), dim3(256), 0, st, T, S.eps, sx0, g, ws);
  auto tiles = [](const NsMat &M) {
    const long long t = (M.mp + kTile - 1) / kTile;
    return t * t;
  };
  const float a = (float)S.a, b = (float)S.b, c = (float)S.c;
  for (int s = 0; s < S.stages; ++s) {
    const NsStage &G = S.stage[s];
    const bool last = s + 1 == S.stages;
    auto product = [&](auto mode, int pa, int pb, int po, float unscale, float unscale_h, float scale) {
      NsProduct p{};
      p.a = pa; p.b = pb; p.out = po;
      p.unscale = unscale; p.unscale_h = unscale_h; p.scale = scale;
      p.ca = a; p.cb = b; p.cc = c;
      hipLaunchKernelGGL((ns_product_kernel<decltype(mode)::value, DT_F32>), dim3(nb), dim3(256), 0, st, T, p, nullptr,
                         nullptr, ws);
    };
    using Gram = std::integral_constant<int, NS_GRAM>;
    using Poly = std::integral_constant<int, NS_POLY>;
    using Prod = std::integral_constant<int, NS_PROD>;
    using Apply = std::integral_constant<int, NS_APPLY>;
    nb = number(&T, [&](const NsMat &M) { return tiles(M) * M.slices; });
    product(Gram{}, 0, 0, 0, 1.f / (G.sx * G.sx), 0.f, 0.f);
    nb = number(&T, [](const NsMat &M) { return ((long long)M.mp * M.mp + 255) / 256; });
    hipLaunchKernelGGL(ns_gram_sum_kernel, dim3(nb), dim3(256), 0, st, T, (int)SQ_H, G.sh[0], ws);
    nb = number(&T, tiles);
    product(Poly{}, SQ_H, SQ_H, SQ_Q, 1.f / (G.sh[0] * G.sh[0]), 1.f / G.sh[0], G.sq[0]);
    int slot = SQ_Q;
    float sp = G.sq[0];
    if (G.steps == 2) {
      product(Prod{}, SQ_Q, SQ_H, SQ_T, 1.f / (G.sq[0] * G.sh[0]), 0.f, G.st);
      product(Prod{}, SQ_T, SQ_Q, SQ_H, 1.f / (G.st * G.sq[0]), 0.f, G.sh[1]);
      product(Poly{}, SQ_H, SQ_H, SQ_Q1, 1.f / (G.sh[1] * G.sh[1]), 1.f / G.sh[1], G.sq[1]);
      product(Prod{}, SQ_Q1, SQ_Q, SQ_P, 1.f / (G.sq[1] * G.sq[0]), 0.f, G.sp);
      slot = SQ_P;
      sp = G.sp;
    }
    nb = number(&T, [](const NsMat &M) { return up(M.mp, kTile) / kTile * (up(M.np, kTile) / kTile); });
    if (!last) {
      product(Apply{}, s & 1, slot, 0, 1.f / (G.sx * sp), 0.f, S.stage[s + 1].sx);
    } else {
      NsProduct p{};
      p.a = s & 1;
      p.b = slot;
      p.unscale = 1.f / (G.sx * sp);
      if (up_) {
        p.update = 1;
        p.eta = up_->eta;
        p.decay = up_->decay;
      }
      if (dtype == DT_BF16)
        hipLaunchKernelGGL((ns_product_kernel<NS_FINAL, DT_BF16>), dim3(nb), dim3(256), 0, st, T, p, out, v16, ws);
      else
        hipLaunchKernelGGL((ns_product_kernel<NS_FINAL, DT_F32>), dim3(nb), dim3(256), 0, st, T, p, out, v16, ws);
    }
  }
  return hipGetLastError();
}

}  // namespace cf
