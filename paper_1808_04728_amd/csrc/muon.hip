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

constexpr int kStep = 32;  // k of one matrix instruction; both sides are padded to it

// A matrix of fp16 pairs: a row is a sequence of 128-byte blocks of 32 columns, 32 hi
// values and 32 lo values, so that a tile's row of one k-step is one cache line.
__device__ __forceinline__ long long pair_row(int ld) { return (long long)ld * 4; }  // bytes; ld columns
__device__ __forceinline__ int pair_col(int c) { return (c >> 5) * 128 + (c & 31) * 2; }

// W consecutive columns (W divides 32) from column c on of the row at p
template <int W> __device__ __forceinline__ void store_pairs(char *p, int c, const float (&x)[W]) {
  typedef _Float16 vec_t __attribute__((ext_vector_type(W)));
  vec_t hi, lo;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const Half2 h = ns_split(x[i]);
    hi[i] = h.hi;
    lo[i] = h.lo;
  }
  *reinterpret_cast<vec_t *>(p + pair_col(c)) = hi;
  *reinterpret_cast<vec_t *>(p + pair_col(c) + 64) = lo;
}

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
  char *nat = ws + (M.tall ? M.ws_xt : M.ws_xn), *tr = ws + (M.tall ? M.ws_xn : M.ws_xt);
  const int nrows = M.tall ? M.np : M.mp, ncols = M.tall ? M.mp : M.np;  // natural array, padded
  const int row = threadIdx.x >> 2, seg = (threadIdx.x & 3) * 16;
#pragma unroll
  for (int h = 0; h < 16; h += 8) {
    float x[8];
    if (rr + row < nrows && cc + seg < ncols) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = tile[row][seg + h + i];
      store_pairs<8>(nat + (rr + row) * pair_row(ncols), cc + seg + h, x);
    }
    if (cc + row < ncols && rr + seg < nrows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = tile[seg + h + i][row];
      store_pairs<8>(tr + (cc + row) * pair_row(nrows), rr + seg + h, x);
    }
  }
}

// ---- products -----------------------------------------------------------------

enum : int { NS_GRAM = 0, NS_POLY = 1, NS_PROD = 2, NS_APPLY = 3, NS_FINAL = 4 };

typedef __attribute__((address_space(3))) void lds_void_t;
typedef const __attribute__((address_space(1))) void global_void_t;

// A square tile of B columns: WR x WC waves of TR x TC matrix instructions each, NS
// k-steps of both factors in LDS.
template <int B_> struct Tile;
template <> struct Tile<64> {
  static constexpr int B = 64, WR = 2, WC = 2, NS = 4;
};
template <> struct Tile<128> {
  static constexpr int B = 128, WR = 2, WC = 2, NS = 2;
};
template <> struct Tile<256> {
  static constexpr int B = 256, WR = 2, WC = 4, NS = 2;
};
template <class G> struct TileGeo {
  static constexpr int NT = 64 * G::WR * G::WC;
  static constexpr int TR = G::B / G::WR / 16, TC = G::B / G::WC / 16;
  static constexpr int STAGE = 2 * G::B * 128;  // bytes of one k-step
  static constexpr int LD = G::B * 8 / NT;      // 16-byte loads a thread and factor
};

// Both factors' rows of one k-step into LDS, 16 bytes a lane straight from memory.  LDS
// rows are 128 bytes; piece c of row r is at piece c ^ ((r >> 1) & 7), which spreads the
// sixteen rows of a fragment over all banks.
template <class G> struct Loader {
  using T = TileGeo<G>;
  const char *a, *b;  // first row of the tile, this k-step
  uint32_t ao[T::LD], bo[T::LD];
  __device__ __forceinline__ Loader(const char *A, int ra, int i0, const char *B, int rb, int j0, int ld, int k0) {
    a = A + i0 * pair_row(ld) + (long long)k0 * 4;
    b = B + j0 * pair_row(ld) + (long long)k0 * 4;
#pragma unroll
    for (int i = 0; i < T::LD; ++i) {
      const int id = i * T::NT + threadIdx.x, row = id >> 3, c = (id & 7) ^ ((row >> 1) & 7);
      ao[i] = (uint32_t)(min(row, ra - 1 - i0) * pair_row(ld)) + c * 16;
      bo[i] = (uint32_t)(min(row, rb - 1 - j0) * pair_row(ld)) + c * 16;
    }
  }
  // the next k-step into `stage`
  __device__ __forceinline__ void issue(char *stage) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = 0; i < T::LD; ++i)
      __builtin_amdgcn_global_load_lds((global_void_t *)(a + ao[i]), (lds_void_t *)(stage + (i * T::NT + wave * 64) * 16), 16,
                                       0, 0);
#pragma unroll
    for (int i = 0; i < T::LD; ++i)
      __builtin_amdgcn_global_load_lds((global_void_t *)(b + bo[i]),
                                       (lds_void_t *)(stage + G::B * 128 + (i * T::NT + wave * 64) * 16), 16, 0, 0);
    a += 128;
    b += 128;
  }
};

// waits until at most N of the wave's loads are in flight
template <int N> __device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

template <class G> using TileAcc = f32x4_t[TileGeo<G>::TR][TileGeo<G>::TC];

// acc = A B' over k-steps [k0, k1) / 32: rows i0.. of A, j0.. of B.  Rows past the
// arrays (ra, rb of them) read their last row; their results are not stored.
template <class G>
__device__ __forceinline__ void tile_product(TileAcc<G> &acc, char *lds, const char *A, int ra, int i0, const char *B, int rb,
                                             int j0, int ld, int k0, int k1) {
  using T = TileGeo<G>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < T::TR; ++i)
#pragma unroll
    for (int j = 0; j < T::TC; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int steps = (k1 - k0) / kStep;
  Loader<G> load(A, ra, i0, B, rb, j0, ld, k0);
#pragma unroll
  for (int s = 0; s < G::NS - 1; ++s)
    if (s < steps) load.issue(lds + s * T::STAGE);
  // this lane's pieces of a fragment: (row r, hi g) and (row r, lo g)
  const int sw = (r >> 1) & 7;
  const int fh = r * 128 + ((g ^ sw) << 4), fl = r * 128 + (((4 + g) ^ sw) << 4);
  const int arow = (wave / G::WC) * T::TR * 2048, brow = G::B * 128 + (wave % G::WC) * T::TC * 2048;
  int slot = 0;
  for (int s = 0; s < steps; ++s) {
    // the k-step's loads have landed (the later ones may be in flight), for every wave;
    // and every wave is done with the slot that the next loads overwrite
    if (s + G::NS - 1 <= steps) wait_loads<(G::NS - 2) * 2 * T::LD>();
    else wait_loads<0>();
    asm volatile("s_barrier" ::: "memory");
    if (s + G::NS - 1 < steps) load.issue(lds + (slot + G::NS - 1) % G::NS * T::STAGE);
    const char *st = lds + slot * T::STAGE;
    f16x8_t bh[T::TC], bl[T::TC];
#pragma unroll
    for (int j = 0; j < T::TC; ++j) {
      bh[j] = *reinterpret_cast<const f16x8_t *>(st + brow + j * 2048 + fh);
      bl[j] = *reinterpret_cast<const f16x8_t *>(st + brow + j * 2048 + fl);
    }
#pragma unroll
    for (int i = 0; i < T::TR; ++i) {
      const f16x8_t ah = *reinterpret_cast<const f16x8_t *>(st + arow + i * 2048 + fh);
      const f16x8_t al = *reinterpret_cast<const f16x8_t *>(st + arow + i * 2048 + fl);
#pragma unroll
      for (int j = 0; j < T::TC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bl[j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < T::TC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al, bh[j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < T::TC; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh[j], acc[i][j], 0, 0, 0);
    }
    slot = slot + 1 == G::NS ? 0 : slot + 1;
  }
}

// tile b of the upper triangle of t x t tiles, row by row
__device__ __forceinline__ void triangle_tile(int b, int t, int *ti, int *tj) {
  // row i starts at i t - i (i - 1) / 2
  const float f = t + 0.5f;
  int i = (int)(f - sqrtf(f * f - 2.f * b));
  i = max(0, min(i, t - 1));
  while (i > 0 && i * t - i * (i - 1) / 2 > b) --i;
  while ((i + 1) * t - (i + 1) * i / 2 <= b) ++i;
  *ti = i;
  *tj = i + b - (i * t - i * (i - 1) / 2);
}

// One product of every matrix of the launch.  A, B and the output are named by their
// slots in the group's workspace:
//   GRAM   part[slice] = X X' over the slice's columns (fp32, tiles of the upper triangle)
//   POLY   out = a I + b A + c A A'          (A = B = H)
//   PROD   out = A B'                        (all m x m, symmetric)
//   APPLY  xt' = xt P, xn' its transpose
//   FINAL  the output: o = xt P, or the parameter update with it
// The m x m products commute and are symmetric: tiles of the upper triangle, stored
// both ways.
template <int MODE, int TB, int DT>
__global__ __launch_bounds__(TileGeo<Tile<TB>>::NT, TB == 256 ? 1 : 2) void ns_product_kernel(NsTable T, NsProduct p, void *out,
                                                                                             uint16_t *v16, char *ws) {
  using G = Tile<TB>;
  using TG = TileGeo<G>;
  __shared__ __attribute__((aligned(16))) char lds[G::NS * TG::STAGE];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int b = blockIdx.x - T.first[l];
  const int tm = (M.mp + TB - 1) / TB;
  constexpr bool kLong = MODE == NS_APPLY || MODE == NS_FINAL;
  int ti, tj, k0 = 0, k1 = M.mp, ra = M.mp, ld = M.mp, slice = 0;
  const char *A, *B;
  const long long sq = (long long)M.mp * M.mp * 4;
  if constexpr (kLong) {
    ti = b / tm;
    tj = b % tm;
    A = ws + (p.a ? M.ws_xt2 : M.ws_xt);
    B = ws + M.ws_sq + sq * p.b;
    ra = M.np;
  } else {
    const int tri = tm * (tm + 1) / 2;
    slice = MODE == NS_GRAM ? b / tri : 0;
    triangle_tile(b - slice * tri, tm, &ti, &tj);
    if constexpr (MODE == NS_GRAM) {
      const int steps = M.np / kStep, per = (steps + M.slices - 1) / M.slices;
      k0 = min(slice * per, steps) * kStep;
      k1 = min((slice + 1) * per, steps) * kStep;
      A = B = ws + M.ws_xn;
      ld = M.np;
    } else {
      A = ws + M.ws_sq + sq * p.a;
      B = ws + M.ws_sq + sq * p.b;
    }
  }
  TileAcc<G> acc;
  tile_product<G>(acc, lds, A, ra, ti * TB, B, M.mp, tj * TB, ld, k0, k1);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if constexpr (MODE == NS_GRAM) {
    // accumulators as they are: [tile][wave tile][lane]
    float4 *part = (float4 *)(ws + M.ws_part) + ((long long)b * TG::NT / 64 * TG::TR * TG::TC) * 64;
#pragma unroll
    for (int i = 0; i < TG::TR; ++i)
#pragma unroll
      for (int j = 0; j < TG::TC; ++j)
        part[((wave * TG::TR + i) * TG::TC + j) * 64 + lane] = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
    return;
  }
#pragma unroll
  for (int ii = 0; ii < TG::TR; ++ii)
#pragma unroll
    for (int jj = 0; jj < TG::TC; ++jj) {
      const int i = ti * TB + ((wave / G::WC) * TG::TR + ii) * 16 + (lane >> 4) * 4;  // rows i .. i + 3
      const int j = tj * TB + ((wave % G::WC) * TG::TC + jj) * 16 + (lane & 15);
      if (j >= M.mp || i >= (kLong ? M.np : M.mp)) continue;
      float x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] = acc[ii][jj][q] * p.unscale;
      if constexpr (MODE == NS_POLY || MODE == NS_PROD) {
        char *o = ws + M.ws_sq + sq * p.out;
        if constexpr (MODE == NS_POLY) {
          // H is symmetric: four consecutive columns of its row j
          const char *h = A + j * pair_row(M.mp) + pair_col(i);
          const f16x4_t hh = *reinterpret_cast<const f16x4_t *>(h), hl = *reinterpret_cast<const f16x4_t *>(h + 64);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            x[q] = p.cc * x[q] + p.cb * (((float)hh[q] + (float)hl[q]) * p.unscale_h);
            if (i + q == j && j < M.m) x[q] += p.ca;
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] *= p.scale;
        store_pairs<4>(o + j * pair_row(M.mp), i, x);
        if (ti != tj) {
#pragma unroll
          for (int q = 0; q < 4; ++q) store_pairs<1>(o + (i + q) * pair_row(M.mp), j, {x[q]});
        }
      } else if constexpr (MODE == NS_APPLY) {
        char *xt = ws + (p.a ? M.ws_xt : M.ws_xt2), *xn = ws + M.ws_xn;
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] *= p.scale;
        store_pairs<4>(xn + j * pair_row(M.np), i, x);
#pragma unroll
        for (int q = 0; q < 4; ++q) store_pairs<1>(xt + (i + q) * pair_row(M.mp), j, {x[q]});
      } else {
        if (j >= M.m) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (i + q >= M.n) continue;
          const long long e = M.off + (M.tall ? (long long)(i + q) * M.m + j : (long long)j * M.n + i + q);
          if (p.update) {
            float *v = (float *)out;
            const float w = v[e] - p.eta * (M.gain * x[q] + p.decay * v[e]);
            v[e] = w;
            if (v16) v16[e] = f2bf(w);
          } else {
            ((typename Store<DT>::T *)out)[e] = from_f32<DT>(x[q]);
          }
        }
      }
    }
}

// H = sum of the slices' Gram matrices, in slice order; one matrix-instruction tile a wave
template <int TB> __global__ __launch_bounds__(256) void ns_gram_sum_kernel(NsTable T, int slot, float scale, char *ws) {
  using G = Tile<TB>;
  using TG = TileGeo<G>;
  constexpr int PER = TB / 16 * (TB / 16);  // instruction tiles of a tile
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int tm = (M.mp + TB - 1) / TB, tri = tm * (tm + 1) / 2;
  const int lane = threadIdx.x & 63, w = (blockIdx.x - T.first[l]) * 4 + (threadIdx.x >> 6);
  const int b = w / PER, k = w % PER, wave = k / (TG::TR * TG::TC);
  int ti, tj;
  triangle_tile(b, tm, &ti, &tj);
  const int i = ti * TB + ((wave / G::WC) * TG::TR + k / TG::TC % TG::TR) * 16 + (lane >> 4) * 4;
  const int j = tj * TB + ((wave % G::WC) * TG::TC + k % TG::TC) * 16 + (lane & 15);
  if (j >= M.mp || i >= M.mp) return;
  const float4 *part = (const float4 *)(ws + M.ws_part) + ((long long)b * PER + k) * 64 + lane;
  float4 s = part[0];
#pragma unroll 4
  for (int n = 1; n < M.slices; ++n) {
    const float4 a = part[(long long)n * tri * PER * 64];
    s.x += a.x; s.y += a.y; s.z += a.z; s.w += a.w;
  }
  const float x[4] = {s.x * scale, s.y * scale, s.z * scale, s.w * scale};
  char *o = ws + M.ws_sq + (long long)M.mp * M.mp * 4 * slot;
  store_pairs<4>(o + j * pair_row(M.mp), i, x);
  if (ti != tj) {
#pragma unroll
    for (int q = 0; q < 4; ++q) store_pairs<1>(o + (i + q) * pair_row(M.mp), j, {x[q]});
  }
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

// the m x m matrices of a group
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
    const long long plane = (long long)M.mp * M.np, sq = (long long)M.mp * M.mp;
    M.ws_norm = take(8LL * M.chunks);
    M.ws_u = momentum ? take(4 * el) : -1;
    M.ws_xn = take(4 * plane);
    M.ws_xt = take(4 * plane);
    M.ws_xt2 = take(4 * plane);
    M.ws_sq = take(4 * sq * SQ_COUNT);
    auto tiles = [](long long rows, long long tb) { return (rows + tb - 1) / tb; };
    auto triangle = [&](long long tb) { return tiles(M.mp, tb) * (tiles(M.mp, tb) + 1) / 2; };
    M.tile_sq = triangle(256) >= 128 ? 256 : triangle(128) >= 256 ? 128 : 64;
    auto rect = [&](long long tb) { return tiles(M.mp, tb) * tiles(M.np, tb); };
    M.tile_long = rect(256) >= 192 ? 256 : rect(128) >= 192 ? 128 : 64;
    // slices of the long side: about two workgroups a compute unit, eight k-steps at least
    const long long tri = triangle(M.tile_sq), ksteps = M.np / kStep;
    long long slices = (2 * kNumCUs + tri - 1) / tri;
    if (slices > ksteps / 8) slices = ksteps / 8 > 0 ? ksteps / 8 : 1;
    M.slices = (int)slices;
    M.ws_part = take(4LL * tri * M.tile_sq * M.tile_sq * slices);
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
  // f(tile) for each tile size that a matrix of the table uses in this product
  auto each_tile = [&](bool is_long, auto f) {
    auto used = [&](int tb) {
      for (int l = 0; l < T.count; ++l)
        if (!T.mat[l].mt && (is_long ? T.mat[l].tile_long : T.mat[l].tile_sq) == tb) return true;
      return false;
    };
    if (used(256)) f(std::integral_constant<int, 256>{});
    if (used(128)) f(std::integral_constant<int, 128>{});
    if (used(64)) f(std::integral_constant<int, 64>{});
  };
  auto product = [&](auto mode, auto dt, NsProduct p) {
    constexpr int MODE = decltype(mode)::value, DT = decltype(dt)::value;
    constexpr bool kLong = MODE == NS_APPLY || MODE == NS_FINAL;
    each_tile(kLong, [&](auto tile) {
      constexpr int TB = decltype(tile)::value;
      const int blocks = number(&T, [](const NsMat &M) {
        if ((kLong ? M.tile_long : M.tile_sq) != TB) return 0LL;
        const long long t = (M.mp + TB - 1) / TB;
        return kLong ? t * ((M.np + TB - 1) / TB) : t * (t + 1) / 2 * (MODE == NS_GRAM ? M.slices : 1);
      });
      hipLaunchKernelGGL((ns_product_kernel<MODE, TB, DT>), dim3(blocks), dim3(TileGeo<Tile<TB>>::NT), 0, st, T, p, out, v16, ws);
    });
  };
  using Gram = std::integral_constant<int, NS_GRAM>;
  using Poly = std::integral_constant<int, NS_POLY>;
  using Prod = std::integral_constant<int, NS_PROD>;
  using Apply = std::integral_constant<int, NS_APPLY>;
  using Final = std::integral_constant<int, NS_FINAL>;
  using F32 = std::integral_constant<int, DT_F32>;
  using BF16 = std::integral_constant<int, DT_BF16>;
  const float a = (float)S.a, b = (float)S.b, c = (float)S.c;
  for (int s = 0; s < S.stages; ++s) {
    const NsStage &G = S.stage[s];
    auto square = [&](auto mode, int pa, int pb, int po, float unscale, float unscale_h, float scale) {
      NsProduct p{};
      p.a = pa; p.b = pb; p.out = po;
      p.unscale = unscale; p.unscale_h = unscale_h; p.scale = scale;
      p.ca = a; p.cb = b; p.cc = c;
      product(mode, F32{}, p);
    };
    square(Gram{}, 0, 0, 0, 1.f, 0.f, 0.f);
    each_tile(false, [&](auto tile) {
      constexpr int TB = decltype(tile)::value;
      nb = number(&T, [](const NsMat &M) {
        const long long t = (M.mp + TB - 1) / TB;
        return M.tile_sq == TB ? t * (t + 1) / 2 * (TB / 16 * (TB / 16) / 4) : 0LL;
      });
      hipLaunchKernelGGL((ns_gram_sum_kernel<TB>), dim3(nb), dim3(256), 0, st, T, (int)SQ_H, G.sh[0] / (G.sx * G.sx), ws);
    });
    square(Poly{}, SQ_H, SQ_H, SQ_Q, 1.f / (G.sh[0] * G.sh[0]), 1.f / G.sh[0], G.sq[0]);
    int slot = SQ_Q;
    float sp = G.sq[0];
    if (G.steps == 2) {
      square(Prod{}, SQ_Q, SQ_H, SQ_T, 1.f / (G.sq[0] * G.sh[0]), 0.f, G.st);
      square(Prod{}, SQ_T, SQ_Q, SQ_H, 1.f / (G.st * G.sq[0]), 0.f, G.sh[1]);
      square(Poly{}, SQ_H, SQ_H, SQ_Q1, 1.f / (G.sh[1] * G.sh[1]), 1.f / G.sh[1], G.sq[1]);
      square(Prod{}, SQ_Q1, SQ_Q, SQ_P, 1.f / (G.sq[1] * G.sq[0]), 0.f, G.sp);
      slot = SQ_P;
      sp = G.sp;
    }
    NsProduct p{};
    p.a = s & 1;
    p.b = slot;
    p.unscale = 1.f / (G.sx * sp);
    if (s + 1 < S.stages) {
      p.scale = S.stage[s + 1].sx;
      product(Apply{}, F32{}, p);
    } else {
      if (up_) {
        p.update = 1;
        p.eta = up_->eta;
        p.decay = up_->decay;
      }
      if (dtype == DT_BF16) product(Final{}, BF16{}, p);
      else product(Final{}, F32{}, p);
    }
  }
  return hipGetLastError();
}

}  // namespace cf
