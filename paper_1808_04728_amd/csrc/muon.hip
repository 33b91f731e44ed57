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
// The groups of a call share launches: those of up to 128 columns or rows have the skinny
// kernels', the others these, a launch for each size of tile; a workgroup finds its matrix
// in the table of its launch.

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "muon_common.h"

namespace cf {
namespace {

constexpr int kStep = 32;  // k of one matrix instruction; both sides are padded to it

// A matrix of fp16 pairs: a row is a sequence of 128-byte blocks of 32 columns, 32 hi
// values and 32 lo values, so that a tile's row of one k-step is one cache line.
__device__ __forceinline__ long long pair_row(int ld) { return (long long)ld * 4; }  // bytes; ld columns
__device__ __forceinline__ int pair_col(int c) { return (c >> 5) * 128 + (c & 31) * 2; }

// columns c .. c + 7 (c a multiple of 8) of the row at p
__device__ __forceinline__ void store_pairs(char *p, int c, const float (&x)[8]) {
  f16x8_t hi, lo;
  ns_split8(x, hi, lo);
  *reinterpret_cast<f16x8_t *>(p + pair_col(c)) = hi;
  *reinterpret_cast<f16x8_t *>(p + pair_col(c) + 64) = lo;
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
    if (k == 4) {
      if (DT == DT_F32) {
        const float4 a = *reinterpret_cast<const float4 *>((const float *)g + M.off + e);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
      } else {
        const ushort4 a = *reinterpret_cast<const ushort4 *>((const uint16_t *)g + M.off + e);
        x[0] = to_f32<DT_BF16>(a.x); x[1] = to_f32<DT_BF16>(a.y); x[2] = to_f32<DT_BF16>(a.z); x[3] = to_f32<DT_BF16>(a.w);
      }
      if constexpr (MOM) {
        float4 v = *reinterpret_cast<const float4 *>(m + M.off + e);
        x[0] = ns_momentum(mom, x[0], v.x);
        x[1] = ns_momentum(mom, x[1], v.y);
        x[2] = ns_momentum(mom, x[2], v.z);
        x[3] = ns_momentum(mom, x[3], v.w);
        *reinterpret_cast<float4 *>(m + M.off + e) = v;
        *reinterpret_cast<float4 *>(u + e) = make_float4(x[0], x[1], x[2], x[3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = i < k ? to_f32<DT>(((const typename Store<DT>::T *)g)[M.off + e + i]) : 0.f;
        if constexpr (MOM) {
          if (i < k) {
            x[i] = ns_momentum(mom, x[i], m[M.off + e + i]);
            u[e + i] = x[i];
          }
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
  const int tm = (M.mp + 63) / 64, b = blockIdx.x - T.first[l];
  const int n0 = b / tm * 64, m0 = b % tm * 64;
  const int c = threadIdx.x & 63, r0 = threadIdx.x >> 6;
  // natural order: tall matrices have the long side as rows
  const int cols = M.tall ? M.m : M.n, rlim = M.tall ? M.n : M.m;
  const int rr = M.tall ? n0 : m0, cc = M.tall ? m0 : n0;
  float x[16];
  // (from an element that exists, whatever the lane: loads under a condition would wait one
  // for the other, 15 us instead of 10 for 517 x 2051)
  auto load = [&](const auto *p, auto value) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[i] = value(p[(long long)min(rr + r0 + 4 * i, rlim - 1) * cols + min(cc + c, cols - 1)]);
  };
  if (M.ws_u >= 0) load((const float *)(ws + M.ws_u), [](float v) { return v; });
  else load((const typename Store<DT>::T *)src + M.off, [](auto v) { return to_f32<DT>(v); });
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (rr + r0 + 4 * i >= rlim || cc + c >= cols) x[i] = 0.f;
  const Scale sc = scale_of(ns_inv_norm(M, ws, eps, red), scale);
#pragma unroll
  for (int i = 0; i < 16; ++i) tile[r0 + 4 * i][c] = x[i] * sc.s1 * sc.s2;
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
      store_pairs(nat + (rr + row) * pair_row(ncols), cc + seg + h, x);
    }
    if (cc + row < ncols && rr + seg < nrows) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = tile[seg + h + i][row];
      store_pairs(tr + (cc + row) * pair_row(nrows), rr + seg + h, x);
    }
  }
}

// ---- products -----------------------------------------------------------------

enum : int { NS_GRAM = 0, NS_POLY = 1, NS_PROD = 2, NS_APPLY = 3, NS_FINAL = 4 };

typedef __attribute__((address_space(3))) void lds_void_t;
typedef const __attribute__((address_space(1))) void global_void_t;

// A square tile of B columns: WR x WC waves of TR x TC matrix instructions each, NS
// turns of KS k-steps of both factors in LDS.  Small tiles have KG such groups of waves,
// each with its own turns (group k the turns k, k + KG, ...) and loads; one group alone
// waits for LDS and the barrier most of a step (64: 0.32 us a step, of which the matrix
// instructions are 0.08; two groups 0.26, two k-steps a turn 0.22).  The smallest tile has
// a wave a group and eight k-steps on their way: 0.1 us a step.
template <int B_> struct Tile;
template <> struct Tile<32> {
  static constexpr int B = 32, WR = 1, WC = 1, NS = 2, KG = 8, KS = 1;
};
template <> struct Tile<64> {
  static constexpr int B = 64, WR = 2, WC = 2, NS = 2, KG = 2, KS = 2;
};
template <> struct Tile<128> {
  static constexpr int B = 128, WR = 2, WC = 2, NS = 2, KG = 2, KS = 1;
};
template <> struct Tile<192> {
  static constexpr int B = 192, WR = 2, WC = 4, NS = 3, KG = 1, KS = 1;
};
template <> struct Tile<256> {
  static constexpr int B = 256, WR = 2, WC = 4, NS = 2, KG = 1, KS = 1;
};
constexpr int pow2_of(int n) { return n & -n; }
// In a wave's part of the tile, instruction tile (ii, jj) has rows 4 g + q and columns r at
// row (4 g + q) TR + ii and column r TC + jj: a lane holds 4 TR consecutive rows of TC
// consecutive columns.  (The factors' rows are put into LDS in that order.)
template <class G> struct TileGeo {
  static constexpr int NG = 64 * G::WR * G::WC, NT = NG * G::KG;  // threads of a group, of the workgroup
  static constexpr int TR = G::B / G::WR / 16, TC = G::B / G::WC / 16;
  static constexpr int STEP = 2 * G::B * 128, STAGE = G::KS * STEP;  // bytes of a k-step, of a turn
  static constexpr int LDS = G::NS * G::KG * STAGE;
  static_assert(G::KS == 1 || G::NS == 2, "a turn of fewer k-steps has fewer loads to wait for");
  static constexpr int LD = G::B * 8 / NG;  // 16-byte loads a thread and factor
  static constexpr int VJ = pow2_of(TC);
  static constexpr int OROW = 16 * TR * 4 + 16;  // bytes of an output row of a wave in LDS
  static_assert(4 * TR % 8 == 0 && TC <= 4, "rows are stored by eights, columns by at most four");
  static_assert(16 * OROW * G::WR * G::WC <= LDS, "every wave's output rows in LDS");
  // tile row of LDS row s, for a factor whose waves have T instruction tiles
  static __device__ __forceinline__ int tile_row(int s, int T) { return s / (16 * T) * (16 * T) + s % 16 * T + s / 16 % T; }
};

// Both factors' rows of one k-step into LDS, 16 bytes a lane straight from memory.  LDS
// rows are 128 bytes; piece c of row r is at piece c ^ ((r >> 1) & 7), which spreads the
// sixteen rows of a fragment over all banks.
template <class G> struct Loader {
  using T = TileGeo<G>;
  const char *a, *b;  // first row of the tile, this k-step
  uint32_t ao[T::LD], bo[T::LD];  // (the plan takes only tiles whose rows they reach)
  __device__ __forceinline__ Loader(const char *A, int ra, int i0, const char *B, int rb, int j0, int ld, int k0) {
    a = A + i0 * pair_row(ld) + (long long)k0 * 4;
    b = B + j0 * pair_row(ld) + (long long)k0 * 4;
#pragma unroll
    for (int i = 0; i < T::LD; ++i) {
      const int id = i * T::NG + threadIdx.x % T::NG, row = id >> 3, c = (id & 7) ^ ((row >> 1) & 7);
      ao[i] = (uint32_t)(min(T::tile_row(row, T::TR), ra - 1 - i0) * pair_row(ld)) + c * 16;
      bo[i] = (uint32_t)(min(T::tile_row(row, T::TC), rb - 1 - j0) * pair_row(ld)) + c * 16;
    }
  }
  // the group's next turn of `have` k-steps into `stage`
  __device__ __forceinline__ void issue(char *stage, int have) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x % T::NG >> 6);
#pragma unroll
    for (int k = 0; k < G::KS; ++k) {
      if (k >= have) break;
      char *st = stage + k * T::STEP;
#pragma unroll
      for (int i = 0; i < T::LD; ++i)
        __builtin_amdgcn_global_load_lds((global_void_t *)(a + k * 128 + ao[i]), (lds_void_t *)(st + (i * T::NG + wave * 64) * 16),
                                         16, 0, 0);
#pragma unroll
      for (int i = 0; i < T::LD; ++i)
        __builtin_amdgcn_global_load_lds((global_void_t *)(b + k * 128 + bo[i]),
                                         (lds_void_t *)(st + G::B * 128 + (i * T::NG + wave * 64) * 16), 16, 0, 0);
    }
    a += 128 * G::KG * G::KS;
    b += 128 * G::KG * G::KS;
  }
};

// waits until at most N of the wave's loads are in flight
template <int N> __device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

template <class G> using TileAcc = f32x4_t[TileGeo<G>::TR][TileGeo<G>::TC];

// acc = A B' over the columns [k0, k1) (multiples of 32): rows i0.. of A, j0.. of B; the
// first group's waves have it.  Rows past the arrays (ra, rb of them) read their last
// row; their results are not stored.
template <class G>
__device__ __forceinline__ void tile_product(TileAcc<G> &acc, char *lds, const char *A, int ra, int i0, const char *B, int rb,
                                             int j0, int ld, int k0, int k1) {
  using T = TileGeo<G>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x % T::NG >> 6, r = lane & 15, g = lane >> 4;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / T::NG);
#pragma unroll
  for (int i = 0; i < T::TR; ++i)
#pragma unroll
    for (int j = 0; j < T::TC; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int all = (k1 - k0) / kStep, sets = (all + G::KS - 1) / G::KS;  // k-steps, turns of all groups
  const int steps = (sets - group + G::KG - 1) / G::KG, turns = (sets + G::KG - 1) / G::KG;
  auto have = [&](int s) { return min(G::KS, all - (s * G::KG + group) * G::KS); };  // k-steps of the group's turn s
  char *ring = lds + group * G::NS * T::STAGE;
  Loader<G> load(A, ra, i0, B, rb, j0, ld, k0 + group * G::KS * kStep);
#pragma unroll
  for (int s = 0; s < G::NS - 1; ++s)
    if (s < steps) load.issue(ring + s * T::STAGE, have(s));
  // this lane's pieces of a fragment: (row r, hi g) and (row r, lo g)
  const int sw = (r >> 1) & 7;
  const int fh = r * 128 + ((g ^ sw) << 4), fl = r * 128 + (((4 + g) ^ sw) << 4);
  const int arow = (wave / G::WC) * T::TR * 2048, brow = G::B * 128 + (wave % G::WC) * T::TC * 2048;
  // Two halves of the waves, the later one a phase behind the other: while the matrix
  // instructions of one run, the fragments of the other come from LDS.  A barrier ends
  // every phase.  (Waves w and w + 4 share a SIMD.)
  static_assert(T::NT == 512, "two waves a SIMD");
  const bool late = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) >= 4;
  auto barrier = [] {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto wait_lds = [] { __builtin_amdgcn_s_waitcnt(0xc07f); };  // lgkmcnt(0)
  // the wave's loads of the k-step s + 1 have landed (later ones may be in flight)
  auto wait_next = [&](int s) {
    if (s + G::NS <= steps) wait_loads<(G::NS - 2) * 2 * T::LD>();
    else wait_loads<0>();
  };
  // phases of a k-step, rows of instruction tiles in one: the fragments of a whole step where
  // the registers hold them beside the accumulators
  constexpr int PH = G::B == 256 ? 2 : 1, HR = T::TR / PH;
  static_assert(T::TR % PH == 0, "phases of equal rows");
  wait_next(-1);
  barrier();
  if (late) barrier();
  int slot = 0;
  for (int s = 0; s < turns; ++s) {
    // every wave has read all of the slot that the next loads overwrite: the reads of
    // both halves were over before the last barrier
    if (s + G::NS - 1 < steps) load.issue(ring + (slot + G::NS - 1) % G::NS * T::STAGE, have(s + G::NS - 1));
    const char *st = ring + slot * T::STAGE;
    f16x8_t bh[G::KS][T::TC], bl[G::KS][T::TC];
#pragma unroll
    for (int k = 0; k < G::KS; ++k)
#pragma unroll
      for (int j = 0; j < T::TC; ++j) {
        bh[k][j] = *reinterpret_cast<const f16x8_t *>(st + k * T::STEP + brow + j * 2048 + fh);
        bl[k][j] = *reinterpret_cast<const f16x8_t *>(st + k * T::STEP + brow + j * 2048 + fl);
      }
#pragma unroll
    for (int half = 0; half < PH; ++half) {
      f16x8_t ah[G::KS][HR], al[G::KS][HR];
#pragma unroll
      for (int k = 0; k < G::KS; ++k)
#pragma unroll
        for (int i = 0; i < HR; ++i) {
          ah[k][i] = *reinterpret_cast<const f16x8_t *>(st + k * T::STEP + arow + (half * HR + i) * 2048 + fh);
          al[k][i] = *reinterpret_cast<const f16x8_t *>(st + k * T::STEP + arow + (half * HR + i) * 2048 + fl);
        }
      wait_lds();
      // (one group: the early half reads the next k-step, all waves' loads of it, right
      // after the barrier that ends the later half's last load phase)
      if (G::KG == 1 && half == PH - 1) wait_next(s);
      barrier();
      if (G::KG == 1 || s < steps) {  // (a group without a last step only keeps the barriers)
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < G::KS; ++k) {
          if (k > 0 && k >= have(s)) break;  // (the last turn's missing k-step)
#pragma unroll
          for (int i = 0; i < HR; ++i)
#pragma unroll
            for (int j = 0; j < T::TC; ++j)
              acc[half * HR + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[k][i], bl[k][j], acc[half * HR + i][j], 0, 0, 0);
#pragma unroll
          for (int i = 0; i < HR; ++i)
#pragma unroll
            for (int j = 0; j < T::TC; ++j)
              acc[half * HR + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(al[k][i], bh[k][j], acc[half * HR + i][j], 0, 0, 0);
#pragma unroll
          for (int i = 0; i < HR; ++i)
#pragma unroll
            for (int j = 0; j < T::TC; ++j)
              acc[half * HR + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah[k][i], bh[k][j], acc[half * HR + i][j], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
      }
      if (G::KG > 1) wait_next(s);  // (two groups: each reads its own loads)
      barrier();
    }
    slot = slot + 1 == G::NS ? 0 : slot + 1;
  }
  if (!late) barrier();
  __syncthreads();  // the output goes through the LDS
  if constexpr (G::KG > 1) {
    // the other groups' accumulators through the LDS, added in group order
    static_assert((G::KG - 1) * G::B * G::B * 4 <= T::LDS, "their tiles in LDS");
    f32x4_t *part = reinterpret_cast<f32x4_t *>(lds);
    constexpr int TILE = G::WR * G::WC * T::TR * T::TC * 64;
#pragma unroll
    for (int i = 0; i < T::TR; ++i)
#pragma unroll
      for (int j = 0; j < T::TC; ++j)
        if (group > 0) part[(group - 1) * TILE + ((wave * T::TR + i) * T::TC + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int o = 0; o < G::KG - 1; ++o)
#pragma unroll
        for (int i = 0; i < T::TR; ++i)
#pragma unroll
          for (int j = 0; j < T::TC; ++j) acc[i][j] += part[o * TILE + ((wave * T::TR + i) * T::TC + j) * 64 + lane];
    }
    __syncthreads();
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

// where a lane's part of the tile begins
template <class G> struct Origin {
  int i, j;
  __device__ __forceinline__ Origin(int ti, int tj, int part) {
    using T = TileGeo<G>;
    const int lane = threadIdx.x & 63;
    i = ti * G::B + part / G::WC * T::TR * 16 + (lane >> 4) * 4 * T::TR;
    j = tj * G::B + part % G::WC * T::TC * 16 + (lane & 15) * T::TC;
  }
};

// value of the lane's row di (0 .. 4 TR - 1) and column jj
template <class G> __device__ __forceinline__ float acc_at(const TileAcc<G> &acc, int di, int jj) {
  return acc[di % TileGeo<G>::TR][jj][di / TileGeo<G>::TR];
}

// The tile times `scale` as pairs: by columns into `cols` (row j has the tile's column j,
// `ldc` columns) and, unless null, by rows into `rows` (`ldr` columns).  Rows past ilim and
// columns past jlim (multiples of 32) are not stored.  By rows sixteen lanes store 64
// bytes in a piece as they are; by columns a lane has a whole line, and sixteen rows at
// a time pass through the wave's part of the LDS so that eight lanes store a line
// together (each its own line took 25 of a 256 tile's 42 us at 256 columns).  `part`: which
// wave's part the accumulators are, that of the wave itself after a product.
template <class G>
__device__ __forceinline__ void store_tile(const TileAcc<G> &acc, char *lds, int ti, int tj, float scale, char *cols, int ldc,
                                           char *rows, int ldr, int ilim, int jlim, int part) {
  using T = TileGeo<G>;
  const Origin<G> at(ti, tj, part);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int iw = ti * G::B + part / G::WC * T::TR * 16, jw = tj * G::B + part % G::WC * T::TC * 16;
  char *mine = lds + wave * 16 * T::OROW;
  f16x8_t hi[T::TR / 2][T::TC], lo[T::TR / 2][T::TC];
#pragma unroll
  for (int jj = 0; jj < T::TC; ++jj) {
#pragma unroll
    for (int e = 0; e < T::TR / 2; ++e) {
      float x[8];
#pragma unroll
      for (int d = 0; d < 8; ++d) x[d] = acc_at<G>(acc, 8 * e + d, jj) * scale;
      ns_split8(x, hi[e][jj], lo[e][jj]);
      char *p = mine + r * T::OROW + pair_col(g * 4 * T::TR + 8 * e);
      *reinterpret_cast<f16x8_t *>(p) = hi[e][jj];
      *reinterpret_cast<f16x8_t *>(p + 64) = lo[e][jj];
    }
    // (the LDS accesses of one wave are in order)
    constexpr int C = T::TR * 4;  // 16-byte pieces of a row
#pragma unroll
    for (int k = 0; k < T::TR; ++k) {
      const int id = k * 64 + lane, row = id / C, c = id % C;
      const u32x4_t v = *reinterpret_cast<const u32x4_t *>(mine + row * T::OROW + c * 16);
      const int j = jw + row * T::TC + jj;
      if (j < jlim && iw + (c >> 3) * 32 < ilim)
        *reinterpret_cast<u32x4_t *>(cols + j * pair_row(ldc) + (iw >> 5) * 128 + c * 16) = v;
    }
  }
  if (!rows) return;
  typedef _Float16 vec_t __attribute__((ext_vector_type(T::VJ)));
  char *rp = rows + at.i * pair_row(ldr);
#pragma unroll
  for (int e = 0; e < T::TR / 2; ++e) {
    if (at.i + 8 * e >= ilim) break;
#pragma unroll
    for (int d = 0; d < 8; ++d)
#pragma unroll
      for (int j0 = 0; j0 < T::TC; j0 += T::VJ) {
        vec_t h, l;
#pragma unroll
        for (int k = 0; k < T::VJ; ++k) {
          h[k] = hi[e][j0 + k][d];
          l[k] = lo[e][j0 + k][d];
        }
        if (at.j + j0 < jlim) {
          char *p = rp + (8 * e + d) * pair_row(ldr) + pair_col(at.j + j0);
          *reinterpret_cast<vec_t *>(p) = h;
          *reinterpret_cast<vec_t *>(p + 64) = l;
        }
      }
  }
}

// One product of every matrix of the launch.  A, B and the output are named by their
// slots in the group's workspace:
//   GRAM   part[slice] = X X' over the slice's columns (fp32, tiles of the upper triangle)
//   POLY   out = a I + b A + c A A'          (A = B = H)
//   PROD   out = A B'                        (all m x m, symmetric)
//   APPLY  xt' = xt P, xn' its transpose
//   FINAL  the output: o = xt P, or the parameter update with it
// The m x m products commute and are symmetric: tiles of the upper triangle, stored
// both ways.  The matrix cores bound large ones: 4096 x 4096 takes 290 us a product
// (256 tiles, 1.42 PFLOP/s of half-precision instructions) and 176 a triangle (192 tiles,
// 1.25).  Small ones wait for their loads: 4.5 us for a launch, its first loads and its
// stores, then 0.1 us a k-step of 32 tiles and 0.22 of 64.
template <int MODE, int TB, int DT>
__global__ __launch_bounds__(TileGeo<Tile<TB>>::NT, 1) void ns_product_kernel(NsTable T, NsProduct p, void *out, uint16_t *v16,
                                                                              char *ws) {
  using G = Tile<TB>;
  using TG = TileGeo<G>;
  __shared__ __attribute__((aligned(16))) char lds[TG::LDS];
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
  if (threadIdx.x >= TG::NG) return;
  const int wave = threadIdx.x >> 6;
  char *o = ws + M.ws_sq + sq * p.out;
  if (MODE == NS_GRAM && M.slices == 1) {
    store_tile<G>(acc, lds, ti, tj, p.unscale * p.scale, o, M.mp, ti != tj ? o : nullptr, M.mp, M.mp, M.mp, wave);
  } else if constexpr (MODE == NS_GRAM) {
    // accumulators as they are: [slice][tile][wave tile][lane]
    float4 *part = (float4 *)(ws + M.ws_part) + (long long)b * (TB * TB / 4) + (threadIdx.x >> 6) * TG::TR * TG::TC * 64 +
                   (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < TG::TR; ++i)
#pragma unroll
      for (int j = 0; j < TG::TC; ++j)
        part[(i * TG::TC + j) * 64] = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
  } else if constexpr (MODE == NS_POLY || MODE == NS_PROD) {
    float scale = p.unscale * p.scale;
    if constexpr (MODE == NS_POLY) {
      // H is symmetric: eight consecutive columns of its row j
      const Origin<G> at(ti, tj, wave);
#pragma unroll
      for (int jj = 0; jj < TG::TC; ++jj)
#pragma unroll
        for (int e = 0; e < 4 * TG::TR; e += 8) {
          if (at.j + jj >= M.mp || at.i + e >= M.mp) continue;
          const char *h = A + (at.j + jj) * pair_row(M.mp) + pair_col(at.i + e);
          const f16x8_t hh = *reinterpret_cast<const f16x8_t *>(h), hl = *reinterpret_cast<const f16x8_t *>(h + 64);
#pragma unroll
          for (int d = 0; d < 8; ++d) {
            const int ii = (e + d) % TG::TR, q = (e + d) / TG::TR;
            float x = p.cc * (acc[ii][jj][q] * p.unscale) + p.cb * (((float)hh[d] + (float)hl[d]) * p.unscale_h);
            if (at.i + e + d == at.j + jj && at.j + jj < M.m) x += p.ca;
            acc[ii][jj][q] = x;
          }
        }
      scale = p.scale;
    }
    store_tile<G>(acc, lds, ti, tj, scale, o, M.mp, ti != tj ? o : nullptr, M.mp, M.mp, M.mp, wave);
  } else if constexpr (MODE == NS_APPLY) {
    store_tile<G>(acc, lds, ti, tj, p.unscale * p.scale, ws + M.ws_xn, M.np, ws + (p.a ? M.ws_xt : M.ws_xt2), M.mp, M.np, M.mp, wave);
  } else {
    const Origin<G> at(ti, tj, wave);
    const Out dst{out, v16, p.update, p.eta, p.decay, M.gain};
    if (M.tall) {
#pragma unroll
      for (int e = 0; e < 4 * TG::TR; ++e)
#pragma unroll
        for (int j0 = 0; j0 < TG::TC; j0 += TG::VJ) {
          float x[TG::VJ];
#pragma unroll
          for (int k = 0; k < TG::VJ; ++k) x[k] = acc_at<G>(acc, e, j0 + k) * p.unscale;
          if (at.i + e < M.n)
            emit<DT, TG::VJ>(dst, M.off + (long long)(at.i + e) * M.m + at.j + j0, x, M.m - at.j - j0);
        }
    } else {
#pragma unroll
      for (int jj = 0; jj < TG::TC; ++jj)
#pragma unroll
        for (int e = 0; e < 4 * TG::TR; e += 4) {
          float x[4];
#pragma unroll
          for (int d = 0; d < 4; ++d) x[d] = acc_at<G>(acc, e + d, jj) * p.unscale;
          if (at.j + jj < M.m)
            emit<DT, 4>(dst, M.off + (long long)(at.j + jj) * M.n + at.i + e, x, M.n - at.i - e);
        }
    }
  }
}

// H = sum of the slices' Gram matrices: a workgroup takes what one wave of the product
// had, its W waves every W-th slice each, and their sums are added in wave order.  (With
// a workgroup a tile that went through all slices 65536 x 256, three tiles of 64 slices,
// took 73 us, so 17.)  W: as many as the call's most slices, up to kSumWaves; a matrix of
// fewer has a wave a slice whatever W is.
template <int TB> constexpr int kSumWaves = TB == 256 ? 4 : 8;
template <int TB> constexpr int sum_lds(int waves) {  // the other waves' sums, or the rows to be stored
  using TG = TileGeo<Tile<TB>>;
  const int sets = (waves - 1) * TG::TR * TG::TC * 1024, rows = 16 * TG::OROW;
  return sets > rows ? sets : rows;
}
template <int TB>
__global__ __launch_bounds__(64 * kSumWaves<TB>) void ns_gram_sum_kernel(NsTable T, int slot, float scale, char *ws) {
  using G = Tile<TB>;
  using TG = TileGeo<G>;
  constexpr int N = TG::TR * TG::TC, PARTS = G::WR * G::WC;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int W = blockDim.x >> 6;
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int tm = (M.mp + TB - 1) / TB, tri = tm * (tm + 1) / 2, b = (blockIdx.x - T.first[l]) / PARTS;
  const int part = (blockIdx.x - T.first[l]) % PARTS, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int ti, tj;
  triangle_tile(b, tm, &ti, &tj);
  const f32x4_t *src = (const f32x4_t *)(ws + M.ws_part) + (long long)b * (TB * TB / 4) + part * N * 64 + lane;
  TileAcc<G> acc;
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i / TG::TC][i % TG::TC] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int n = wave; n < M.slices; n += W) {
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i / TG::TC][i % TG::TC] += src[(long long)n * tri * (TB * TB / 4) + i * 64];
  }
  f32x4_t *sets = reinterpret_cast<f32x4_t *>(lds);
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) sets[((wave - 1) * N + i) * 64 + lane] = acc[i / TG::TC][i % TG::TC];
  }
  __syncthreads();
  if (wave > 0) return;
  for (int o = 0; o < min(W, M.slices) - 1; ++o) {
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i / TG::TC][i % TG::TC] += sets[(o * N + i) * 64 + lane];
  }
  char *o = ws + M.ws_sq + (long long)M.mp * M.mp * 4 * slot;
  store_tile<G>(acc, lds, ti, tj, scale, o, M.mp, ti != tj ? o : nullptr, M.mp, M.mp, M.mp, part);
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

namespace {
double most(double x, double y) { return x > y ? x : y; }

// The largest |f(h)| for 0 <= h <= top, f a polynomial whose derivative is a multiple of
// d2 h^2 + d1 h + d0: at an end or at one of its roots.
template <class F> double largest(double top, double d2, double d1, double d0, F f) {
  double r = most(fabs(f(0.0)), fabs(f(top)));
  auto at = [&](double h) {
    if (h > 0.0 && h < top) r = most(fabs(f(h)), r);
  };
  if (d2 == 0.0) {
    if (d1 != 0.0) at(-d0 / d1);
  } else if (const double disc = d1 * d1 - 4.0 * d2 * d0; disc >= 0.0) {
    const double t = -0.5 * (d1 + copysign(sqrt(disc), d1));
    at(t / d2);
    if (t != 0.0) at(d0 / t);
  }
  return r;
}
}  // namespace

// The polynomial's largest values are where its derivatives vanish, not at sampled points: a
// range narrower than their distance could grow unseen from pair to pair of steps.
bool ns_scales(double a, double b, double c, int steps, NsSteps *S) {
  S->a = a;
  S->b = b;
  S->c = c;
  S->stages = (steps + 1) / 2;
  // (what stays below 1024 on [0, 1] has coefficients of at most 8 times that)
  if (!(fabs(a) <= 8192.0 && fabs(b) <= 8192.0 && fabs(c) <= 8192.0)) return false;
  // the largest power of two that keeps values up to `bound` and twice that below 2^16
  auto scale = [](double bound) {
    int e = 0;
    (void)frexp(32768.0 / (1.05 * (bound > 0.125 ? bound : 0.125)), &e);
    return (float)ldexp(1.0, e - 1 < 14 ? e - 1 : 14);
  };
  auto q = [=](double h) { return a + b * h + c * h * h; };
  // of |q(s^2)|, |s^2 q(s^2)| and |s q(s^2)| for singular values s up to x
  auto most_q = [&](double x) { return largest(x * x, 0.0, 2.0 * c, b, q); };
  auto most_qh = [&](double x) { return largest(x * x, 3.0 * c, 2.0 * b, a, [&](double h) { return h * q(h); }); };
  auto most_step = [&](double x) { return largest(x * x, 5.0 * c, 3.0 * b, a, [&](double h) { return sqrt(h) * q(h); }); };
  // A singular value may be larger than its bound by the roundings of the norm and of a pair
  // of steps; a polynomial that multiplies that from step to step is refused.
  constexpr double kRound = 1.0 + 1.0 / 65536.0;
  double sigma = kRound;  // bound of the singular values
  for (int s = 0; s < S->stages; ++s) {
    NsStage &G = S->stage[s];
    G = NsStage{};
    G.steps = 2 * s + 1 < steps ? 2 : 1;
    G.sx = scale(sigma);
    // the first step's values are all from 0 to `step`, the second's bounds those over them
    const double step = most_step(sigma);
    const double hb[2] = {sigma * sigma, step * step};
    const double qb[2] = {most_q(sigma), G.steps == 2 ? most_q(step) : 1.0};
    const double tb = most_qh(sigma), pb = qb[0] * qb[1], next = G.steps == 2 ? most_step(step) : step;
    if (!(qb[0] < 1024.0 && qb[1] < 1024.0 && pb < 16384.0 && tb < 1024.0 && hb[1] < 1024.0 && next < 32.0)) return false;
    for (int k = 0; k < 2; ++k) {
      G.sh[k] = scale(hb[k]);
      G.sq[k] = scale(qb[k]);
    }
    G.st = scale(tb);
    G.sp = scale(pb);
    sigma = most(next, 0.125) * kRound;
  }
  return true;
}

namespace {
// Time of a product of `tiles` tiles over `ksteps` k-steps, in us: rounds of a tile a
// compute unit, each a launch's and tile's fixed share and its k-steps, which take 1.4
// times as long on a full machine as on an empty one.  Measured on square matrices (tiles
// of the triangle; m x m products of 32 / 64 / 128 / 192 / 256 in us): 256 5.6 / 6.1 / 9.5,
// 512 6.1 / 8.2 / 13 / 26 / 34, 640 7.2 / 8.8 / 15, 768 12.6 / 9.6 / 17, 1024 22 / 11.8 / 19 /
// 39 / 56, 1536 45 / 31 / 29 / 53 / 81, 2048 - / 62 / 39 / 69 / 106, 3200 - / - / 123 / 113 /
// 170, 4096 - / - / 242 / 173 / 230.
struct TileCost {
  int tile;
  double fixed, step;
};
constexpr TileCost kTileCost[] = {{32, 4.7, 0.095}, {64, 4.5, 0.225}, {128, 6.5, 0.42}, {192, 11.5, 0.94}, {256, 21.5, 1.45}};
double tile_time(const TileCost &c, long long tiles, long long ksteps) {
  const long long full = tiles / kNumCUs, rest = tiles % kNumCUs;
  double t = full * (c.fixed + 1.4 * c.step * ksteps);
  if (rest) t += c.fixed + (1.0 + 0.4 * rest / kNumCUs) * c.step * ksteps;
  return t;
}
}  // namespace

size_t ns_plan(int count, const long long *off, const int *rows, const int *cols, int dtype, bool momentum, NsTable *T) {
  long long at = 0;
  auto take = [&](long long bytes) {
    const long long p = at;
    at += up(bytes, 256);
    return p;
  };
  T->count = count;
  T->wholes = 0;
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
      // One workgroup runs what takes it no longer than the large matrices' Gram launch,
      // beside which it runs: 512 x 16 and 256 x 32 24 us, 64 x 64 23 (1024 x 32 66, 256 x 64 32;
      // the other kernels' launches take about 35 for any small matrix).
      M.whole = (long long)M.n * mt <= (mt <= 32 ? 8192 : 4096) && mt <= 64;
      if (M.whole) T->whole[T->wholes++] = l;
      // chunks of about 8192 elements, at most 512
      M.prow = (int)up(8192 / mt, 64);
      while (((long long)M.n + M.prow - 1) / M.prow > 512) M.prow *= 2;
      M.chunks = (M.n + M.prow - 1) / M.prow;
      // Workgroups of the long side: 256 rows at a time (128 of 128 columns), on at most
      // two thirds of the compute units so that a call's other matrices run beside: on all
      // of them 65536 x 128 takes 133 us instead of 150, but the 128^3 network's update 241
      // instead of 197.
      const long long wgs = ((long long)M.n + (mt == 128 ? 127 : 255)) / (mt == 128 ? 128 : 256);
      M.slices = (int)(wgs < kNsSlices ? wgs : kNsSlices);
      const int tt = mt / 16;
      const bool direct = !momentum && dtype == DT_F32 && M.tall && M.m == mt;
      M.ws_norm = take(8LL * M.chunks);
      const long long x = take(4LL * M.n * mt);
      M.ws_u = direct ? -1 : x;
      M.ws_xn = x;
      M.ws_part = take(1024LL * (tt * (tt + 1) / 2) * M.slices);
      M.ws_part2 = M.slices > kNsFewSlices ? M.ws_part : take(1024LL * (tt * (tt + 1) / 2) * M.slices);
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
    double best_sq = 1e30, best_long = 1e30, best_gram = 1e30;
    const long long ksteps = M.np / kStep;
    for (const TileCost &c : kTileCost) {
      const double sq = tile_time(c, triangle(c.tile), M.mp / kStep);
      if (sq < best_sq) best_sq = sq, M.tile_sq = c.tile;
      const double lng = tile_time(c, tiles(M.mp, c.tile) * tiles(M.np, c.tile), M.mp / kStep);
      if (lng < best_long) best_long = lng, M.tile_long = c.tile;
      // the Gram product also in slices of the long side, whose sums another launch adds (4 us,
      // 8 TB/s, and 1.2 us for a turn of its waves: 64 slices of 3 tiles of 128 17 us, 25 of 10
      // 10.8).  It reads rows of the long side, whose offsets from the tile's first have 32 bits
      // (a tile of 64 fits at any length, one of 256 up to 4.2 million).
      if ((std::min<long long>(c.tile, M.mp) - 1) * 4 * M.np + 128 > 1LL << 32) continue;
      for (long long s = 1; s <= 64 && (s == 1 || s * 8 <= ksteps); ++s) {
        const double bytes = 8.0 * s * triangle(c.tile) * c.tile * c.tile;  // written and read
        const double gram = tile_time(c, triangle(c.tile) * s, (ksteps + s - 1) / s) + (s > 1 ? 4.0 + bytes / 8e6 + 1.2 * ((s + 7) / 8) : 0.0);
        if (gram < best_gram) best_gram = gram, M.tile_gram = c.tile, M.slices = (int)s;
      }
    }
    M.ws_part = M.slices > 1 ? take(4LL * triangle(M.tile_gram) * M.tile_gram * M.tile_gram * M.slices) : 0;
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
  auto each_tile = [&](int NsMat::*side, auto f) {
    auto used = [&](int tb) {
      for (int l = 0; l < T.count; ++l)
        if (!T.mat[l].mt && T.mat[l].*side == tb) return true;
      return false;
    };
    if (used(256)) f(std::integral_constant<int, 256>{});
    if (used(192)) f(std::integral_constant<int, 192>{});
    if (used(128)) f(std::integral_constant<int, 128>{});
    if (used(64)) f(std::integral_constant<int, 64>{});
    if (used(32)) f(std::integral_constant<int, 32>{});
  };
  auto product = [&](auto mode, auto dt, NsProduct p) {
    constexpr int MODE = decltype(mode)::value, DT = decltype(dt)::value;
    constexpr bool kLong = MODE == NS_APPLY || MODE == NS_FINAL;
    constexpr int NsMat::*side = kLong ? &NsMat::tile_long : MODE == NS_GRAM ? &NsMat::tile_gram : &NsMat::tile_sq;
    each_tile(side, [&](auto tile) {
      constexpr int TB = decltype(tile)::value;
      const int blocks = number(&T, [=](const NsMat &M) {
        if (M.*side != TB) return 0LL;
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
    square(Gram{}, 0, 0, SQ_H, 1.f / (G.sx * G.sx), 0.f, G.sh[0]);
    each_tile(&NsMat::tile_gram, [&](auto tile) {
      constexpr int TB = decltype(tile)::value;
      nb = number(&T, [](const NsMat &M) {
        const long long t = (M.mp + TB - 1) / TB;
        return M.tile_gram == TB && M.slices > 1 ? t * (t + 1) / 2 * (Tile<TB>::WR * Tile<TB>::WC) : 0LL;
      });
      int waves = 0;
      for (int l = 0; l < T.count; ++l)
        if (!T.mat[l].mt && T.mat[l].tile_gram == TB) waves = max(waves, min(T.mat[l].slices, kSumWaves<TB>));
      if (nb)
        hipLaunchKernelGGL((ns_gram_sum_kernel<TB>), dim3(nb), dim3(64 * waves), sum_lds<TB>(waves), st, T, (int)SQ_H,
                           G.sh[0] / (G.sx * G.sx), ws);
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
