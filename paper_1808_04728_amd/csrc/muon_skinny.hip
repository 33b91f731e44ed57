// muon_skinny.hip -- the Newton-Schulz products (see muon.hip) of matrices whose
// shorter side m is at most 128: every weight matrix of the network.
//
// The long side is touched once a pair of steps.  A wave takes 32 of its rows at a
// time from memory to registers, multiplies them by P and adds their share of the
// next Gram matrix without leaving the registers:
//   D = X P     the result of a matrix instruction has a column of D in a lane and
//               four rows of it in the lane's registers;
//   H += D' D   reads, for both factors, a lane with a column and eight rows: two
//               results of the first product as they are.  Which rows these are does
//               not matter as long as both factors agree.
// The Gram matrix's upper tiles stay in accumulators; a workgroup's four waves add
// theirs through LDS, the workgroups' sums are added in a fixed order.
//
// The m x m polynomials run at the start of every launch that applies them, in each of
// its workgroups.  Their waves own columns: for a symmetric M and any product C = M B, a
// wave's columns of B are its own, so a chain of products needs only M in LDS and no
// exchange between them.  That repeats the work (128 columns: 63 million operations, 13 us
// at the matrix rate), but one workgroup's launch for it takes as long and its way through
// memory longer: the 128^3 network's update took 220 us so and takes 177 to 197 on several cards.
//
// What bounds it, 65536 x 128 (144 to 150 us of five steps on several cards): the norm's pass 9 us and the first
// Gram matrix 12 at memory's rate; two products with their Gram matrices 46 each, 28 of
// them the polynomial; the last product 25; the sums between them 5 each.
//
// Columns are handled in slots: slot 16 (4 u + c) + r is column 64 u + 4 r + c, so that
// a lane's four tiles c hold four consecutive columns and rows load and store in
// 16-byte vectors.  The polynomials do not care; P is written with rows in slot order
// and columns in their own, which is how the product with X reads it.
//
// Up to 32 columns factors are fp32 (the fp32 matrix rate covers them), above they
// are fp16 pairs as in muon.hip.

#include <utility>

#include "muon_common.h"

namespace cf {
namespace {

template <int MT> struct Geo {
  static constexpr int TT = MT / 16;              // 16-column tiles
  static constexpr int VW = TT < 4 ? TT : 4;      // columns of a vector
  static constexpr int U = TT / VW;               // 64-column groups
  static constexpr int KB = (TT + 1) / 2;         // 32-deep products over the columns
  static constexpr bool F32 = MT <= 32;           // factor format
  static constexpr int TRI = TT * (TT + 1) / 2;   // tiles of the upper triangle
  static constexpr int LROW = KB * 128 + 16;      // bytes of a matrix row in LDS
  static constexpr int MAT = MT * LROW;           // bytes of a matrix in LDS
  static constexpr int SET = TRI * 1024;          // bytes of a Gram matrix's tiles
};

// eight values of a factor, k = (g, 0..7) of a 32-deep product
template <bool F32> struct Frag;
template <> struct Frag<true> {
  float v[8];
};
template <> struct Frag<false> {
  f16x8_t hi, lo;
};

template <bool F32> __device__ __forceinline__ Frag<F32> make_frag(const float (&x)[8]) {
  Frag<F32> f;
  if constexpr (F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = x[j];
  } else {
    ns_split8(x, f.hi, f.lo);
  }
  return f;
}

// acc += A B over the 32 k of the fragments
template <bool F32> __device__ __forceinline__ void mma(f32x4_t &acc, const Frag<F32> &a, const Frag<F32> &b) {
  if constexpr (F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], acc, 0, 0, 0);
  } else {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.hi, b.lo, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.lo, b.hi, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.hi, b.hi, acc, 0, 0, 0);
  }
}

// a fragment is 32 bytes in memory: eight floats, or eight hi then eight lo
template <bool F32> __device__ __forceinline__ Frag<F32> load_frag(const char *p) {
  Frag<F32> f;
  const u32x4_t a = *reinterpret_cast<const u32x4_t *>(p), b = *reinterpret_cast<const u32x4_t *>(p + 16);
  if constexpr (F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f.v[j] = __uint_as_float(a[j]);
      f.v[4 + j] = __uint_as_float(b[j]);
    }
  } else {
    f.hi = __builtin_bit_cast(f16x8_t, a);
    f.lo = __builtin_bit_cast(f16x8_t, b);
  }
  return f;
}

template <bool F32> __device__ __forceinline__ void store_frag(char *p, const Frag<F32> &f) {
  if constexpr (F32) {
    *reinterpret_cast<float4 *>(p) = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
    *reinterpret_cast<float4 *>(p + 16) = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
  } else {
    *reinterpret_cast<f16x8_t *>(p) = f.hi;
    *reinterpret_cast<f16x8_t *>(p + 16) = f.lo;
  }
}

// elements j .. j + N - 1 of the fragment at p (j a multiple of N)
template <bool F32, int N> __device__ __forceinline__ void store_elements(char *p, int j, const float (&x)[N]) {
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<float *>(p + 4 * j)[i] = x[i];
  } else {
    typedef _Float16 vec_t __attribute__((ext_vector_type(N)));
    vec_t hi, lo;
    if constexpr (N == 1) {
      const Half2 s = ns_split(x[0]);
      hi[0] = s.hi;
      lo[0] = s.lo;
    } else {
      ns_split_pairs<N>(x, hi, lo);
    }
    *reinterpret_cast<vec_t *>(p + 2 * j) = hi;
    *reinterpret_cast<vec_t *>(p + 16 + 2 * j) = lo;
  }
}

// four elements from j on of the fragment at p
template <bool F32> __device__ __forceinline__ void load_elements(const char *p, int j, float (&x)[4]) {
  if constexpr (F32) {
    load_cols<4>(reinterpret_cast<const float *>(p + 4 * j), x);
  } else {
    const f16x4_t hi = *reinterpret_cast<const f16x4_t *>(p + 2 * j), lo = *reinterpret_cast<const f16x4_t *>(p + 16 + 2 * j);
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = (float)hi[q] + (float)lo[q];
  }
}

// ---- Gram matrix of 32 rows ----------------------------------------------------

template <int MT> struct Acc {
  f32x4_t t[Geo<MT>::TRI];
};

template <int MT> __device__ __forceinline__ void gram_add(Acc<MT> &acc, const Frag<Geo<MT>::F32> (&f)[Geo<MT>::TT]) {
  constexpr int TT = Geo<MT>::TT;
  int k = 0;
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = i; j < TT; ++j) mma<Geo<MT>::F32>(acc.t[k++], f[i], f[j]);
}

// Rows n0 .. n0 + 31 of X [n][MT] as the Gram product's factors: a lane has rows
// 8 g .. 8 g + 7 of its columns.
template <int MT> struct GramRows {
  using G = Geo<MT>;
  float v[8][G::U][G::VW];
  __device__ __forceinline__ void load(const float *X, int n, int n0) {
    const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < G::U; ++u)
        load_cols<G::VW>(X + (long long)min(n0 + 8 * g + j, n - 1) * MT + 64 * u + G::VW * r, v[j][u]);
  }
  __device__ __forceinline__ void factors(Frag<G::F32> (&f)[G::TT], int n, int n0, const Scale &sc) {
    const int g = (threadIdx.x & 63) >> 4;
    if (sc.s1 != 1.f) each([&](float &x, int) { x *= sc.s1; });
    if (n0 + 32 > n) each([&](float &x, int j) { x = n0 + 8 * g + j < n ? x : 0.f; });
#pragma unroll
    for (int t = 0; t < G::TT; ++t) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = v[j][t / G::VW][t % G::VW] * sc.s2;
      f[t] = make_frag<G::F32>(x);
    }
  }
  template <class F> __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int u = 0; u < G::U; ++u)
#pragma unroll
        for (int c = 0; c < G::VW; ++c) f(v[j][u][c], j);
  }
};

// The sum of SETS Gram matrices in LDS, tile by tile, in order, to out [TRI][64 lanes][4]
template <int MT, int SETS> __device__ __forceinline__ void gram_sum(const char *lds, float unscale, float *out) {
  constexpr int N = Geo<MT>::TRI * 64;
  const float4 *red = reinterpret_cast<const float4 *>(lds);
  __syncthreads();
  for (int i = threadIdx.x; i < N; i += blockDim.x) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < SETS; ++k) {
      const float4 a = red[k * N + i];
      s += f32x4_t{a.x, a.y, a.z, a.w};
    }
    reinterpret_cast<float4 *>(out)[i] = make_float4(s[0] * unscale, s[1] * unscale, s[2] * unscale, s[3] * unscale);
  }
}

// the waves' accumulators added in wave order
template <int MT, int WAVES> __device__ __forceinline__ void gram_out(const Acc<MT> &acc, char *lds, float unscale, float *out) {
  using G = Geo<MT>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();  // whatever the LDS held has been read
#pragma unroll
  for (int t = 0; t < G::TRI; ++t)
    reinterpret_cast<float4 *>(lds)[(wave * G::TRI + t) * 64 + lane] =
        make_float4(acc.t[t][0], acc.t[t][1], acc.t[t][2], acc.t[t][3]);
  gram_sum<MT, WAVES>(lds, unscale, out);
}

// ---- X P of 32 rows ------------------------------------------------------------

// Rows n0 .. n0 + 31 of X as the left factors of X P: a lane has row 16 s + r, columns
// 32 kb + 8 g .. + 7.  (16 columns fill half a product: lanes g >= 2 are zero.)
template <int MT> struct ApplyRows {
  using G = Geo<MT>;
  float v[2][G::KB][8];
  __device__ __forceinline__ void load(const float *X, int n, int n0) {
    const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float *p = X + (long long)min(n0 + 16 * s + r, n - 1) * MT + (MT >= 32 ? 8 * g : 8 * (g & 1));
#pragma unroll
      for (int kb = 0; kb < G::KB; ++kb) {
        float a[4], b[4];
        load_cols<4>(p + 32 * kb, a);
        load_cols<4>(p + 32 * kb + 4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[s][kb][j] = a[j];
          v[s][kb][4 + j] = b[j];
        }
      }
    }
  }
  __device__ __forceinline__ void factors(Frag<G::F32> (&a)[2][G::KB], int n, int n0, const Scale &sc) {
    const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    if (sc.on) {
      if (sc.s1 != 1.f) each([&](float &x, int) { x *= sc.s1; });
      each([&](float &x, int) { x *= sc.s2; });
    }
    if (n0 + 32 > n || MT < 32) each([&](float &x, int s) { x = n0 + 16 * s + r < n && (MT >= 32 || g < 2) ? x : 0.f; });
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int kb = 0; kb < G::KB; ++kb) a[s][kb] = make_frag<G::F32>(v[s][kb]);
  }
  template <class F> __device__ __forceinline__ void each(F f) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int kb = 0; kb < G::KB; ++kb)
#pragma unroll
        for (int j = 0; j < 8; ++j) f(v[s][kb][j], s);
  }
};

// d[s][t] = rows 16 s + 4 g + 0..3 of slot 16 t + r of X P, P in LDS from its first of
// N tiles on
template <int MT, int N>
__device__ __forceinline__ void apply_product(f32x4_t (&d)[2][N], const Frag<Geo<MT>::F32> (&a)[2][Geo<MT>::KB], const char *P) {
  using G = Geo<MT>;
  const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int t = 0; t < N; ++t) d[s][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kb = 0; kb < G::KB; ++kb) {
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const Frag<G::F32> b = load_frag<G::F32>(P + (16 * t + r) * G::LROW + kb * 128 + g * 32);
#pragma unroll
      for (int s = 0; s < 2; ++s) mma<G::F32>(d[s][t], a[s][kb], b);
    }
    // (without this the loads of all of P move to the front and the registers spill)
    if (G::KB > 1) __builtin_amdgcn_sched_barrier(0);
  }
}

// d scaled, and as Gram factors
template <int MT, int N>
__device__ __forceinline__ void scale_rows(f32x4_t (&d)[2][N], Frag<Geo<MT>::F32> (&f)[N], float unscale) {
  using G = Geo<MT>;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      d[j >> 2][t][j & 3] *= unscale;
      v[j] = d[j >> 2][t][j & 3];
    }
    f[t] = make_frag<G::F32>(v);
  }
}

// d as rows n0 .. n0 + 31 of X, groups of VW tiles from column col0 on
template <int MT, int N>
__device__ __forceinline__ void store_rows(const f32x4_t (&d)[2][N], float *X, int n, int n0, int col0) {
  using G = Geo<MT>;
  const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = n0 + 16 * s + 4 * g + q;
      if (row < n) {
#pragma unroll
        for (int u = 0; u < N / G::VW; ++u) {
          float v[G::VW];
#pragma unroll
          for (int c = 0; c < G::VW; ++c) v[c] = d[s][u * G::VW + c][q];
          store_cols<G::VW>(X + (long long)row * MT + col0 + 64 * u + G::VW * r, v);
        }
      }
    }
}

// X <- X P for the waves' rows, in place or from another buffer, and their Gram matrix.
// `x` holds the wave's first rows (asked for before P was); the next are asked for as
// soon as these are factors.
template <int MT>
__device__ __forceinline__ void apply_gram_steps(Acc<MT> &acc, ApplyRows<MT> &x, const float *src, float *dst, int n, int first,
                                                 int stride, const Scale &sc, float unscale, const char *P) {
  using G = Geo<MT>;
  for (int n0 = first * 32; n0 < n; n0 += stride * 32) {
    f32x4_t d[2][G::TT];
    Frag<G::F32> a[2][G::KB], f[G::TT];
    x.factors(a, n, n0, sc);
    if (n0 + stride * 32 < n) x.load(src, n, n0 + stride * 32);
    apply_product<MT, G::TT>(d, a, P);
    scale_rows<MT, G::TT>(d, f, unscale);
    store_rows<MT, G::TT>(d, dst, n, n0, 0);
    gram_add<MT>(acc, f);
  }
}

// The same of 128 columns by pairs of waves: all 36 Gram tiles and the factors fill one
// wave's registers and leave a SIMD one wave.  Two waves have the same rows; each
// multiplies them by half of P, hands its columns' factors to the other through LDS, and
// adds 18 tiles.  Then two waves share a SIMD and cover each other's waits: 4.5 us for a
// turn of four pairs, of which the matrix instructions are 2.8.
struct PairAcc {
  f32x4_t own[10], cross[8];  // tiles inside the wave's half, tiles of both
};
constexpr int kPairs = 4;
constexpr int kPairLds = kPairs * 2 * 4 * 64 * 32;  // bytes: every wave's four factors

__device__ __forceinline__ void apply_gram_pairs(PairAcc &acc, ApplyRows<128> &x, const float *src, float *dst, int n, int b,
                                                 int slices, const Scale &sc, float unscale, const char *P, char *swap) {
  using G = Geo<128>;
  using F = Frag<false>;
  const int lane = threadIdx.x & 63, pair = threadIdx.x >> 6 & 3, h = threadIdx.x >> 8;
  char *mine = swap + (pair * 2 + h) * 4 * 2048 + lane * 32, *other = swap + (pair * 2 + 1 - h) * 4 * 2048 + lane * 32;
  for (int base = b * kPairs; base * 32 < n; base += slices * kPairs) {  // (the same turns for every wave)
    const int n0 = (base + pair) * 32;
    F a[2][G::KB], f[4], o[4];
    f32x4_t d[2][4];
    x.factors(a, n, n0, sc);
    apply_product<128, 4>(d, a, P + h * 64 * G::LROW);
    if ((base + slices * kPairs) * 32 < n) x.load(src, n, n0 + slices * kPairs * 32);
    scale_rows<128, 4>(d, f, unscale);
#pragma unroll
    for (int t = 0; t < 4; ++t) store_frag<false>(mine + t * 2048, f[t]);
    __syncthreads();
    // (not before: in place, the other wave has read the rows by now)
    store_rows<128, 4>(d, dst, n, n0, 64 * h);
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = load_frag<false>(other + t * 2048);
    int k = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = i; j < 4; ++j) mma<false>(acc.own[k++], f[i], f[j]);
    // tiles (i, 4 + j): the first wave i = 0, 1, the second i = 2, 3
    if (h == 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mma<false>(acc.cross[4 * i + j], f[i], o[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mma<false>(acc.cross[4 * i + j], o[2 + i], f[j]);
    }
    __syncthreads();  // both have read before the next factors are written
  }
}

// the pairs' tiles to their places, added in pair order
__device__ __forceinline__ void pairs_out(const PairAcc &acc, char *lds, float unscale, float *out) {
  using G = Geo<128>;
  const int lane = threadIdx.x & 63, pair = threadIdx.x >> 6 & 3, h = threadIdx.x >> 8;
  float4 *red = reinterpret_cast<float4 *>(lds) + pair * G::TRI * 64 + lane;
  auto put = [&](int i, int j, const f32x4_t &v) {  // tile (i, j) of the upper triangle
    red[(i * G::TT - i * (i - 1) / 2 + j - i) * 64] = make_float4(v[0], v[1], v[2], v[3]);
  };
  __syncthreads();  // P has been read
  int k = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = i; j < 4; ++j) put(4 * h + i, 4 * h + j, acc.own[k++]);
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) put(2 * h + i, 4 + j, acc.cross[4 * i + j]);
  gram_sum<128, kPairs>(lds, unscale, out);
}

template <int MT, int DT>
__device__ __forceinline__ void final_steps(const NsMat &M, const Out &o, ApplyRows<MT> &x, const float *src, int first,
                                            int stride, const Scale &sc, float unscale, const char *P) {
  using G = Geo<MT>;
  const int r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  for (int n0 = first * 32; n0 < M.n; n0 += stride * 32) {
    f32x4_t d[2][G::TT];
    Frag<G::F32> a[2][G::KB];
    x.factors(a, M.n, n0, sc);
    apply_product<MT, G::TT>(d, a, P);
    if (n0 + stride * 32 < M.n) x.load(src, M.n, n0 + stride * 32);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int u = 0; u < G::U; ++u) {
        const int row = n0 + 16 * s + 4 * g, col = 64 * u + G::VW * r;
        if (M.tall) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float v[G::VW];
#pragma unroll
            for (int c = 0; c < G::VW; ++c) v[c] = d[s][u * G::VW + c][q] * unscale;
            if (row + q < M.n)
              emit<DT, G::VW>(o, M.off + (long long)(row + q) * M.m + col, v, M.m - col);
          }
        } else {
#pragma unroll
          for (int c = 0; c < G::VW; ++c) {
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = d[s][u * G::VW + c][q] * unscale;
            if (col + c < M.m) emit<DT, 4>(o, M.off + (long long)(col + c) * M.n + row, v, M.n - row);
          }
        }
      }
  }
}

// ---- the m x m polynomials --------------------------------------------------------

// P of one or two steps from the Gram matrix (upper tiles, the sum of `parts` arrays
// in order), rows in slot order, to dst in LDS (lds itself or apart from it), by NW waves.
// lds: two matrices.  A wave has NC tile columns, and with eight waves half of
// their rows.
template <int MT, int NW>
__device__ __forceinline__ void polynomial(const float *gram, int parts, const NsStage &st, float ca, float cb, float cc,
                                           char *lds, char *dst) {
  using G = Geo<MT>;
  constexpr bool F = G::F32;
  constexpr int NC = G::TT > 4 ? G::TT / 4 : 1, RH = NW == 8 && G::TT > 1 ? 2 : 1, RT = G::TT / RH;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const float sh0 = F ? 1.f : st.sh[0], sq0 = F ? 1.f : st.sq[0], sh1 = F ? 1.f : st.sh[1], sq1 = F ? 1.f : st.sq[1];
  const float stt = F ? 1.f : st.st, sp = F ? 1.f : st.sp;
  char *H = lds, *Q = lds + G::MAT;
  {
    constexpr int N = (G::TRI + NW - 1) / NW;  // tiles of a wave
    const int w = __builtin_amdgcn_readfirstlane(wave);
    float4 s[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (w + NW * k < G::TRI) s[k] = reinterpret_cast<const float4 *>(gram)[(w + NW * k) * 64 + lane];
    for (int p = 1; p < parts; ++p) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (w + NW * k < G::TRI) {
          const float4 a = reinterpret_cast<const float4 *>(gram)[((long long)p * G::TRI + w + NW * k) * 64 + lane];
          s[k].x += a.x; s[k].y += a.y; s[k].z += a.z; s[k].w += a.w;
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (w + NW * k >= G::TRI) continue;
      int tj = w + NW * k, ti = 0;
      while (tj >= G::TT - ti) {
        tj -= G::TT - ti;
        ++ti;
      }
      tj += ti;
      // elements (16 ti + 4 g + q, 16 tj + r): as row 16 tj + r, and mirrored
      const float x[4] = {s[k].x * sh0, s[k].y * sh0, s[k].z * sh0, s[k].w * sh0};
      char *row = H + (16 * tj + r) * G::LROW + (ti >> 1) * 128 + g * 32;
      char *col = H + (16 * ti + 4 * g) * G::LROW + (tj >> 1) * 128 + (r >> 2) * 32;
      const int jc = 4 * (tj & 1) + (r & 3);
      if constexpr (F) {
        store_elements<F, 4>(row, 4 * (ti & 1), x);
        if (ti != tj) {
#pragma unroll
          for (int q = 0; q < 4; ++q) store_elements<F, 1>(col + q * G::LROW, jc, {x[q]});
        }
      } else {
        f16x4_t hi, lo;
        ns_split_pairs<4>(x, hi, lo);
        *reinterpret_cast<f16x4_t *>(row + 8 * (ti & 1)) = hi;
        *reinterpret_cast<f16x4_t *>(row + 16 + 8 * (ti & 1)) = lo;
        if (ti != tj) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            *reinterpret_cast<_Float16 *>(col + q * G::LROW + 2 * jc) = hi[q];
            *reinterpret_cast<_Float16 *>(col + q * G::LROW + 16 + 2 * jc) = lo[q];
          }
        }
      }
      if (G::TT == 1) {  // 16 columns are half a product's depth
        store_elements<F, 4>(H + r * G::LROW + g * 32, 4, {0.f, 0.f, 0.f, 0.f});
        store_elements<F, 4>(Q + r * G::LROW + g * 32, 4, {0.f, 0.f, 0.f, 0.f});
      }
    }
  }
  const int t0 = wave / 4 * RT;                            // the wave's first tile row
  const bool active = (wave & 3) * NC < G::TT && t0 < G::TT;
  const int mine = (16 * (wave & 3) * NC + r) * G::LROW + g * 32;  // its first column, as a row
  f32x4_t d[NC][RT];  // element (16 (t0 + t) + 4 g + q, own column c)
  auto product = [&](const char *A, const char *B) {  // d = A B, B's columns as its rows
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < RT; ++t) d[c][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < G::KB; ++kb) {
      Frag<F> b[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) b[c] = load_frag<F>(B + mine + 16 * c * G::LROW + kb * 128);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const Frag<F> a = load_frag<F>(A + (16 * (t0 + t) + r) * G::LROW + kb * 128 + g * 32);
#pragma unroll
        for (int c = 0; c < NC; ++c) mma<F>(d[c][t], a, b[c]);
      }
    }
  };
  auto put = [&](char *A, float scale) {  // the wave's part of a symmetric matrix = d * scale
    if (!active) return;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < RT; ++t)
        store_elements<F, 4>(A + mine + 16 * c * G::LROW + ((t0 + t) >> 1) * 128, 4 * ((t0 + t) & 1),
                             {d[c][t][0] * scale, d[c][t][1] * scale, d[c][t][2] * scale, d[c][t][3] * scale});
  };
  auto poly = [&](float sh) {  // d = ca I + cb H + cc d, d the square of sh H
    const float uh = cb / sh, us = cc / (sh * sh);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float h[4];
        load_elements<F>(H + mine + 16 * c * G::LROW + ((t0 + t) >> 1) * 128, 4 * ((t0 + t) & 1), h);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x = uh * h[q] + us * d[c][t][q];
          if (t0 + t == (wave & 3) * NC + c && 4 * g + q == r) x += ca;
          d[c][t][q] = x;
        }
      }
  };
  // a matrix in LDS is overwritten only when every wave has read it
  float out = sq0;  // scale of d when P is written
  __syncthreads();
  if (active) {
    product(H, H);
    poly(sh0);
  }
  if (st.steps == 2) {
    put(Q, sq0);
    __syncthreads();
    if (active) product(Q, H);  // T = Q H
    __syncthreads();
    put(H, stt / (sq0 * sh0));
    __syncthreads();
    if (active) product(Q, H);  // H' = Q T
    __syncthreads();
    put(H, sh1 / (sq0 * stt));
    __syncthreads();
    if (active) {
      product(H, H);
      poly(sh1);
    }
    __syncthreads();
    put(H, sq1);
    __syncthreads();
    if (active) product(Q, H);  // P = Q Q'
    out = sp / (sq0 * sq1);
  }
  __syncthreads();  // (dst may be lds)
#pragma unroll
  for (int c = 0; c < NC && active; ++c) {
    char *row = dst + (16 * ((wave & 3) * NC + c) + r) * G::LROW;
#pragma unroll
    for (int t = 0; t < RT; t += RT < G::VW ? RT : G::VW)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // columns of the tiles t0 + t ..: consecutive within a group of VW tiles
        constexpr int W = RT < G::VW ? RT : G::VW;
        const int col = 64 * ((t0 + t) / G::VW) + G::VW * (4 * g + q) + (t0 + t) % G::VW;
        float v[W];
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = d[c][t + k][q] * out;
        store_elements<F, W>(row + col / 8 * 32, col % 8, v);
        if (G::TT == 1) store_elements<F, 1>(row + (16 + 4 * g) / 8 * 32, (4 * g + q) % 8, {0.f});
      }
  }
  __syncthreads();
}

// ---- kernels ----------------------------------------------------------------------

// CALL(MT) for the matrix's width mt, MT <= MAX
#define CF_NS_WIDTH(MAX, mt, CALL)                        \
  {                                                       \
    if (MAX >= 128 && (mt) == 128) CALL(128)              \
    else if (MAX >= 64 && (mt) == 64) CALL(64)            \
    else if ((mt) == 32) CALL(32)                         \
    else CALL(16)                                         \
  }

constexpr int most(int a, int b) { return a > b ? a : b; }

__device__ __forceinline__ const float *ns_source(const NsMat &M, const char *ws, const void *g) {
  return M.ws_u >= 0 ? (const float *)(ws + M.ws_u) : (const float *)g + M.off;
}

// Rows [r0, r1) of the long side: momentum, the update into u [n][mt] (zero padding
// columns) unless the matrix is read where it is, and the sum of its squares.
template <int DT, bool MOM>
__device__ __forceinline__ double prep_rows(const NsMat &M, const NsMomentum &mom, const void *g, float *m, float *u, int r0,
                                            int r1, float *tile) {
  using S = typename Store<DT>::T;
  const S *gp = (const S *)g + M.off;
  double s = 0.0;
  if (M.tall) {
    const long long beg = (long long)r0 * M.m, end = (long long)r1 * M.m;
    if (M.m == M.mt) {  // the layouts agree
      for (long long e = beg + 4 * threadIdx.x; e < end; e += 4 * 256) {
        float x[4];
        if constexpr (DT == DT_F32) {
          load_cols<4>((const float *)gp + e, x);
        } else {
          const uint2 a = *reinterpret_cast<const uint2 *>(gp + e);
          x[0] = __uint_as_float(a.x << 16);
          x[1] = __uint_as_float(a.x & 0xffff0000u);
          x[2] = __uint_as_float(a.y << 16);
          x[3] = __uint_as_float(a.y & 0xffff0000u);
        }
        if constexpr (MOM) {
          float mv[4];
          load_cols<4>(m + M.off + e, mv);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = ns_momentum(mom, x[i], mv[i]);
          store_cols<4>(m + M.off + e, mv);
        }
        if (M.ws_u >= 0) store_cols<4>(u + e, x);
        s += ((double)x[0] * x[0] + (double)x[1] * x[1]) + ((double)x[2] * x[2] + (double)x[3] * x[3]);
      }
    } else {
      for (long long k = (long long)r0 * M.mt + threadIdx.x; k < (long long)r1 * M.mt; k += 256) {
        const long long row = k / M.mt;
        const int col = (int)(k % M.mt);
        float x = 0.f;
        if (col < M.m) {
          const long long e = row * M.m + col;
          x = to_f32<DT>(gp[e]);
          if constexpr (MOM) x = ns_momentum(mom, x, m[M.off + e]);
        }
        u[k] = x;
        s += (double)x * x;
      }
    }
    return s;
  }
  // wide: 64 columns at a time through a tile, rows of u are columns of the matrix
  const int c = threadIdx.x & 63;
  for (int n0 = r0; n0 < r1; n0 += 64) {
    for (int i = threadIdx.x >> 6; i < M.mt; i += 4) {
      float x = 0.f;
      if (i < M.m && n0 + c < r1) {
        const long long e = (long long)i * M.n + n0 + c;
        x = to_f32<DT>(gp[e]);
        if constexpr (MOM) x = ns_momentum(mom, x, m[M.off + e]);
      }
      tile[i * 65 + c] = x;
      s += (double)x * x;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 64 * M.mt; k += 256) {
      const int row = k / M.mt, col = k % M.mt;
      if (n0 + row < r1) u[(long long)(n0 + row) * M.mt + col] = tile[col * 65 + row];
    }
    __syncthreads();
  }
  return s;
}

template <int DT, bool MOM>
__global__ __launch_bounds__(256) void skinny_prep_kernel(NsTable T, NsMomentum mom, const void *g, float *m, char *ws) {
  __shared__ double red[4];
  __shared__ float tile[128 * 65];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int chunk = blockIdx.x - T.first[l], r0 = chunk * M.prow, r1 = min(r0 + M.prow, M.n);
  const double s = ns_block_sum(prep_rows<DT, MOM>(M, mom, g, m, (float *)(ws + M.ws_u), r0, r1, tile), red);
  if (threadIdx.x == 0) ((double *)(ws + M.ws_norm))[chunk] = s;
}

// The whole iteration of a small matrix in one workgroup: what the other kernels do in
// eight launches of 2 to 4 us and 3 us of the host each (27 x 16: 23 us so, 9.7 here).
// Factors in fp32 take one step from each Gram matrix instead of two: the products are
// cheap, and the result is as exact as the plain iteration's in fp32 (7e-7 against 1.1e-6
// with pairs of steps).
template <int MAX> struct Whole {
  static constexpr int W = MAX < 64 ? MAX : 64;  // widest matrix
  using G = Geo<W>;
  static constexpr int TILE = W * 65 * 4;  // of prep_rows
  static constexpr int FRONT = most(4 * G::SET, TILE);
  static constexpr int BYTES = FRONT + 3 * G::MAT + G::TRI * 1024;
};
struct WholeArgs {
  NsMomentum mom;
  const void *g;
  float *m;
  Out o;
  int steps;
};

template <int MAX, int DT, bool MOM>
__device__ __forceinline__ void whole_matrix(const NsMat &M, const NsSteps &S, WholeArgs a, char *ws, char *lds, double *red) {
  using L = Whole<MAX>;
  char *mats = lds + L::FRONT, *P = mats + 2 * L::G::MAT;
  float *gram = (float *)(P + L::G::MAT);
  float *X = (float *)(ws + M.ws_xn);
  const double norm = sqrt(ns_block_sum(prep_rows<DT, MOM>(M, a.mom, a.g, a.m, (float *)(ws + M.ws_u), 0, M.n, (float *)lds), red));
  __syncthreads();  // u is written
  const float *src = ns_source(M, ws, a.g);
  const int first = threadIdx.x >> 6;
  a.o.gain = M.gain;
#define CALL(MT)                                                                                              \
  {                                                                                                           \
    constexpr bool F = Geo<MT>::F32;                                                                          \
    const int stages = F ? a.steps : S.stages;                                                                \
    Scale sc = scale_of(1.0 / (norm + S.eps), F ? 1.f : S.stage[0].sx);                                       \
    Acc<MT> acc{};                                                                                            \
    GramRows<MT> rows;                                                                                        \
    for (int n0 = first * 32; n0 < M.n; n0 += 128) {                                                          \
      Frag<F> f[Geo<MT>::TT];                                                                                 \
      rows.load(src, M.n, n0);                                                                                \
      rows.factors(f, M.n, n0, sc);                                                                           \
      gram_add<MT>(acc, f);                                                                                   \
    }                                                                                                         \
    float sx = F ? 1.f : S.stage[0].sx;                                                                       \
    for (int s = 0; s < stages; ++s) {                                                                        \
      NsStage st = S.stage[F ? 0 : s];                                                                        \
      if (F) st.steps = 1;                                                                                    \
      gram_out<MT, 4>(acc, lds, 1.f / (sx * sx), gram);                                                         \
      __syncthreads();                                                                                        \
      polynomial<MT, 4>(gram, 1, st, (float)S.a, (float)S.b, (float)S.c, mats, P);                            \
      const float sp = F ? 1.f : st.steps == 2 ? st.sp : st.sq[0];                                            \
      ApplyRows<MT> x;                                                                                        \
      if (first * 32 < M.n) x.load(src, M.n, first * 32);                                                     \
      if (s + 1 < stages) {                                                                                   \
        const float sn = F ? 1.f : S.stage[s + 1].sx;                                                         \
        acc = Acc<MT>{};                                                                                      \
        apply_gram_steps<MT>(acc, x, src, X, M.n, first, 4, sc, sn / (sx * sp), P);                           \
        src = X;                                                                                              \
        sc = Scale{false, 1.f, 1.f};                                                                          \
        sx = sn;                                                                                              \
      } else {                                                                                                \
        final_steps<MT, DT>(M, a.o, x, src, first, 4, sc, 1.f / (sx * sp), P);                                \
      }                                                                                                       \
    }                                                                                                         \
  }
  CF_NS_WIDTH(L::W, M.mt, CALL)
#undef CALL
}

// a table of nothing but such matrices
template <int MAX, int DT, bool MOM>
__global__ __launch_bounds__(256) void skinny_whole_kernel(NsTable T, NsSteps S, WholeArgs a, char *ws) {
  __shared__ __attribute__((aligned(16))) char lds[Whole<MAX>::BYTES];
  __shared__ double red[4];
  whole_matrix<MAX, DT, MOM>(T.mat[T.whole[blockIdx.x]], S, a, ws, lds, red);
}

// Gram matrix of X = u / (||u|| + eps).  The first workgroups run the table's small
// matrices as a whole beside it: they take no longer than the large ones here.
template <int MAX, int DT, bool MOM>
__global__ __launch_bounds__(256) void skinny_gram_kernel(NsTable T, NsSteps S, WholeArgs a, char *ws) {
  __shared__ __attribute__((aligned(16))) char lds[most(4 * Geo<MAX>::SET, Whole<MAX>::BYTES)];
  __shared__ double red[4];
  if ((int)blockIdx.x < T.wholes) {
    whole_matrix<MAX, DT, MOM>(T.mat[T.whole[blockIdx.x]], S, a, ws, lds, red);
    return;
  }
  const NsStage &st = S.stage[0];
  const int l = ns_find(T, blockIdx.x - T.wholes);
  const NsMat &M = T.mat[l];
  const int b = blockIdx.x - T.wholes - T.first[l];
  const float *X = ns_source(M, ws, a.g);
  const int first = b * 4 + (threadIdx.x >> 6), stride = M.slices * 4;
#define CALL(MT)                                                                                              \
  {                                                                                                           \
    GramRows<MT> x;                                                                                           \
    x.load(X, M.n, first * 32);                                                                               \
    const float sx = Geo<MT>::F32 ? 1.f : st.sx;                                                              \
    const Scale sc = scale_of(ns_inv_norm(M, ws, S.eps, red), sx);                                           \
    Acc<MT> acc{};                                                                                            \
    for (int n0 = first * 32; n0 < M.n; n0 += stride * 32) {                                                  \
      Frag<Geo<MT>::F32> f[Geo<MT>::TT];                                                                      \
      x.factors(f, M.n, n0, sc);                                                                              \
      if (n0 + stride * 32 < M.n) x.load(X, M.n, n0 + stride * 32);                                           \
      gram_add<MT>(acc, f);                                                                                   \
    }                                                                                                         \
    gram_out<MT, 4>(acc, lds, 1.f / (sx * sx), (float *)(ws + M.ws_part) + (long long)b * (Geo<MT>::TRI * 256));  \
  }
  CF_NS_WIDTH(MAX, M.mt, CALL)
#undef CALL
}

// sums of many workgroups' Gram matrices: 16 columns of float4 by 16 phases a workgroup
__global__ __launch_bounds__(256) void skinny_sum_kernel(NsTable T, char *ws) {
  __shared__ float4 red[256];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int tt = M.mt / 16, cols = tt * (tt + 1) / 2 * 64;  // float4 of a Gram matrix
  const int c = (blockIdx.x - T.first[l]) * 16 + (threadIdx.x & 15), ph = threadIdx.x >> 4;
  const float4 *part = (const float4 *)(ws + M.ws_part);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = ph; i < M.slices; i += 16) {
    const float4 a = part[(long long)i * cols + c];
    s.x += a.x; s.y += a.y; s.z += a.z; s.w += a.w;
  }
  red[threadIdx.x] = s;
  __syncthreads();
  for (int st = 8; st > 0; st >>= 1) {
    if (ph < st) {
      const float4 a = red[threadIdx.x + st * 16];
      float4 b = red[threadIdx.x];
      b.x += a.x; b.y += a.y; b.z += a.z; b.w += a.w;
      red[threadIdx.x] = b;
    }
    __syncthreads();
  }
  if (ph == 0) ((float4 *)(ws + M.ws_sum))[c] = red[threadIdx.x];
}

// the Gram matrix of all slices, in as many arrays as `parts` says
__device__ __forceinline__ const float *gram_of(const NsMat &M, const char *ws, int *parts) {
  const bool summed = M.slices > kNsFewSlices;
  *parts = summed ? 1 : M.slices;
  return (const float *)(ws + (summed ? M.ws_sum : M.ws_part));
}

// X <- X P (from the matrix itself in the first stage) and the Gram matrix of the result,
// into the other of the two buffers of slices.  Every workgroup computes P for itself: a
// launch of one workgroup a matrix for it and the way through memory take longer.
template <int MAX>
__global__ __launch_bounds__(512) void skinny_apply_kernel(NsTable T, NsStage st, float ca, float cb, float cc, float next_sx,
                                                           int first_stage, double eps, const void *g, char *ws) {
  constexpr int SETS = MAX == 128 ? most(kPairs * Geo<128>::SET, Geo<128>::MAT + kPairLds) : 8 * Geo<MAX>::SET;
  __shared__ __attribute__((aligned(16))) char lds[most(SETS, 2 * Geo<MAX>::MAT)];
  __shared__ double red[8];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int b = blockIdx.x - T.first[l];
  float *X = (float *)(ws + M.ws_xn);
  const float *src = first_stage ? ns_source(M, ws, g) : X;
  const int first = b * 8 + (threadIdx.x >> 6), stride = M.slices * 8;
  int parts;
  const float *gram = gram_of(M, ws, &parts);
  // (with few slices the sums' launch does not run, and others still read this buffer)
  float *part = (float *)(ws + M.ws_part2);
  if (MAX == 128 && M.mt == 128) {
    const float sx = st.sx, sp = st.steps == 2 ? st.sp : st.sq[0];
    const Scale sc = first_stage ? scale_of(ns_inv_norm<8>(M, ws, eps, red), sx) : Scale{false, 1.f, 1.f};
    ApplyRows<128> x;
    x.load(src, M.n, (b * kPairs + (threadIdx.x >> 6 & 3)) * 32);
    polynomial<128, 8>(gram, parts, st, ca, cb, cc, lds, lds);
    PairAcc acc{};
    apply_gram_pairs(acc, x, src, X, M.n, b, M.slices, sc, next_sx / (sx * sp), lds, lds + Geo<128>::MAT);
    pairs_out(acc, lds, 1.f / (next_sx * next_sx), part + (long long)b * (Geo<128>::TRI * 256));
    return;
  }
#define CALL(MT)                                                                                               \
  {                                                                                                            \
    constexpr bool F = Geo<MT>::F32;                                                                           \
    const float sx = F ? 1.f : st.sx, sp = F ? 1.f : st.steps == 2 ? st.sp : st.sq[0], sn = F ? 1.f : next_sx; \
    ApplyRows<MT> x;                                                                                           \
    x.load(src, M.n, first * 32);                                                                              \
    const Scale sc = first_stage ? scale_of(ns_inv_norm<8>(M, ws, eps, red), sx) : Scale{false, 1.f, 1.f};     \
    polynomial<MT, 8>(gram, parts, st, ca, cb, cc, lds, lds);                                                  \
    Acc<MT> acc{};                                                                                             \
    apply_gram_steps<MT>(acc, x, src, X, M.n, first, stride, sc, sn / (sx * sp), lds);                         \
    gram_out<MT, 8>(acc, lds, 1.f / (sn * sn), part + (long long)b * (Geo<MT>::TRI * 256));                     \
  }
  CF_NS_WIDTH((MAX < 64 ? MAX : 64), M.mt, CALL)
#undef CALL
}

// workgroups of the last product, eight waves of 32 rows at a time
__host__ __device__ inline int final_groups(const NsMat &M) { return min((M.n + 255) / 256, kNsSlices); }

template <int MAX, int DT>
__global__ __launch_bounds__(512) void skinny_final_kernel(NsTable T, NsStage st, float ca, float cb, float cc, int first_stage,
                                                           double eps, const void *g, Out o, char *ws) {
  __shared__ __attribute__((aligned(16))) char lds[2 * Geo<MAX>::MAT];
  __shared__ double red[8];
  const int l = ns_find(T, blockIdx.x);
  const NsMat &M = T.mat[l];
  const int b = blockIdx.x - T.first[l];
  const float *src = first_stage ? ns_source(M, ws, g) : (const float *)(ws + M.ws_xn);
  const int first = b * 8 + (threadIdx.x >> 6), stride = final_groups(M) * 8;
  int parts;
  const float *gram = gram_of(M, ws, &parts);
  o.gain = M.gain;
#define CALL(MT)                                                                                                   \
  {                                                                                                                \
    ApplyRows<MT> x;                                                                                               \
    x.load(src, M.n, first * 32);                                                                                  \
    constexpr bool F = Geo<MT>::F32;                                                                               \
    const float sx = F ? 1.f : st.sx, sp = F ? 1.f : st.steps == 2 ? st.sp : st.sq[0];                              \
    const Scale sc = first_stage ? scale_of(ns_inv_norm<8>(M, ws, eps, red), sx) : Scale{false, 1.f, 1.f};         \
    polynomial<MT, 8>(gram, parts, st, ca, cb, cc, lds, lds);                                                      \
    final_steps<MT, DT>(M, o, x, src, first, stride, sc, 1.f / (sx * sp), lds);                                    \
  }
  CF_NS_WIDTH(MAX, M.mt, CALL)
#undef CALL
}

template <int MAX, int DT, bool MOM>
hipError_t run(const NsTable &T0, const NsSteps &S, const WholeArgs &a, char *ws, hipStream_t st) {
  NsTable T = T0;
  auto number = [&](auto blocks) {
    int at = 0;
    for (int l = 0; l < T.count; ++l) {
      T.first[l] = at;
      if (T.mat[l].mt && !T.mat[l].whole) at += blocks(T.mat[l]);
    }
    T.first[T.count] = at;
    return at;
  };
  const void *g = a.g;
  int nb = number([](const NsMat &M) { return M.chunks; });
  if (nb == 0) {
    hipLaunchKernelGGL((skinny_whole_kernel<(MAX < 64 ? MAX : 64), DT, MOM>), dim3(T.wholes), dim3(256), 0, st, T, S, a, ws);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((skinny_prep_kernel<DT, MOM>), dim3(nb), dim3(256), 0, st, T, a.mom, g, a.m, ws);
  const int slabs = number([](const NsMat &M) { return M.slices; });
  hipLaunchKernelGGL((skinny_gram_kernel<MAX, DT, MOM>), dim3(slabs + T.wholes), dim3(256), 0, st, T, S, a, ws);
  for (int s = 0; s < S.stages; ++s) {
    nb = number([](const NsMat &M) {
      const int tt = M.mt / 16;
      return M.slices > kNsFewSlices ? tt * (tt + 1) / 2 * 4 : 0;
    });
    if (nb) hipLaunchKernelGGL(skinny_sum_kernel, dim3(nb), dim3(256), 0, st, T, ws);
    const float ca = (float)S.a, cb = (float)S.b, cc = (float)S.c;
    if (s + 1 < S.stages) {
      number([](const NsMat &M) { return M.slices; });
      hipLaunchKernelGGL((skinny_apply_kernel<MAX>), dim3(slabs), dim3(512), 0, st, T, S.stage[s], ca, cb, cc, S.stage[s + 1].sx,
                         s == 0, S.eps, g, ws);
      // the slices just written are the next stage's
      for (int l = 0; l < T.count; ++l) std::swap(T.mat[l].ws_part, T.mat[l].ws_part2);
    } else {
      nb = number([](const NsMat &M) { return final_groups(M); });
      hipLaunchKernelGGL((skinny_final_kernel<MAX, DT>), dim3(nb), dim3(512), 0, st, T, S.stage[s], ca, cb, cc, s == 0, S.eps, g,
                         a.o, ws);
    }
  }
  return hipGetLastError();
}

template <int MAX>
hipError_t run_type(const NsTable &T, const NsSteps &S, int dtype, bool momentum, const WholeArgs &a, char *ws, hipStream_t st) {
  if (momentum) return run<MAX, DT_F32, true>(T, S, a, ws, st);
  if (dtype == DT_BF16) return run<MAX, DT_BF16, false>(T, S, a, ws, st);
  return run<MAX, DT_F32, false>(T, S, a, ws, st);
}

}  // namespace

hipError_t launch_ns_skinny(const NsTable &T, const NsSteps &S, int dtype, const void *g, const NsMomentum *mom, float *m,
                            const NsUpdate *up, void *out, uint16_t *v16, void *ws, hipStream_t st) {
  int most = 0;
  for (int l = 0; l < T.count; ++l) most = T.mat[l].mt > most ? T.mat[l].mt : most;
  if (most == 0) return hipSuccess;
  int steps = 0;
  for (int s = 0; s < S.stages; ++s) steps += S.stage[s].steps;
  const WholeArgs a{mom ? *mom : NsMomentum{}, g, m,
                    Out{out, v16, up != nullptr, up ? up->eta : 0.f, up ? up->decay : 0.f, 0.f}, steps};
  if (most > 64) return run_type<128>(T, S, dtype, mom, a, (char *)ws, st);
  if (most > 32) return run_type<64>(T, S, dtype, mom, a, (char *)ws, st);
  return run_type<32>(T, S, dtype, mom, a, (char *)ws, st);
}

}  // namespace cf
