// linear.h -- what the kernels of linear.hip and linear_bf16.hip share.
#pragma once

#include <algorithm>

#include "activation.h"
#include "cf_common.h"
#include "cf_kernels.h"

namespace cf {

// Which operand has the sum's axis innermost.
enum : int { FORM_FWD = 0, FORM_DATA = 1, FORM_WEIGHT = 2 };
template <int FORM> struct Form;
template <> struct Form<FORM_FWD> { static constexpr bool AK = true, BK = false; };
template <> struct Form<FORM_DATA> { static constexpr bool AK = true, BK = true; };
template <> struct Form<FORM_WEIGHT> { static constexpr bool AK = false, BK = false; };

constexpr int kCUs = 256;
constexpr long long kChain = 65536;  // most terms of one fp32 sum, where the partial sums' size allows

// How a product C [M][N], a sum over L terms, is cut: tiles of bm x bn, the sum into slices
// of `per` terms, joined by a second launch.
struct LinearPlan {
  long long M, L;
  int N;
  int kernel;  // LIN_*
  int tm, tn;
  int slices;
  long long per;
  // row lengths of A and B as the kernel reads them, and (bf16) whether they are copies in
  // the workspace, of rows of whole 16-byte pieces
  long long lda, ldb;
  int copy_a, copy_b;
};
enum : int { LIN_ANY = 0, LIN_256 = 1, LIN_128 = 2, LIN_64 = 3 };

// A grid's x dimension holds fewer than 2^32 threads: workgroups past 2^22 go on in y.
inline dim3 long_grid(long long n) {
  const long long x = std::min(n, 1LL << 22);
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ long long long_index() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// Rows and row length of a factor as it lies in memory.
inline long long row_length(int form, bool a, long long M, int N, long long L) {
  return a ? (form == FORM_WEIGHT ? M : L) : form == FORM_DATA ? L : N;
}
inline long long row_count(int form, bool a, long long M, int N, long long L) {
  return a ? (form == FORM_WEIGHT ? L : M) : form == FORM_DATA ? N : L;
}

// The bf16 kernels (linear_bf16.hip).  part: the slices' sums [slices][M][N] where there are
// several.  db (backward weights, may be null): sums over B's rows, [slices][db_turns][N].
bool linear_bf16_plan(int form, long long M, int N, long long L, LinearPlan *p);
hipError_t launch_linear_bf16(int form, const LinearPlan &p, const void *A, const void *B, const LinearEpilogue &E, void *out,
                              float *part, float *db, hipStream_t st);

// The fp32 kernels (linear_f32.hip): any sizes whose rows 32-bit offsets reach.
bool linear_f32_plan(int form, long long M, int N, long long L, LinearPlan *p);
hipError_t launch_linear_f32(int form, const LinearPlan &p, const void *A, const void *B, const LinearEpilogue &E, void *out,
                             float *part, float *db, hipStream_t st);

// ---- device helpers -----------------------------------------------------------------

typedef __attribute__((address_space(3))) void lds_void_t;

constexpr uint32_t kOut = 0x80000000u;  // past every buffer: the load gives zeros

// The exchange of the 16-byte pieces of 128-byte rows in LDS: the sixteen rows of a fragment
// at one piece touch all banks.  Rows of a fragment: 16 t + r, or (COLS), of every 64, 8 t + r
// (r < 8) and 32 + 8 t + r - 8: after the epilogue's exchange a lane then has twice eight
// columns, and four lanes eight by eight 64 neighbouring values of a row of C.
template <bool COLS> __device__ __forceinline__ int swizzle(int row) {
  return COLS ? ((row >> 1) & 3) | ((row >> 5) & 1) << 2 : (row >> 1) & 7;
}

// waits until at most N of the wave's loads are in flight, and for its LDS reads
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xc07f); }  // lgkmcnt(0)
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Four registers of four lanes (those 16 apart) transposed: register k of lane g gets
// register g of lane k.
__device__ __forceinline__ void transpose4(float &a, float &b, float &c, float &d) {
  auto swap32 = [](float &x, float &y) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    x = __uint_as_float(s[0]);
    y = __uint_as_float(s[1]);
  };
  auto swap16 = [](float &x, float &y) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    x = __uint_as_float(s[0]);
    y = __uint_as_float(s[1]);
  };
  swap32(a, c);
  swap32(b, d);
  swap16(a, b);
  swap16(c, d);
}

// Sums of B's columns over the terms, for the bias gradient, out of the fragments that the
// products read anyway: the first tiles of a column of tiles take turns, a step each, so that
// none is much longer than the others.  (32768 x 4096 x 1024 bf16: 243 us with db, 241
// without; a pass of its own over dz took 14 us more.)  A short sum that is not cut has one
// tile do it all, which writes db itself: the launch that joins rows takes 3 us.
__host__ __device__ inline int db_turns(const LinearPlan &p) {
  return p.slices == 1 && p.L <= 1024 ? 1 : p.tm < 16 ? p.tm : 16;
}
template <int TN> struct ColumnSums {
  float s[TN];  // of the lane's column of each fragment, over the lane's terms
  bool use, mine;
  int turn, turns;
  __device__ __forceinline__ ColumnSums(bool use_, int ti, int turns_) : use(use_), mine(use_ && ti == 0), turn(ti), turns(turns_) {
#pragma unroll
    for (int j = 0; j < TN; ++j) s[j] = 0.f;
  }
  __device__ __forceinline__ void next_step() {
    turn = turn == 0 ? turns - 1 : turn - 1;
    mine = use && turn == 0;
  }
  // the wave's 64 columns from j0 on
  __device__ __forceinline__ void store(float *row, int j0, int N) {
    const int lane = threadIdx.x & 63, r = lane & 15;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      s[j] += __shfl_xor(s[j], 16, 64);
      s[j] += __shfl_xor(s[j], 32, 64);
      const int c = j0 + 8 * j + (r & 7) + 32 * (r >> 3);
      if (lane < 16 && c < N) row[c] = s[j];
    }
  }
};

// Eight neighbouring values of a row, of which n exist; rows start anywhere.
typedef uint32_t u32x4e4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4e2_t __attribute__((ext_vector_type(4), aligned(2)));
template <int DT> struct Eight;
template <> struct Eight<DT_BF16> {
  u32x4_t a;
  __device__ __forceinline__ void load(const uint16_t *p, int n) {
    if (n >= 8) {
      a = *reinterpret_cast<const u32x4e2_t *>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = (2 * i < n ? p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ float operator[](int i) const {
    return __uint_as_float(i % 2 ? a[i / 2] & 0xffff0000u : a[i / 2] << 16);
  }
};
template <> struct Eight<DT_F32> {
  u32x4_t a, b;
  __device__ __forceinline__ void load(const float *p, int n) {
    if (n >= 8) {
      a = reinterpret_cast<const u32x4e4_t *>(p)[0];
      b = reinterpret_cast<const u32x4e4_t *>(p)[1];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = i < n ? __float_as_uint(p[i]) : 0u;
        b[i] = 4 + i < n ? __float_as_uint(p[4 + i]) : 0u;
      }
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i < 4 ? a[i % 4] : b[i % 4]); }
};
// (non-temporal stores of outputs of half the last-level cache and more: forward and backward
// of 32768 x 1024 x 4096 bf16 1697 -> 1648 us, of 16384 rows 904 -> 886; of 8192 rows 516 -> 519,
// what reads them next finds less of them)
__device__ __forceinline__ void store8(uint16_t *p, int n, const float (&x)[8], bool stream) {
  if (n >= 8 && stream) {
    __builtin_nontemporal_store(pack_bf16x8(x), reinterpret_cast<u32x4e2_t *>(p));
  } else if (n >= 8) {
    *reinterpret_cast<u32x4e2_t *>(p) = pack_bf16x8(x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = f2bf(x[i]);
  }
}
__device__ __forceinline__ void store8(float *p, int n, const float (&x)[8], bool) {
  if (n >= 8) {
    u32x4_t a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __float_as_uint(x[i]);
      b[i] = __float_as_uint(x[4 + i]);
    }
    reinterpret_cast<u32x4e4_t *>(p)[0] = a;
    reinterpret_cast<u32x4e4_t *>(p)[1] = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = x[i];
  }
}

// What an epilogue reads of the outputs' shape.  All of a wave's such loads go out in front
// of its first store: behind a store, which may have changed what they read, each would wait
// for memory by itself (data gradient of 32768 x 4096 x 1024 with GELU 373 -> 355 us).  Where
// both a slope and a residual are read, the residual's loads wait.
template <int DT, int FORM, int ACT>
__device__ __forceinline__ void fetch8(const LinearEpilogue &E, long long at, int n, Eight<DT> &x) {
  typedef typename Store<DT>::T T;
  if constexpr (FORM == FORM_DATA && ACT != ACT_NONE) x.load((const T *)E.zin + at, n);
  else if (FORM != FORM_WEIGHT && E.residual) x.load((const T *)E.residual + at, n);
}

// Slopes of all bf16 values of sizes from 2^-16 to 32 (nearer 0 and further out they change
// by less than 2^-15, or from less than 1e-12 to 0), a value's at 4 times its bits, negative ones 16384
// bytes on.  The epilogue of a 256 x 256 tile looks 65536 of them up in less time than it
// computes them (data gradient of 32768 x 4096 x 1024 with GELU 355 -> 332 us); smaller tiles
// have too few outputs for a table's worth of work.
struct SlopeTable {
  static constexpr int LO = 0x3780, HI = 0x4200, BYTES = 16384 + (HI - LO + 1) * 4;
  template <int ACT> static __device__ __forceinline__ void fill(unsigned char *t, float alpha) {
    for (int i = threadIdx.x; i < 2 * (HI - LO + 1); i += blockDim.x) {
      const int half = i > HI - LO, a = half ? i - (HI - LO + 1) : i;
      *reinterpret_cast<float *>(t + half * 16384 + a * 4) = act_slope<ACT>(__uint_as_float((uint32_t)(LO + a + half * 0x8000) << 16), alpha);
    }
  }
  // value i of x (a NaN or an infinity gives NaN, as the formula does)
  static __device__ __forceinline__ float at(const unsigned char *t, const Eight<DT_BF16> &x, int i) {
    const uint32_t b = i % 2 ? x.a[i / 2] >> 14 : x.a[i / 2] << 2;
    const uint32_t a = min(max(b & 0x1fffcu, LO * 4u), HI * 4u) + (b >> 3 & 0x4000u);
    return __builtin_fmaf(x[i], 0.f, *reinterpret_cast<const float *>(t + (int)a - LO * 4));
  }
};

// The normal distribution function from -8 to 8 in steps of 1/256: value and difference, in
// between a straight line, off by an eighth of the step's square of its curvature |u| phi(u):
// below 2^-21, and for u < 0 below 2^-19 (u^2 + 1) of itself (2^-13 of itself at -8, where it is
// 6e-16, 2^-14.9 and less from -4 on; an output's rounding to bf16 is 2^-8); below -8 it is 0.
// GELU of 32768 x 1024 x 4096 by formula 295 us, from here 268.
struct PhiTable {
  static constexpr int N = 4096, BYTES = N * 8;
  static __device__ __forceinline__ void fill(unsigned char *t) {
    for (int i = threadIdx.x; i < N; i += blockDim.x) {
      auto phi = [](int k) {
        const float u = (k - N / 2) * (1.f / 256), q = bell(u) * normal_tail(fabsf(u));
        return u >= 0.f ? 1.f - q : q;
      };
      const float a = phi(i), b = phi(i + 1);
      *reinterpret_cast<float2 *>(t + i * 8) = i == 0 ? float2{0.f, 0.f} : i == N - 1 ? float2{1.f, 0.f} : float2{a, b - a};
    }
  }
  static __device__ __forceinline__ float gelu(const unsigned char *t, float u) {
    const float k = __builtin_amdgcn_fmed3f(__builtin_fmaf(u, 256.f, (float)(N / 2)), 0.f, N - 1.f);
    const float2 e = *reinterpret_cast<const float2 *>(t + (uint32_t)k * 8);
    return u * __builtin_fmaf(__builtin_amdgcn_fractf(k), e.y, e.x);
  }
};

// eight neighbouring outputs; x: what fetch8 read for them; TABLE: slopes, or values, from `table`
template <int DT, int FORM, int ACT, bool TABLE = false>
__device__ __forceinline__ void put8(const LinearEpilogue &E, const float (&bias)[8], void *out, long long at, int n,
                                     const Eight<DT> &x, float (&v)[8], const unsigned char *table = nullptr) {
  typedef typename Store<DT>::T T;
  if constexpr (FORM == FORM_WEIGHT) {
    store8((float *)out + at, n, v, false);
  } else if constexpr (FORM == FORM_FWD) {
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] += bias[q];
    if (E.z) store8((T *)E.z + at, n, v, E.stream);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if constexpr (TABLE) v[q] = PhiTable::gelu(table, v[q]);
      else v[q] = act<ACT>(v[q], E.alpha);
    }
    if (E.residual) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += x[q];
    }
    store8((T *)out + at, n, v, E.stream);
  } else {
    if (E.residual) {
      Eight<DT> r = x;
      if constexpr (ACT != ACT_NONE) r.load((const T *)E.residual + at, n);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] += r[q];
    }
    if constexpr (ACT != ACT_NONE) {
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if constexpr (TABLE) v[q] *= SlopeTable::at(table, x, q);
        else v[q] *= act_slope<ACT>(x[q], E.alpha);
      }
    }
    store8((T *)out + at, n, v, E.stream);
  }
}

// the bias of columns j .. j + 7 (a multiple of 8)
template <int FORM>
__device__ __forceinline__ void load_bias(const LinearEpilogue &E, int j, int N, float (&b)[8]) {
  Eight<DT_F32> x{};
  if (FORM == FORM_FWD && E.bias) x.load(E.bias + j, N - j);
#pragma unroll
  for (int q = 0; q < 8; ++q) b[q] = x[q];
}

}  // namespace cf
