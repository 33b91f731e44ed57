// linear.hip -- matrix products with bias, activation and residual in their epilogue, and
// their gradients (gfx950).
//
//   forward        z = x W + b,  y = act(z) + r           x [M][K], W [K][N]
//   backward data  dx = (dz W' + r) act'(z)               z: of the layer before
//   backward weights  dW = x' dz,  db = sum of dz's rows
//
// All three are C[i][j] = sum_l A(i, l) B(l, j) with the sum's axis innermost in memory or
// not: forward has A by rows of l and B by columns, backward data both by rows of l,
// backward weights neither.

#include "linear.h"

namespace cf {
namespace {

constexpr int kThreads = 256;

// one value of the output, C[i][j] = v
template <int DT, int FORM, int ACT>
__device__ __forceinline__ void put(const LinearEpilogue &E, void *out, long long i, int j, int N, float v) {
  typedef typename Store<DT>::T T;
  const long long at = i * N + j;
  if constexpr (FORM == FORM_WEIGHT) {
    ((float *)out)[at] = v;
  } else if constexpr (FORM == FORM_FWD) {
    if (E.bias) v += E.bias[j];
    if (E.z) ((T *)E.z)[at] = from_f32<DT>(v);
    v = act<ACT>(v, E.alpha);
    if (E.residual) v += to_f32<DT>(((const T *)E.residual)[at]);
    ((T *)out)[at] = from_f32<DT>(v);
  } else {
    if (E.residual) v += to_f32<DT>(((const T *)E.residual)[at]);
    if constexpr (ACT != ACT_NONE) v *= act_slope<ACT>(to_f32<DT>(((const T *)E.zin)[at]), E.alpha);
    ((T *)out)[at] = from_f32<DT>(v);
  }
}

// Any sizes and alignment: tiles of 64 x 64, four waves of 32 x 32, both factors element by
// element into LDS with the sum's axis innermost.
template <int DT, int FORM, int ACT>
__global__ __launch_bounds__(kThreads) void any_kernel(LinearPlan S, const void *A_, const void *B_, LinearEpilogue E, void *out,
                                                       float *part) {
  typedef typename Store<DT>::T T;
  constexpr int TB = 64, KS = DT == DT_BF16 ? 32 : 16, LD = KS + (DT == DT_BF16 ? 8 : 4);
  __shared__ __attribute__((aligned(16))) T la[TB * LD], lb[TB * LD];
  const T *A = (const T *)A_, *B = (const T *)B_;
  const long long index = long_index(), tiles = (long long)S.tm * S.tn, tile = index % tiles, slice = index / tiles;
  if (slice >= S.slices) return;
  const long long i0 = tile / S.tn * TB;
  const int j0 = (int)(tile % S.tn) * TB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
  const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
  f32x4_t acc[2][2];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b) acc[a][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const long long l1 = min((slice + 1) * S.per, S.L);
  for (long long l0 = slice * S.per; l0 < l1; l0 += KS) {
#pragma unroll
    for (int q = 0; q < TB * KS / kThreads; ++q) {
      const int id = q * kThreads + tid;
      {
        const int i = Form<FORM>::AK ? id / KS : id % TB, l = Form<FORM>::AK ? id % KS : id / TB;
        const bool in = i0 + i < S.M && l0 + l < l1;
        la[i * LD + l] = in ? A[Form<FORM>::AK ? (i0 + i) * S.L + l0 + l : (l0 + l) * S.M + i0 + i] : (T)0;
      }
      {
        const int j = Form<FORM>::BK ? id / KS : id % TB, l = Form<FORM>::BK ? id % KS : id / TB;
        const bool in = j0 + j < S.N && l0 + l < l1;
        lb[j * LD + l] = in ? B[Form<FORM>::BK ? (j0 + j) * S.L + l0 + l : (l0 + l) * S.N + j0 + j] : (T)0;
      }
    }
    __syncthreads();
    if constexpr (DT == DT_BF16) {
      bf16x8_t a[2], b[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        a[t] = *reinterpret_cast<const bf16x8_t *>(la + (wi + 16 * t + r) * LD + 8 * g);
        b[t] = *reinterpret_cast<const bf16x8_t *>(lb + (wj + 16 * t + r) * LD + 8 * g);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b[u], acc[t][u], 0, 0, 0);
    } else {
#pragma unroll
      for (int k = 0; k < KS; k += 4) {
        float a[2], b[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          a[t] = la[(wi + 16 * t + r) * LD + k + g];
          b[t] = lb[(wj + 16 * t + r) * LD + k + g];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t], b[u], acc[t][u], 0, 0, 0);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const long long i = i0 + wi + 16 * t + 4 * g + e;
        const int j = j0 + wj + 16 * u + r;
        if (i >= S.M || j >= S.N) continue;
        if (S.slices > 1) part[(slice * S.M + i) * S.N + j] = acc[t][u][e];
        else put<DT, FORM, ACT>(E, out, i, j, S.N, acc[t][u][e]);
      }
}

// The slices' sum, in slice order, and the epilogue.
template <int DT, int FORM, int ACT>
__global__ __launch_bounds__(kThreads) void join_kernel(long long M, int N, int slices, const float *part, LinearEpilogue E,
                                                        void *out) {
  const long long n = M * N, at = long_index() * kThreads + threadIdx.x;
  if (at >= n) return;
  float v = part[at];
  for (int s = 1; s < slices; ++s) v += part[s * n + at];
  put<DT, FORM, ACT>(E, out, at / N, (int)(at % N), N, v);
}

// The same for rows of whole 16-byte pieces of bf16: eight outputs a thread.
template <int FORM, int ACT>
__global__ __launch_bounds__(kThreads) void join8_kernel(LinearPlan p, const float *part, LinearEpilogue E, void *out) {
  const long long n = p.M * p.N, at = (long_index() * kThreads + threadIdx.x) * 8;
  if (at >= n) return;
  Eight<DT_BF16> in;
  fetch8<DT_BF16, FORM, ACT>(E, at, 8, in);
  float v[8];
  for (int s = 0; s < p.slices; ++s) {
    const float4 a = *reinterpret_cast<const float4 *>(part + s * n + at), b = *reinterpret_cast<const float4 *>(part + s * n + at + 4);
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = s ? v[q] + x[q] : x[q];
  }
  float bias[8];
  load_bias<FORM>(E, (int)(at % p.N), p.N, bias);
  put8<DT_BF16, FORM, ACT>(E, bias, out, at, 8, in, v);
}

// part[slice][N] = sums of the slice's rows of dz
template <int DT>
__global__ __launch_bounds__(kThreads) void colsum_kernel(long long M, int N, long long per, const void *dz_, float *part) {
  __shared__ float red[kThreads];
  const int tiles = (N + 63) / 64;
  const long long s = blockIdx.x / tiles;
  const int j = (int)(blockIdx.x % tiles) * 64 + (threadIdx.x & 63), ph = threadIdx.x >> 6;
  const typename Store<DT>::T *dz = (const typename Store<DT>::T *)dz_;
  float a = 0.f;
  if (j < N)
    for (long long i = s * per + ph; i < min((s + 1) * per, M); i += 4) a += to_f32<DT>(dz[i * N + j]);
  red[threadIdx.x] = a;
  __syncthreads();
  if (ph == 0 && j < N)
    part[s * N + j] = (red[threadIdx.x] + red[threadIdx.x + 64]) + (red[threadIdx.x + 128] + red[threadIdx.x + 192]);
}

// The same for rows of whole 16-byte pieces: 32 pieces of a row by 8 rows a workgroup, four
// rows of a thread on their way.
template <int DT>
__global__ __launch_bounds__(kThreads) void colsum_vec_kernel(long long M, int N, long long per, const void *dz_, float *part) {
  constexpr int V = Store<DT>::VEC;
  __shared__ float red[8][32 * V + 1];
  const int pieces = N / V, tiles = (pieces + 31) / 32;
  const long long s = blockIdx.x / tiles;
  const int q = (int)(blockIdx.x % tiles) * 32 + (threadIdx.x & 31), ph = threadIdx.x >> 5;
  const typename Store<DT>::T *dz = (const typename Store<DT>::T *)dz_;
  float a[V];
#pragma unroll
  for (int i = 0; i < V; ++i) a[i] = 0.f;
  if (q < pieces) {
    const long long end = min((s + 1) * per, M);
    long long i = s * per + ph;
    for (; i + 24 < end; i += 32) {
      Vec16<DT> v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u].u = ld16<false>(dz + (i + 8 * u) * N + q * V);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < V; ++k) a[k] += to_f32<DT>(v[u].e[k]);
    }
    for (; i < end; i += 8) {
      Vec16<DT> v;
      v.u = ld16<false>(dz + i * N + q * V);
#pragma unroll
      for (int k = 0; k < V; ++k) a[k] += to_f32<DT>(v.e[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < V; ++k) red[ph][(threadIdx.x & 31) * V + k] = a[k];
  __syncthreads();
  for (int c = threadIdx.x; c < 32 * V; c += kThreads) {
    const int j = (int)(blockIdx.x % tiles) * 32 * V + c;
    if (j < N)
      part[s * N + j] = ((red[0][c] + red[1][c]) + (red[2][c] + red[3][c])) + ((red[4][c] + red[5][c]) + (red[6][c] + red[7][c]));
  }
}

bool colsum_vec(int N, int dtype) { return N % (dtype == DT_BF16 ? 8 : 4) == 0; }
int colsum_tiles(int N, int dtype) { return colsum_vec(N, dtype) ? (N + (dtype == DT_BF16 ? 255 : 127)) / (dtype == DT_BF16 ? 256 : 128) : (N + 63) / 64; }
int colsum_slices(long long M, int N, int dtype) {
  return (int)std::max(1LL, std::min<long long>((M + 63) / 64, 1024 / colsum_tiles(N, dtype)));
}

// Slices of the sum: where the output's tiles leave compute units idle, as many as fill
// them twice (each of at least 256 terms), and none of more than kChain terms while the
// partial sums stay below 2^28 values.
int slices_of(long long M, int N, long long L) {
  const long long tiles = (M + 63) / 64 * ((N + 63) / 64), out = M * N;
  const long long fill = std::min(2 * kCUs / tiles, L / 256);
  const long long chain = std::min((L + kChain - 1) / kChain, (1LL << 28) / out);
  return (int)std::max(1LL, std::max(fill, chain));
}
// form, and the output's rows and columns and the sum's terms
LinearPlan plan_of(int form, long long M, int N, long long L, int dtype) {
  LinearPlan p;
  if (dtype == DT_BF16 ? linear_bf16_plan(form, M, N, L, &p) : linear_f32_plan(form, M, N, L, &p)) return p;
  const int slices = slices_of(M, N, L);
  const long long per = ((L + slices - 1) / slices + 31) / 32 * 32;
  return LinearPlan{M, L, N, LIN_ANY, (int)((M + 63) / 64), (N + 63) / 64, (int)((L + per - 1) / per), per, 0, 0, 0, 0};
}
// the workspace holds the slices' sums, then the copies of A and of B
size_t slices_bytes(const LinearPlan &p) {
  return p.slices > 1 ? ((size_t)p.slices * p.M * p.N * 4 + 15) / 16 * 16 : 0;
}
size_t copy_bytes(int form, bool a, const LinearPlan &p) {
  return (a ? p.copy_a : p.copy_b) ? (size_t)row_count(form, a, p.M, p.N, p.L) * (a ? p.lda : p.ldb) * 2 : 0;
}
size_t plan_bytes(int form, const LinearPlan &p) {
  return slices_bytes(p) + copy_bytes(form, true, p) + copy_bytes(form, false, p);
}

// rows of n values to rows of ld, a multiple of 8, the rest zeros; a thread a piece of eight
__global__ __launch_bounds__(kThreads) void pad_rows_kernel(long long rows, int n, int ld, const uint16_t *in, uint16_t *out) {
  const long long id = long_index() * kThreads + threadIdx.x, row = id / (ld / 8);
  if (row >= rows) return;
  const int c = (int)(id % (ld / 8)) * 8;
  const uint16_t *p = in + row * n + c;
  u32x4_t v;
  if (c + 8 <= n) {
    v = *reinterpret_cast<const u32x4e2_t *>(p);
  } else {
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = c + i < n ? p[i] : 0u;
    v = u32x4_t{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
  }
  *reinterpret_cast<u32x4_t *>(out + row * ld + c) = v;
}

template <int FORM>
hipError_t product(const LinearPlan &p, int dtype, const void *A, const void *B, LinearEpilogue E, void *out, float *db,
                   void *ws, hipStream_t st) {
  const long long M = p.M, L = p.L;
  const int N = p.N;
  E.stream = dtype == DT_BF16 && M * N * 2 >= kStreamBytes / 2;
  float *part = (float *)ws;
  auto padded = [&](bool a, const void *src, char *dst) -> const void * {
    if (!copy_bytes(FORM, a, p)) return src;
    const long long rows = row_count(FORM, a, M, N, L), ld = a ? p.lda : p.ldb;
    hipLaunchKernelGGL(pad_rows_kernel, long_grid((rows * (ld / 8) + kThreads - 1) / kThreads), dim3(kThreads), 0, st, rows,
                       (int)row_length(FORM, a, M, N, L), (int)ld, (const uint16_t *)src, (uint16_t *)dst);
    return dst;
  };
  char *copies = (char *)ws + slices_bytes(p);
  A = padded(true, A, copies);
  B = padded(false, B, copies + copy_bytes(FORM, true, p));
  if (p.kernel != LIN_ANY && dtype == DT_BF16) {
    const hipError_t r = launch_linear_bf16(FORM, p, A, B, E, out, part, db, st);
    if (r != hipSuccess) return r;
  } else if (p.kernel != LIN_ANY) {
    const hipError_t r = launch_linear_f32(FORM, p, A, B, E, out, part, db, st);
    if (r != hipSuccess) return r;
  }
  const dim3 grid = long_grid((long long)p.tm * p.tn * p.slices), block(kThreads);
  with_act(E.act, [&](auto a) {
    constexpr int ACT = FORM == FORM_WEIGHT ? (int)ACT_NONE : decltype(a)::value;
    if (p.kernel != LIN_ANY) {
    } else if (dtype == DT_BF16) hipLaunchKernelGGL((any_kernel<DT_BF16, FORM, ACT>), grid, block, 0, st, p, A, B, E, out, part);
    else hipLaunchKernelGGL((any_kernel<DT_F32, FORM, ACT>), grid, block, 0, st, p, A, B, E, out, part);
    if (p.slices > 1 && FORM != FORM_WEIGHT && p.kernel != LIN_ANY && dtype == DT_BF16 && N % 8 == 0) {
      hipLaunchKernelGGL((join8_kernel<FORM, ACT>), long_grid((M * N / 8 + kThreads - 1) / kThreads), block, 0, st, p,
                         (const float *)part, E, out);
    } else if (p.slices > 1 && FORM != FORM_WEIGHT) {
      const dim3 all = long_grid((M * N + kThreads - 1) / kThreads);
      if (dtype == DT_BF16)
        hipLaunchKernelGGL((join_kernel<DT_BF16, FORM, ACT>), all, block, 0, st, M, N, p.slices, (const float *)part, E, out);
      else hipLaunchKernelGGL((join_kernel<DT_F32, FORM, ACT>), all, block, 0, st, M, N, p.slices, (const float *)part, E, out);
    }
  });
  return hipGetLastError();
}

}  // namespace

size_t linear_fwd_workspace(long long M, int K, int N, int dtype) { return plan_bytes(FORM_FWD, plan_of(FORM_FWD, M, N, K, dtype)); }
size_t linear_bwd_data_workspace(long long M, int K, int N, int dtype) {
  return plan_bytes(FORM_DATA, plan_of(FORM_DATA, M, K, N, dtype));
}
// the rows of column sums that a bias gradient is joined from, behind the product's workspace
int db_rows(const LinearPlan &p, long long M, int N, int dtype) {
  return p.kernel == LIN_ANY ? colsum_slices(M, N, dtype) : p.slices * db_turns(p);
}
size_t linear_bwd_weight_workspace(long long M, int K, int N, int dtype) {
  const LinearPlan p = plan_of(FORM_WEIGHT, K, N, M, dtype);
  return plan_bytes(FORM_WEIGHT, p) + ((size_t)db_rows(p, M, N, dtype) * N * 4 + 15) / 16 * 16;
}

hipError_t launch_linear_fwd(long long M, int K, int N, int dtype, const void *x, const void *w, const LinearEpilogue &e,
                             void *y, void *ws, hipStream_t st) {
  return product<FORM_FWD>(plan_of(FORM_FWD, M, N, K, dtype), dtype, x, w, e, y, nullptr, ws, st);
}

hipError_t launch_linear_bwd_data(long long M, int K, int N, int dtype, const void *dz, const void *w,
                                  const LinearEpilogue &e, void *dx, void *ws, hipStream_t st) {
  return product<FORM_DATA>(plan_of(FORM_DATA, M, K, N, dtype), dtype, dz, w, e, dx, nullptr, ws, st);
}

hipError_t launch_linear_bwd_weight(long long M, int K, int N, int dtype, const void *x, const void *dz, float *dw, float *db,
                                    void *ws, hipStream_t st) {
  const LinearEpilogue none{nullptr, nullptr, nullptr, nullptr, ACT_NONE, 0.f};
  const LinearPlan p = plan_of(FORM_WEIGHT, K, N, M, dtype);
  const int rows = db_rows(p, M, N, dtype);
  float *sums = (float *)((char *)ws + plan_bytes(FORM_WEIGHT, p));
  hipError_t r = product<FORM_WEIGHT>(p, dtype, x, dz, none, dw, !db || p.kernel == LIN_ANY ? nullptr : rows == 1 ? db : sums, ws, st);
  if (r != hipSuccess) return r;
  if (db && p.kernel == LIN_ANY) {
    const long long per = (M + rows - 1) / rows;
    const dim3 grid((unsigned)((long long)rows * colsum_tiles(N, dtype))), block(kThreads);
    auto run = [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      if (colsum_vec(N, dtype)) hipLaunchKernelGGL((colsum_vec_kernel<DT>), grid, block, 0, st, M, N, per, dz, sums);
      else hipLaunchKernelGGL((colsum_kernel<DT>), grid, block, 0, st, M, N, per, dz, sums);
    };
    if (dtype == DT_BF16) run(std::integral_constant<int, DT_BF16>{});
    else run(std::integral_constant<int, DT_F32>{});
    if ((r = hipGetLastError()) != hipSuccess) return r;
  }
  // (slices of more than one have fewer than 2^28 values in all, or fill 512 tiles of 4096)
  SumJob jobs[2];
  int n = 0;
  if (p.slices > 1) jobs[n++] = SumJob{(const float *)ws, dw, p.slices, (int)((long long)K * N)};
  if (db && (rows > 1 || p.kernel == LIN_ANY)) jobs[n++] = SumJob{sums, db, rows, N};
  return n ? launch_sum_batch(jobs, n, st) : hipSuccess;
}

}  // namespace cf
