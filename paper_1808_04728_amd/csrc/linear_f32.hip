// linear_f32.hip -- fp32 matrix products on tiles of 128 and 64 (gfx950).
//
// As the bf16 kernels' tiles, with the fp32 matrix instructions (16 x 16 x 4: a sixteenth of
// the bf16 rate, so the matrix units are busy eight times as long for the same bytes).  Rows
// may start on any element and end anywhere: then every lane loads single values, for which
// the matrix instructions leave time enough, and 16 bytes where all rows are whole 16-byte
// pieces.  What is past a row's or the sum's end reads as zeros.  A step is 32 terms.  A factor
// with the sum's axis innermost lies in LDS by rows of 32 terms and is read four terms a lane;
// one with the sum's axis outermost lies by terms and is read value by value, a lane's four
// terms the same four as the other factor's.
//
// Bound by the matrix cores (4096^3 140 TFLOP/s, the library's product 149), and small or ragged
// products by their last round of tiles: 4097 x 515 x 1027 is 1105 tiles of 64 for 256 compute
// units, 64 us at 68 TFLOP/s.

#include "linear.h"

namespace cf {
namespace {

// A tile: WM x WN waves of TM x TN instruction tiles of 16 x 16; NS steps in LDS.
template <int KERNEL> struct Tile;
template <> struct Tile<LIN_128> {
  static constexpr int B = 128, WM = 2, WN = 2, NS = 2, WAVES = 2;
};
template <> struct Tile<LIN_64> {
  static constexpr int B = 64, WM = 4, WN = 1, NS = 3, WAVES = 3;
};
constexpr int BK = 32, NT = 256;

// The rows r0 .. r0 + ROWS - 1 of a factor, a step of BK terms at a time; NT lanes load V values
// each.  KC: the sum's axis is innermost.  Otherwise the columns of term k are exchanged by 16
// (COLS: by 8) with k / 4, so that the four lanes of a column that read four terms apart
// touch different banks.
template <bool COLS> constexpr int kExchange = COLS ? 8 : 16;
template <bool KC, bool COLS, int ROWS, int V> struct Loader {
  static constexpr int N = ROWS * BK / (NT * V), LINE = (KC ? BK : ROWS) / V;  // loads; lanes of a line in LDS
  const char *base;
  long long advance;  // bytes of a step
  uint32_t off[N];
  int term[2];  // the lane's (first) term: in loads of kind 0 and 1, or (not KC) of load 0
  __device__ __forceinline__ Loader(const float *p, long long rows, long long terms, int r0, long long k0) {
    const long long ld = KC ? terms : rows;
    base = (const char *)(p + (KC ? r0 * ld + k0 : k0 * ld + r0));
    advance = (KC ? 1 : ld) * BK * 4;
    const long long have = rows - r0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int line = (i * NT + threadIdx.x) / LINE, at = threadIdx.x % LINE * V;
      if constexpr (KC) {
        const int k = ((at >> 2) ^ swizzle<COLS>(line)) * 4 + (at & 3);
        off[i] = line < have ? (uint32_t)(line * ld * 4) + k * 4 : kOut;
        term[kind(i)] = k;
      } else {
        const int c = at ^ ((line >> 2) & 3) * kExchange<COLS>;
        off[i] = c < have ? (uint32_t)(line * ld * 4) + c * 4 : kOut;
        if (i == 0) term[0] = term[1] = line;
      }
    }
  }
  // KC: what load i's lines have in their exchange beyond those of load 0 or 1
  static constexpr int kind(int i) {
    constexpr int PER = NT / LINE;  // lines of a load: 8 or 32
    return COLS ? (i * PER >> 5) & 1 : (i * PER >> 3) & 1;
  }
  // Load i of the next step to `stage` (bytes from the LDS's start); `rest` terms are left.
  // (Written out, with the kernel's own waits, as in the bf16 kernels.)
  __device__ __forceinline__ void load(int i, int wave, uint32_t stage, int rest) const {
    const uint32_t o = (KC ? term[kind(i)] < rest : term[0] < rest - i * (NT / LINE)) ? off[i] : kOut;
    const u32x4_t r = {(uint32_t)(uintptr_t)base, (uint32_t)((uintptr_t)base >> 32) & 0xffffu, 0x7ffffff0u, 0x00020000u};
    const uint32_t to = stage + (uint32_t)(i * NT + wave * 64) * 4 * V;
    if constexpr (V == 4)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to), "v"(o), "s"(r) : "memory");
    else
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(to), "v"(o), "s"(r) : "memory");
  }
  __device__ __forceinline__ void next() { base += advance; }
};

// A lane's place in the fragments of 16 rows (see swizzle) and 16 terms: its terms 4 g .. 4 g + 3.
template <bool KC, bool COLS, int ROWS> struct Reader {
  int lane_off, swz;
  __device__ __forceinline__ Reader() {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int row = COLS ? (r & 7) + 32 * (r >> 3) : r;
    lane_off = KC ? row * BK * 4 : 4 * g * ROWS * 4 + row * 4;
    swz = KC ? swizzle<COLS>(row) : g;
  }
  // fragment t of the stage, terms 16 k ..
  __device__ __forceinline__ f32x4_t frag(const unsigned char *stage, int t, int k) const {
    if constexpr (KC) {
      const int g = (threadIdx.x & 63) >> 4, row = COLS ? t / 4 * 64 + t % 4 * 8 : t * 16;
      return *reinterpret_cast<const f32x4_t *>(stage + lane_off + row * BK * 4 + (((4 * k + g) ^ swz) << 4));
    } else {
      const unsigned char *p = stage + lane_off + (t / 4 * 64 + ((t % 4) ^ swz) * kExchange<COLS>) * 4 + 16 * k * ROWS * 4;
      f32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const float *>(p + e * ROWS * 4);
      return v;
    }
  }
};

template <int KERNEL, int FORM, int ACT, int V>
__global__ __launch_bounds__(NT, Tile<KERNEL>::WAVES) void product_kernel(LinearPlan p, long long per_xcd, const float *A,
                                                                          const float *B, LinearEpilogue E, void *out,
                                                                          float *part, float *db) {
  using C = Tile<KERNEL>;
  constexpr int TM = C::B / C::WM / 16, TN = C::B / C::WN / 16, AB = C::B * BK * 4, STAGE = 2 * AB;
  static_assert(TN == 4 && 64 * C::WM * C::WN == NT, "a lane's row of the epilogue is sixteen columns of 64");
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::NS * STAGE];

  // (the order of tiles of the bf16 kernels)
  const long long index = long_index(), job = (index & 7) * per_xcd + (index >> 3);
  const long long tiles = (long long)p.tm * p.tn;
  if (job >= tiles * p.slices) return;
  const long long slice = job / tiles, t = job % tiles, group = t / (8 * p.tn), in = t % (8 * p.tn);
  const int high = (int)min(8LL, p.tm - 8 * group);
  const int i0 = (int)(8 * group + in % high) * C::B, j0 = (int)(in / high) * C::B;
  const long long k0 = slice * p.per, k1 = min(k0 + p.per, p.L);
  const int steps = k1 > k0 ? (int)((k1 - k0 + BK - 1) / BK) : 0;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  Loader<Form<FORM>::AK, false, C::B, V> la(A, p.M, p.L, i0, k0);
  Loader<Form<FORM>::BK, true, C::B, V> lb(B, p.N, p.L, j0, k0);
  const Reader<Form<FORM>::AK, false, C::B> ra;
  const Reader<Form<FORM>::BK, true, C::B> rb;
  constexpr int NA = decltype(la)::N, LOADS = NA + decltype(lb)::N;
  static_assert((C::NS - 1) * LOADS < 64, "loads that a wait can leave in flight");
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t *)lds;
  int rest = (int)(p.L - k0);  // terms from the next step to load on
  auto load = [&](int q, int stage) {  // load q of the next step
    if (q < NA) la.load(q, wave, lds0 + stage * STAGE, rest);
    else lb.load(q - NA, wave, lds0 + stage * STAGE + AB, rest);
  };
  auto next = [&] {
    la.next();
    lb.next();
    rest -= BK;
  };

  f32x4_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // As in the bf16 kernels: the fragments of the next 16 terms are read, and the step NS
  // further is loaded, between the matrix instructions of these; one barrier a step.
  f32x4_t fb[2][TN], fa[2][TM];
  auto read = [&](int f, int q, const unsigned char *stage, int k) {
    if (q < TN) fb[f][q] = rb.frag(stage + AB, wn * TN + q, k);
    else fa[f][q - TN] = ra.frag(stage, wm * TM + q - TN, k);
  };
  const int ti = i0 / C::B;
  const int turns = FORM == FORM_WEIGHT ? db_turns(p) : 0;
  const bool sum_db = FORM == FORM_WEIGHT && db && wm == 0 && ti < turns;
  ColumnSums<TN> sums(sum_db, ti, turns);
  auto half = [&](int f, const unsigned char *rs, int k, auto loads, int ls) {
    if constexpr (FORM == FORM_WEIGHT) {
      if (sums.mine) {
#pragma unroll
        for (int j = 0; j < TN; ++j) sums.s[j] += (fb[f][j][0] + fb[f][j][1]) + (fb[f][j][2] + fb[f][j][3]);
      }
    }
    constexpr int GROUPS = 4 * TM, FIRST = 3 * TM;  // reads go out in the first groups
#pragma unroll
    for (int n = 0; n < GROUPS; ++n) {
#pragma unroll
      for (int q = n * (TM + TN) / FIRST; q < (n + 1) * (TM + TN) / FIRST && q < TM + TN; ++q) read(1 - f, q, rs, k);
#pragma unroll
      for (int q = n * decltype(loads)::value / GROUPS; q < (n + 1) * decltype(loads)::value / GROUPS; ++q) load(q, ls);
      __builtin_amdgcn_sched_barrier(0);
      const int i = n / 4, e = n % 4;
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[f][j][e], fa[f][i][e], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int n = 0; n < C::NS; ++n) {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) load(q, n);
    next();
  }
  wait_loads<(C::NS - 1) * LOADS>();
  barrier();
#pragma unroll
  for (int q = 0; q < TM + TN; ++q) read(0, q, lds, 0);
  int slot = 0;
  for (int s = 0; s < steps; ++s) {
    const int after = slot + 1 == C::NS ? 0 : slot + 1;
    half(0, lds + slot * STAGE, 1, std::integral_constant<int, 0>{}, 0);
    wait_lds();
    wait_loads<(C::NS - 2) * LOADS>();
    barrier();
    half(1, lds + after * STAGE, 0, std::integral_constant<int, LOADS>{}, slot);
    next();
    slot = after;
    if constexpr (FORM == FORM_WEIGHT) sums.next_step();
  }
  wait_loads<0>();  // no load outlives the workgroup
  if (sum_db) sums.store(db + (slice * turns + ti) * p.N, j0 + wn * 64, p.N);

  // lane (r, g) gets row r of each instruction tile, columns 8 g .. 8 g + 7 and 32 + 8 g .. of 64
  const int r = lane & 15, g = lane >> 4, j = j0 + wn * 64 + 8 * g;
  const bool whole = p.slices == 1;
  const float none[8] = {};
  float bias[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) load_bias<FORM>(E, j + 32 * h, p.N, bias[h]);
  Eight<DT_F32> ahead[TM][2];
  if (whole) {
#pragma unroll
    for (int ii = 0; ii < TM; ++ii) {
      const long long i = (long long)i0 + (wm * TM + ii) * 16 + r;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = p.N - j - 32 * h;
        if (i < p.M && n > 0) fetch8<DT_F32, FORM, ACT>(E, i * p.N + j + 32 * h, n, ahead[ii][h]);
      }
    }
  }
#pragma unroll
  for (int ii = 0; ii < TM; ++ii) {
    float row[16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int k = 0; k < 4; ++k) row[4 * k + e] = acc[ii][k][e];
      transpose4(row[e], row[4 + e], row[8 + e], row[12 + e]);
    }
    const long long i = (long long)i0 + (wm * TM + ii) * 16 + r;
    if (i >= p.M) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = p.N - j - 32 * h;
      if (n <= 0) continue;
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = row[8 * h + q];
      if (whole) put8<DT_F32, FORM, ACT>(E, bias[h], out, i * p.N + j + 32 * h, n, ahead[ii][h], v);
      else put8<DT_F32, FORM_WEIGHT, ACT_NONE>(E, none, part, (slice * p.M + i) * p.N + j + 32 * h, n, ahead[ii][h], v);
    }
  }
}

// What a launch takes: `fixed` us and, of each 32 terms, `step` us for the first workgroup on a
// CU and `more` for each further one: the matrix pipes are shared.  Measured, us: 64 x 64
// outputs of 1024 terms 69.9 and 24.4 with tiles of 128 and 64; 512^3 37.9, 14.4; 1024^3 69.8,
// 25.8; 2048 x 1024 of 512 39.1, 23.7; 2048^3 139, 145; 4096 x 4096 of 1024 256, 280.  Cut
// sums: 64 x 512 of 4096 with tiles of 64 in 1, 4, 8, 16, 32 slices 86, 27.5, 18.3, 15.6, 17.1;
// 512 x 512 of 8192 169, 51.4, 47.2, 49.0, 54.9; 1024^3 in 1 and 2 slices 25.8 and 30.0.
struct Cost {
  int kernel, b;
  double fixed, step, more;
};
constexpr Cost kCost[] = {{LIN_128, 128, 2.0, 2.05, 1.95}, {LIN_64, 64, 1.5, 0.65, 0.53}};

}  // namespace

bool linear_f32_plan(int form, long long M, int N, long long L, LinearPlan *p) {
  // 32-bit offsets inside a tile's rows, and its first row's and column's numbers
  const long long la = row_length(form, true, M, N, L), lb = row_length(form, false, M, N, L);
  if (la >= (1LL << 22) || lb >= (1LL << 22) || M >= (1LL << 31) - 256) return false;
  double best = 1e30;
  for (const Cost &c : kCost) {
    const long long tm = (M + c.b - 1) / c.b, tn = (N + c.b - 1) / c.b, tiles = tm * tn, steps = (L + BK - 1) / BK;
    const long long chain = std::max(1LL, std::min((L + kChain - 1) / kChain, (1LL << 28) / (M * N)));
    for (long long s = 1; s <= 64; s = s < 4 ? s + 1 : s * 2) {
      const long long slices = std::max(s, chain);
      if (s > 1 && (steps / s < 4 || slices * M * N > (1LL << 28) || tiles * s > 8 * kCUs)) break;
      const long long rounds = (tiles * slices + kCUs - 1) / kCUs;
      double t = c.fixed + (c.step + (rounds - 1) * c.more) * ((steps + slices - 1) / slices);
      if (slices > 1) t += 3.5 + 0.15 * slices + slices * (double)M * N * 8 / 4e6;
      if (t < best) {
        best = t;
        const long long per = ((L + slices - 1) / slices + BK - 1) / BK * BK;
        *p = LinearPlan{M, L, N, c.kernel, (int)tm, (int)tn, (int)((L + per - 1) / per), per, la, lb, 0, 0};
      }
    }
  }
  return true;
}

namespace {
template <int FORM>
hipError_t launch_form(const LinearPlan &p, const float *A, const float *B, const LinearEpilogue &E, void *out, float *part,
                       float *db, hipStream_t st) {
  const long long per_xcd = ((long long)p.tm * p.tn * p.slices + 7) / 8;
  with_act(E.act, [&](auto a) {
    constexpr int ACT = FORM == FORM_WEIGHT ? (int)ACT_NONE : decltype(a)::value;
    const dim3 grid = long_grid(8 * per_xcd), block(NT);
    auto run = [&](auto k, auto v) {
      hipLaunchKernelGGL((product_kernel<decltype(k)::value, FORM, ACT, decltype(v)::value>), grid, block, 0, st, p, per_xcd, A, B,
                         E, out, part, db);
    };
    constexpr std::integral_constant<int, LIN_128> big;
    constexpr std::integral_constant<int, LIN_64> small;
    constexpr std::integral_constant<int, 4> pieces;
    constexpr std::integral_constant<int, 1> values;
    const bool whole = p.lda % 4 == 0 && p.ldb % 4 == 0;
    if (p.kernel == LIN_128) whole ? run(big, pieces) : run(big, values);
    else whole ? run(small, pieces) : run(small, values);
  });
  return hipGetLastError();
}
}  // namespace

hipError_t launch_linear_f32(int form, const LinearPlan &p, const void *A, const void *B, const LinearEpilogue &E, void *out,
                             float *part, float *db, hipStream_t st) {
  const float *a = (const float *)A, *b = (const float *)B;
  if (form == FORM_FWD) return launch_form<FORM_FWD>(p, a, b, E, out, part, db, st);
  if (form == FORM_DATA) return launch_form<FORM_DATA>(p, a, b, E, out, part, db, st);
  return launch_form<FORM_WEIGHT>(p, a, b, E, out, part, db, st);
}

}  // namespace cf
