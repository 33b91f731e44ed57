// linear_bf16.hip -- bf16 matrix products on tiles of up to 256 x 256 (gfx950).
//
// C[i][j] = sum_l A(i, l) B(l, j).  A workgroup's step brings BK terms of its tile's rows of
// both factors into LDS, 16 bytes a lane straight from memory (buffer loads to LDS, whose
// range check gives zeros past a tensor's end).  A factor with the sum's axis innermost lies
// there by rows of BK terms and is read 8 terms a lane; one with the sum's axis outermost
// lies as it is in memory, by terms, 64 columns a line, and is read with the transposing
// loads.  Both orders are swizzled so that the reads of a fragment touch all banks.
//
// The matrix instructions take B's columns as their rows: a lane's four results are then
// four neighbours of a row of C, and exchanging registers between the four lanes of a row
// leaves each with sixteen, so the epilogue reads and writes 16 bytes a lane.
//
// Large products are bound by the matrix cores, whose clock falls under their load: 8192^3 in
// 745 us (1.48 PFLOP/s; a plain library product 1.37, 1.60 with its right factor transposed).
// Those with few terms and wide outputs are bound by their epilogues' memory and arithmetic: a
// compute unit holds one 256 x 256 tile and runs no products meanwhile (32768 x 1024 x 4096
// with GELU and z 321 us, without either 251).  Half the outputs in each of two workgroups a
// compute unit, loads two steps further ahead from steps of 32 terms, and halves of the waves
// taking turns at LDS and the matrix cores were all slower.

#include "linear.h"

namespace cf {
namespace {

typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef short v8i16_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4i16_t lds_v4i16_t;

// A tile: WM x WN waves of TM x TN instruction tiles of 16 x 16; NS steps of 64 terms in LDS.
template <int KERNEL> struct Tile;
template <> struct Tile<LIN_256> {
  static constexpr int BM = 256, BN = 256, WM = 2, WN = 4, NS = 2, WAVES = 2;
};
template <> struct Tile<LIN_128> {
  static constexpr int BM = 128, BN = 128, WM = 2, WN = 2, NS = 2, WAVES = 2;
};
template <> struct Tile<LIN_64> {
  static constexpr int BM = 64, BN = 64, WM = 4, WN = 1, NS = 3, WAVES = 3;
};

constexpr int BK = 64, KK = BK / 32;

// The rows r0 .. r0 + ROWS - 1 of a factor, a step of BK terms at a time.  KC: the sum's axis
// is innermost.  Pieces past the rows' or the sum's end read as zeros: their offset is out of
// the buffer's range.
template <bool KC, bool COLS, int ROWS, int NT> struct Loader {
  static constexpr int BYTES = ROWS * BK * 2, N = BYTES / 16 / NT;
  static_assert(BYTES % (16 * NT) == 0, "whole loads");
  static_assert(NT / 8 % 64 == 0 || NT / 8 == 32, "a lane's pieces are of one term, or of two in turn");
  // bit 5 of a lane's term (of its odd pieces) where a load is 32 rows
  static constexpr int FLIP = NT / 8 == 32 && (!KC || COLS) ? 32 : 0;
  const char *base;
  long long advance;  // bytes of a step
  uint32_t off[N];
  int term;  // the lane's first piece's (first) term of a step
  __device__ __forceinline__ Loader(const uint16_t *p, long long rows, long long ld, int r0, long long k0) {
    base = (const char *)(p + (KC ? r0 * ld + k0 : k0 * ld + r0));
    advance = KC ? BK * 2 : BK * ld * 2;
    const long long have = rows - r0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = i * NT + threadIdx.x;
      if constexpr (KC) {
        const int row = id / (BK / 8), piece = id % (BK / 8);
        const int c = piece ^ swizzle<COLS>(row);
        off[i] = row < have ? (uint32_t)(row * (ld * 2)) + c * 16 : kOut;
        if (i == 0) term = c * 8;
      } else {
        const int sub = id / (BK * 8), row = id / 8 % BK, piece = id & 7;
        const int x = ((row >> 1) & 1) | (((row >> 3) & 1) << 1), c = piece ^ (COLS ? x : 2 * x);
        off[i] = sub * 64 + c * 8 < have ? (uint32_t)(row * (ld * 2)) + sub * 128 + c * 16 : kOut;
        if (i == 0) term = row;
      }
    }
  }
  // Load i of the next step to `stage` (bytes from the LDS's start); `rest` terms are left.
  // Written out because the compiler, which cannot tell the stages apart in the transposing
  // reads, would wait for every load before each of them; the waits are the kernel's own.
  __device__ __forceinline__ void load(int i, int wave, uint32_t stage, int rest) const {
    const uint32_t o = (term ^ (i % 2 * FLIP)) < rest ? off[i] : kOut;
    const u32x4_t r = {(uint32_t)(uintptr_t)base, (uint32_t)((uintptr_t)base >> 32) & 0xffffu, 0x7ffffff0u, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(stage + (uint32_t)(i * NT + wave * 64) * 16), "v"(o), "s"(r)
                 : "memory");
  }
  __device__ __forceinline__ void next() { base += advance; }
};

// A lane's place in the fragments of 16 rows and 32 terms.  Fragment t of A has rows 16 t + r;
// fragment t of B (COLS) has, of every 64 columns, 8 t' + r (r < 8) and 32 + 8 t' + r - 8, t' =
// t % 4: after the epilogue's exchange a lane then has twice eight columns, and four lanes
// eight by eight 64 neighbouring bytes of a row of C.
template <bool KC, bool COLS> struct Reader {
  int lane_off, swz;
  __device__ __forceinline__ Reader() {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    if constexpr (KC) {
      const int row = COLS ? (r & 7) + 32 * (r >> 3) : r;
      lane_off = row * BK * 2;
      swz = swizzle<COLS>(row);
    } else {
      lane_off = (8 * g + (r >> 2)) * 128 + (COLS ? (r & 1) * 8 + (r & 2) * 32 : (r & 3) * 8);
      swz = ((r >> 3) & 1) | ((g & 1) << 1);
    }
  }
  // fragment t of the stage, terms 32 k ..
  __device__ __forceinline__ bf16x8_t frag(const unsigned char *stage, int t, int k) const {
    if constexpr (KC) {
      const int g = (threadIdx.x & 63) >> 4, row = COLS ? t / 4 * 64 + t % 4 * 8 : t * 16;
      return *reinterpret_cast<const bf16x8_t *>(stage + lane_off + row * BK * 2 + (((4 * k + g) ^ swz) << 4));
    } else {
      const unsigned char *p = stage + (t >> 2) * (BK * 128) + k * 32 * 128 + lane_off + (((t & 3) ^ swz) << (COLS ? 4 : 5));
      const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)p);
      const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)(p + 512));
      const v8i16_t v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(bf16x8_t, v);
    }
  }
};

template <class C> constexpr int threads_of() { return 64 * C::WM * C::WN; }

template <int KERNEL, int FORM, int ACT>
__global__ __launch_bounds__(threads_of<Tile<KERNEL>>(), Tile<KERNEL>::WAVES) void product_kernel(
    LinearPlan p, long long per_xcd, const uint16_t *A, const uint16_t *B, LinearEpilogue E, void *out, float *part,
    float *db) {
  using C = Tile<KERNEL>;
  constexpr int NT = threads_of<C>(), TM = C::BM / C::WM / 16, TN = C::BN / C::WN / 16;
  static_assert(TN % 4 == 0, "a lane's row of the epilogue is sixteen columns of 64");
  constexpr int AB = C::BM * BK * 2, STAGE = AB + C::BN * BK * 2;
  // (the large tile leaves 32 KB free)
  constexpr bool PHI = KERNEL == LIN_256 && FORM == FORM_FWD && ACT == ACT_GELU;
  constexpr bool SLOPES = KERNEL == LIN_256 && FORM == FORM_DATA && (ACT == ACT_SILU || ACT == ACT_GELU);
  __shared__ __attribute__((aligned(16))) unsigned char lds[C::NS * STAGE + (SLOPES ? SlopeTable::BYTES : PHI ? PhiTable::BYTES : 0)];

  // the workgroups of an XCD (every eighth) take neighbouring tiles, eight tiles down before
  // one across: 32 at a time read 8 + 4 tiles' factors through its L2
  const long long index = long_index(), job = (index & 7) * per_xcd + (index >> 3);
  const long long tiles = (long long)p.tm * p.tn;
  if (job >= tiles * p.slices) return;
  const long long slice = job / tiles;
  const int t = (int)(job % tiles), group = t / (8 * p.tn), in = t % (8 * p.tn), high = min(8, p.tm - 8 * group);
  const int ti = 8 * group + in % high, tj = in / high;
  const int j0 = tj * C::BN;
  const int i0 = ti * C::BM;
  const long long k0 = slice * p.per, k1 = min(k0 + p.per, p.L);
  const int steps = k1 > k0 ? (int)((k1 - k0 + BK - 1) / BK) : 0;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  Loader<Form<FORM>::AK, false, C::BM, NT> la(A, p.M, p.lda, i0, k0);
  Loader<Form<FORM>::BK, true, C::BN, NT> lb(B, p.N, p.ldb, j0, k0);
  const Reader<Form<FORM>::AK, false> ra;
  const Reader<Form<FORM>::BK, true> rb;
  constexpr int LOADS = decltype(la)::N + decltype(lb)::N;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t *)lds;
  int rest = (int)(p.L - k0);  // terms from the next step to load on
  constexpr int NA = decltype(la)::N;
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

  // While the matrix instructions of 32 terms run, the fragments of the next 32 come from
  // LDS; one barrier a step, in front of its last 32 terms: by then every wave has read all
  // of the step's stage, which the loads of the step NS further overwrite, and has waited for
  // its own loads of the next.  (Steps past the end load zeros.)
  bf16x8_t fb[2][TN], fa[2][TM];
  auto read = [&](int f, int q, const unsigned char *stage, int k) {  // fragment q of the 32 terms k
    if (q < TN) fb[f][q] = rb.frag(stage + AB, wn * TN + q, k);
    else fa[f][q - TN] = ra.frag(stage, wm * TM + q - TN, k);
  };
  // The matrix instructions of fragments f, the reads of the others and `loads` loads between
  // them: a load's issue takes its wave sixteen cycles and more, in front of all matrix
  // instructions a third of their time.
  constexpr int EARLY = TM > 2 ? TM - 2 : TM;  // the reads are under way this many rows before the end
  const int turns = FORM == FORM_WEIGHT ? db_turns(p) : 0;
  const bool sum_db = FORM == FORM_WEIGHT && db && wm == 0 && ti < turns;
  ColumnSums<TN> sums(sum_db, ti, turns);
  auto half = [&](int f, const unsigned char *rs, int k, auto loads, int ls) {
    if constexpr (FORM == FORM_WEIGHT) {
      if (sums.mine) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const u32x4_t b = __builtin_bit_cast(u32x4_t, fb[f][j]);
#pragma unroll
          for (int q = 0; q < 4; ++q) sums.s[j] += __uint_as_float(b[q] << 16) + __uint_as_float(b[q] & 0xffff0000u);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int q = i * (TM + TN) / EARLY; q < (i + 1) * (TM + TN) / EARLY && q < TM + TN; ++q) read(1 - f, q, rs, k);
#pragma unroll
      for (int q = i * decltype(loads)::value / TM; q < (i + 1) * decltype(loads)::value / TM; ++q) load(q, ls);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[f][j], fa[f][i], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
#pragma unroll
  for (int n = 0; n < C::NS; ++n) {
#pragma unroll
    for (int q = 0; q < LOADS; ++q) load(q, n);
    next();
  }
  // (a step's barrier is in front of the tables' use)
  if constexpr (SLOPES) SlopeTable::fill<ACT>(lds + C::NS * STAGE, E.alpha);
  if constexpr (PHI) PhiTable::fill(lds + C::NS * STAGE);
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
  const int r = lane & 15, g = lane >> 4;
  const bool whole = p.slices == 1;
  const float none[8] = {};
#pragma unroll
  for (int jj = 0; jj < TN; jj += 4) {
    const int j = j0 + (wn * TN + jj) * 16 + 8 * g;
    float bias[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_bias<FORM>(E, j + 32 * h, p.N, bias[h]);
    Eight<DT_BF16> ahead[TM][2];
    if (whole) {
#pragma unroll
      for (int ii = 0; ii < TM; ++ii) {
        const long long i = (long long)i0 + (wm * TM + ii) * 16 + r;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n = p.N - j - 32 * h;
          if (i < p.M && n > 0) fetch8<DT_BF16, FORM, ACT>(E, i * p.N + j + 32 * h, n, ahead[ii][h]);
        }
      }
    }
#pragma unroll
    for (int ii = 0; ii < TM; ++ii) {
      float row[16];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int k = 0; k < 4; ++k) row[4 * k + e] = acc[ii][jj + k][e];
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
        if (whole) put8<DT_BF16, FORM, ACT, SLOPES || PHI>(E, bias[h], out, i * p.N + j + 32 * h, n, ahead[ii][h], v, lds + C::NS * STAGE);
        else put8<DT_BF16, FORM_WEIGHT, ACT_NONE>(E, none, part, (slice * p.M + i) * p.N + j + 32 * h, n, ahead[ii][h], v);
      }
    }
  }
}

// What a launch takes: `fixed` us of a workgroup and, of each 64 terms, `alone` and, the more
// of the `at_once` workgroups that the card holds there are, up to `shared` more.  Measured,
// us: 64 x 64 outputs of 1024 terms 22.8, 12.4, 8.0 with tiles of 256, 128, 64; 1024^3 25.4,
// 13.2, 8.5; 1536^3 35.1, 20.4, 17.5; 8192 x 1024 of 1024 terms 30.9, 23.3, 32.5; 2048^3 44.6,
// 28.4, 30.4; 4096 x 4096 of 1024 36.4, 43.4, 64.7.  Cut sums: 64 x 512 of 4096 with tiles of
// 64 in 1, 4, 8, 16 slices 20.7, 12.1, 11.1, 12.0; 512 x 512 of 8192 37.7, 17.9, 18.3, 22.3;
// 1024^3 in 1 and 2 slices 8.5 and 14.3.
struct Cost {
  int kernel, b, at_once;
  double fixed, alone, shared;
};
constexpr Cost kCost[] = {
    {LIN_256, 256, kCUs, 6.0, 1.05, 0.50}, {LIN_128, 128, 2 * kCUs, 3.0, 0.55, 0.45}, {LIN_64, 64, 3 * kCUs, 1.5, 0.26, 0.34}};

}  // namespace

bool linear_bf16_plan(int form, long long M, int N, long long L, LinearPlan *p) {
  // 32-bit offsets inside a tile's rows, and its first row's and column's numbers.  Rows that
  // are not whole 16-byte pieces are copied to such ones first: a copy of both factors costs
  // what it reads and writes, and a kernel that loaded them value by value ten times as much.
  const long long la = row_length(form, true, M, N, L), lb = row_length(form, false, M, N, L);
  if (la >= (1LL << 22) || lb >= (1LL << 22) || M >= (1LL << 31) - 256) return false;
  double best = 1e30;
  for (const Cost &c : kCost) {
    const long long tm = (M + c.b - 1) / c.b, tn = (N + c.b - 1) / c.b, tiles = tm * tn, steps = (L + 63) / 64;
    const long long chain = std::max(1LL, std::min((L + kChain - 1) / kChain, (1LL << 28) / (M * N)));
    for (long long s = 1; s <= 64; s = s < 4 ? s + 1 : s * 2) {
      const long long slices = std::max(s, chain);
      if (s > 1 && (steps / s < 4 || slices * M * N > (1LL << 28) || tiles * s > 4 * kCUs)) break;
      const double full = (double)(tiles * slices) / c.at_once, step = c.alone + c.shared * std::min(1.0, full);
      // (one workgroup a CU goes in whole rounds, several make room for the next one by one)
      const double rounds = c.at_once == kCUs ? std::ceil(full) : std::max(1.0, full);
      double t = rounds * (c.fixed + step * ((steps + slices - 1) / slices));
      if (slices > 1) t += 3.5 + 0.15 * slices + slices * (double)M * N * 8 / 4e6;
      if (t < best) {
        best = t;
        const long long per = ((L + slices - 1) / slices + 63) / 64 * 64;
        *p = LinearPlan{M, L, N, c.kernel, (int)tm, (int)tn, (int)((L + per - 1) / per), per,
                       (la + 7) / 8 * 8, (lb + 7) / 8 * 8, la % 8 != 0, lb % 8 != 0};
      }
    }
  }
  return true;
}

namespace {
template <int FORM>
hipError_t launch_form(const LinearPlan &p, const uint16_t *A, const uint16_t *B, const LinearEpilogue &E, void *out, float *part,
                       float *db, hipStream_t st) {
  const long long per_xcd = ((long long)p.tm * p.tn * p.slices + 7) / 8;
  with_act(E.act, [&](auto a) {
    constexpr int ACT = FORM == FORM_WEIGHT ? (int)ACT_NONE : decltype(a)::value;
    auto run = [&](auto k) {
      constexpr int KERNEL = decltype(k)::value;
      hipLaunchKernelGGL((product_kernel<KERNEL, FORM, ACT>), long_grid(8 * per_xcd), dim3(threads_of<Tile<KERNEL>>()), 0, st, p,
                         per_xcd, A, B, E, out, part, db);
    };
    if (p.kernel == LIN_256) run(std::integral_constant<int, LIN_256>{});
    else if (p.kernel == LIN_128) run(std::integral_constant<int, LIN_128>{});
    else run(std::integral_constant<int, LIN_64>{});
  });
  return hipGetLastError();
}
}  // namespace

hipError_t launch_linear_bf16(int form, const LinearPlan &p, const void *A, const void *B, const LinearEpilogue &E, void *out,
                              float *part, float *db, hipStream_t st) {
  const uint16_t *a = (const uint16_t *)A, *b = (const uint16_t *)B;
  if (form == FORM_FWD) return launch_form<FORM_FWD>(p, a, b, E, out, part, db, st);
  if (form == FORM_DATA) return launch_form<FORM_DATA>(p, a, b, E, out, part, db, st);
  return launch_form<FORM_WEIGHT>(p, a, b, E, out, part, db, st);
}

}  // namespace cf
