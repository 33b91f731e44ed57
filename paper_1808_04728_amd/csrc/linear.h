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
};
enum : int { LIN_ANY = 0, LIN_256 = 1, LIN_128 = 2, LIN_64 = 3 };

// A grid's x dimension holds fewer than 2^32 threads: workgroups past 2^22 go on in y.
inline dim3 long_grid(long long n) {
  const long long x = std::min(n, 1LL << 22);
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ long long long_index() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

// The bf16 kernels (linear_bf16.hip): rows of whole 16-byte pieces.  part: the slices' sums
// [slices][M][N] where there are several.
bool linear_bf16_plan(int form, long long M, int N, long long L, LinearPlan *p);
hipError_t launch_linear_bf16(int form, const LinearPlan &p, const void *A, const void *B, const LinearEpilogue &E, void *out,
                              float *part, hipStream_t st);

}  // namespace cf
