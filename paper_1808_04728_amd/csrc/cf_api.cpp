// cf_api.cpp -- the C ABI (include/cosmoflow.h): host-side argument
// validation, geometry, and dispatch to the gfx950 kernel launchers.
//
// Every check runs on the host before anything is launched, so a rejected
// call touches neither the device nor the outputs.

#include "../../include/cosmoflow.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "activation.h"
#include "cf_common.h"
#include "cf_kernels.h"

namespace {

thread_local std::string g_last_error;

cf_status fail(cf_status code, const std::string &msg) {
  g_last_error = msg;
  return code;
}

cf_status ok() {
  g_last_error.clear();
  return CF_OK;
}

bool debug_sync() {
  static int v = [] {
    const char *e = std::getenv("CF_DEBUG_SYNC");
    return (e && e[0] && e[0] != '0') ? 1 : 0;
  }();
  return v != 0;
}

cf_status finish(hipError_t e, hipStream_t st, const char *what) {
  if (e == hipSuccess && debug_sync()) e = hipStreamSynchronize(st);
  if (e != hipSuccess)
    return fail(CF_ERR_LAUNCH, std::string(what) + ": " + hipGetErrorString(e));
  return ok();
}

size_t elem_size(int dtype) { return dtype == CF_BF16 ? 2 : 4; }

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + nb && b0 < a0 + na;
}

constexpr long long kMaxRows = (1LL << 31) - 1;

// Validate a convolution descriptor and resolve its geometry.
cf_status resolve(const cf_conv3d_desc *d, cf::ConvShape *s) {
  if (!d) return fail(CF_ERR_INVALID_ARG, "desc is NULL");
  if (d->n < 0) return fail(CF_ERR_INVALID_ARG, "batch n must be >= 0");
  if (d->d <= 0 || d->h <= 0 || d->w <= 0)
    return fail(CF_ERR_INVALID_ARG, "spatial extents d, h, w must be > 0");
  if (d->c_in <= 0 || d->c_out <= 0) return fail(CF_ERR_INVALID_ARG, "channels must be > 0");
  if (d->kd <= 0 || d->kh <= 0 || d->kw <= 0) return fail(CF_ERR_INVALID_ARG, "kernel extents must be > 0");
  if (d->sd <= 0 || d->sh <= 0 || d->sw <= 0) return fail(CF_ERR_INVALID_ARG, "strides must be > 0");
  if (d->pad != CF_PAD_SAME_TF && d->pad != CF_PAD_VALID) return fail(CF_ERR_INVALID_ARG, "unknown pad mode");
  if (d->dtype != CF_F32 && d->dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  const int in[3] = {d->d, d->h, d->w}, k[3] = {d->kd, d->kh, d->kw}, st[3] = {d->sd, d->sh, d->sw};
  int out[3], pb[3];
  for (int a = 0; a < 3; ++a) {
    if (d->pad == CF_PAD_SAME_TF) {
      out[a] = (in[a] + st[a] - 1) / st[a];
      long long tot = (long long)(out[a] - 1) * st[a] + k[a] - in[a];
      if (tot < 0) tot = 0;
      pb[a] = (int)(tot / 2);
    } else {
      if (k[a] > in[a]) return fail(CF_ERR_INVALID_ARG, "VALID convolution: kernel larger than input");
      out[a] = (in[a] - k[a]) / st[a] + 1;
      pb[a] = 0;
    }
  }
  const long long taps = (long long)k[0] * k[1] * k[2];
  if (taps * d->c_in >= kMaxRows || taps * d->c_out >= kMaxRows)
    return fail(CF_ERR_INVALID_ARG, "kernel volume x channels overflows 32 bits");
  const long long vin = (long long)d->n * in[0] * in[1] * in[2];
  const long long vout = (long long)d->n * out[0] * out[1] * out[2];
  if (vin >= kMaxRows || vout >= kMaxRows) return fail(CF_ERR_INVALID_ARG, "too many voxels (>= 2^31)");
  s->n = d->n; s->d = in[0]; s->h = in[1]; s->w = in[2];
  s->ci = d->c_in; s->co = d->c_out;
  s->kd = k[0]; s->kh = k[1]; s->kw = k[2];
  s->sd = st[0]; s->sh = st[1]; s->sw = st[2];
  s->pd = pb[0]; s->ph = pb[1]; s->pw = pb[2];
  s->od = out[0]; s->oh = out[1]; s->ow = out[2];
  s->dtype = d->dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32;
  return CF_OK;
}

struct Sizes {
  size_t x, w, z;
};

Sizes conv_bytes(const cf::ConvShape &s) {
  const size_t es = s.dtype == cf::DT_BF16 ? 2 : 4;
  Sizes r;
  r.x = (size_t)s.n * s.d * s.h * s.w * s.ci * es;
  r.w = (size_t)s.kd * s.kh * s.kw * s.ci * s.co * es;
  r.z = (size_t)s.n * s.od * s.oh * s.ow * s.co * es;
  return r;
}

cf_status check_ptrs(std::initializer_list<const void *> ptrs) {
  for (const void *p : ptrs) {
    if (!p) return fail(CF_ERR_INVALID_ARG, "NULL tensor pointer");
    if (!aligned16(p)) return fail(CF_ERR_ALIGNMENT, "tensor pointer not 16-byte aligned");
  }
  return CF_OK;
}

}  // namespace

namespace {
// runs `call` with the fixed-order column sums recorded instead of launched
template <class F>
cf_status deferred(cf_reduction *pending, int32_t *npending, F call) {
  if (!pending || !npending) return fail(CF_ERR_INVALID_ARG, "pending / npending is NULL");
  *npending = 0;
  cf::SumCollector col{};
  cf::set_sum_collector(&col);
  const cf_status r = call();
  cf::set_sum_collector(nullptr);
  if (r != CF_OK) return r;
  for (int i = 0; i < col.n; ++i)
    pending[i] = cf_reduction{col.job[i].part, col.job[i].out, col.job[i].rows, col.job[i].cols};
  *npending = col.n;
  return CF_OK;
}
}  // namespace

namespace {
// validates the group table and fills the kernel's plan; chunks = 0 when every group is empty
cf_status adam_plan(int32_t ngroups, const int64_t *offsets, cf::OptGroups *G, int *chunks) {
  if (ngroups < 0) return fail(CF_ERR_INVALID_ARG, "adam_larc: ngroups must be >= 0");
  if (ngroups > CF_ADAM_MAX_GROUPS) return fail(CF_ERR_UNSUPPORTED, "adam_larc: more than CF_ADAM_MAX_GROUPS groups");
  if (!offsets) return fail(CF_ERR_INVALID_ARG, "adam_larc: offsets is NULL");
  if (offsets[0] < 0) return fail(CF_ERR_INVALID_ARG, "adam_larc: negative offset");
  for (int l = 0; l < ngroups; ++l) {
    if (offsets[l + 1] < offsets[l]) return fail(CF_ERR_INVALID_ARG, "adam_larc: offsets must be non-decreasing");
    if (offsets[l] % 4 != 0) return fail(CF_ERR_ALIGNMENT, "adam_larc: a group start is not a multiple of 4");
  }
  if (offsets[ngroups] >= (1LL << 40)) return fail(CF_ERR_INVALID_ARG, "adam_larc: too many elements");
  static_assert(cf::kOptMaxGroups == CF_ADAM_MAX_GROUPS, "group table size");
  std::vector<long long> off(offsets, offsets + ngroups + 1);
  *chunks = cf::plan_opt_groups(ngroups, off.data(), G);
  return CF_OK;
}
}  // namespace

extern "C" {

const char *cf_version(void) { return "cosmoflow-gfx950 0.1.0"; }

const char *cf_last_error(void) { return g_last_error.c_str(); }

cf_status cf_conv3d_out_shape(const cf_conv3d_desc *desc, int32_t out_dhw[3]) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  if (!out_dhw) return fail(CF_ERR_INVALID_ARG, "out_dhw is NULL");
  out_dhw[0] = s.od;
  out_dhw[1] = s.oh;
  out_dhw[2] = s.ow;
  return ok();
}

cf_status cf_conv3d_fwd(const cf_conv3d_desc *desc, const void *x, const void *w, void *z,
                        void *stream) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  if (s.n == 0) return ok();
  if ((r = check_ptrs({x, w, z})) != CF_OK) return r;
  Sizes b = conv_bytes(s);
  if (overlap(z, b.z, x, b.x) || overlap(z, b.z, w, b.w))
    return fail(CF_ERR_ALIAS, "conv3d_fwd: z overlaps x or W");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_conv_fwd(s, x, w, z, st), st, "cf_conv3d_fwd");
}

// check_only: validate every argument and return without launching
static cf_status bwd_data(const cf_conv3d_desc *desc, const void *dz, const void *w, void *dx, void *stream,
                          bool check_only) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  if (s.n == 0) return ok();
  if ((r = check_ptrs({dz, w, dx})) != CF_OK) return r;
  Sizes b = conv_bytes(s);
  if (overlap(dx, b.x, dz, b.z) || overlap(dx, b.x, w, b.w))
    return fail(CF_ERR_ALIAS, "conv3d_bwd_data: dx overlaps dz or W");
  if (check_only) return CF_OK;
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_conv_bwd_data(s, dz, w, dx, st), st, "cf_conv3d_bwd_data");
}

cf_status cf_conv3d_bwd_data(const cf_conv3d_desc *desc, const void *dz, const void *w, void *dx,
                             void *stream) {
  return bwd_data(desc, dz, w, dx, stream, false);
}

size_t cf_conv3d_bwd_weight_workspace_size(const cf_conv3d_desc *desc) {
  cf::ConvShape s;
  std::string keep = g_last_error;
  if (resolve(desc, &s) != CF_OK) {
    g_last_error = keep;
    return 0;
  }
  if (s.n == 0) return 0;
  return cf::conv_bwd_weight_workspace(s);
}

static cf_status bwd_weight(const cf_conv3d_desc *desc, const void *x, const void *dz, float *dw, void *ws,
                            size_t ws_bytes, void *stream, bool check_only) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  hipStream_t st = (hipStream_t)stream;
  Sizes b = conv_bytes(s);
  const size_t dw_bytes = (size_t)s.kd * s.kh * s.kw * s.ci * s.co * sizeof(float);
  if (s.n == 0) {
    if ((r = check_ptrs({dw})) != CF_OK) return r;
    if (check_only) return CF_OK;
    // the sum over an empty batch is zero
    return finish(cf::launch_fill_zero(dw, (long long)(dw_bytes / sizeof(float)), st), st,
                  "cf_conv3d_bwd_weight");
  }
  if ((r = check_ptrs({x, dz, dw})) != CF_OK) return r;
  const size_t need = cf::conv_bwd_weight_workspace(s);
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(CF_ERR_WORKSPACE, "conv3d_bwd_weight: workspace smaller than cf_conv3d_bwd_weight_workspace_size()");
  if (ws && !aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  if (overlap(dw, dw_bytes, x, b.x) || overlap(dw, dw_bytes, dz, b.z))
    return fail(CF_ERR_ALIAS, "conv3d_bwd_weight: dW overlaps x or dz");
  if (overlap(ws, need, x, b.x) || overlap(ws, need, dz, b.z) || overlap(ws, need, dw, dw_bytes))
    return fail(CF_ERR_ALIAS, "conv3d_bwd_weight: workspace overlaps a tensor");
  if (check_only) return CF_OK;
  return finish(cf::launch_conv_bwd_weight(s, x, dz, dw, ws, st), st, "cf_conv3d_bwd_weight");
}

cf_status cf_conv3d_bwd_weight(const cf_conv3d_desc *desc, const void *x, const void *dz, float *dw,
                               void *ws, size_t ws_bytes, void *stream) {
  return bwd_weight(desc, x, dz, dw, ws, ws_bytes, stream, false);
}

cf_status cf_conv3d_bwd(const cf_conv3d_desc *desc, const void *x, const void *dz, const void *w, float *dw,
                        void *dx, void *ws, size_t ws_bytes, void *stream) {
  cf_status r = bwd_weight(desc, x, dz, dw, ws, ws_bytes, stream, true);
  if (r != CF_OK) return r;
  if ((r = bwd_data(desc, dz, w, dx, stream, true)) != CF_OK) return r;
  cf::ConvShape s;
  resolve(desc, &s);
  if (s.n == 0) return bwd_weight(desc, x, dz, dw, ws, ws_bytes, stream, false);  // dW = 0, dx empty
  const size_t dxb = conv_bytes(s).x, dwb = (size_t)s.kd * s.kh * s.kw * s.ci * s.co * sizeof(float);
  if (overlap(dx, dxb, dw, dwb) || overlap(dx, dxb, x, conv_bytes(s).x) ||
      overlap(dx, dxb, ws, cf::conv_bwd_weight_workspace(s)))
    return fail(CF_ERR_ALIAS, "cf_conv3d_bwd: dx overlaps x, dW or the workspace");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_conv_bwd(s, x, dz, w, dw, dx, ws, st), st, "cf_conv3d_bwd");
}

static_assert(cf::kNoallocScratchBytes == CF_NOALLOC_SCRATCH_BYTES, "scratch region size");

cf_status cf_conv3d_bwd_weight_noalloc(const cf_conv3d_desc *desc, const void *x, const void *dz, float *dw,
                                       void *stream) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  const size_t need = s.n == 0 ? 0 : cf::conv_bwd_weight_workspace(s);
  if (need > cf::kNoallocScratchBytes)
    return fail(CF_ERR_UNSUPPORTED, "cf_conv3d_bwd_weight_noalloc: the split reduction needs " +
                                        std::to_string(need) + " bytes of partials, more than the " +
                                        std::to_string(cf::kNoallocScratchBytes) +
                                        "-byte library scratch region (use cf_conv3d_bwd_weight with a workspace)");
  void *ws = nullptr;
  if (need > 0) {
    const hipError_t e = cf::noalloc_scratch(&ws);
    if (e != hipSuccess)
      return fail(CF_ERR_LAUNCH, std::string("cf_conv3d_bwd_weight_noalloc: scratch region: ") + hipGetErrorString(e));
  }
  return cf_conv3d_bwd_weight(desc, x, dz, dw, ws, need, stream);
}

cf_status cf_bias_lrelu_fwd(int64_t nvox, int32_t c, int32_t dtype, const void *z, const float *bias,
                            float alpha, void *y, void *stream) {
  if (nvox < 0) return fail(CF_ERR_INVALID_ARG, "nvox must be >= 0");
  if (c <= 0) return fail(CF_ERR_INVALID_ARG, "channels must be > 0");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  if (!std::isfinite(alpha)) return fail(CF_ERR_INVALID_ARG, "alpha must be finite");
  if (nvox == 0) return ok();
  cf_status r;
  if ((r = check_ptrs({z, y})) != CF_OK) return r;
  if (!bias) return fail(CF_ERR_INVALID_ARG, "bias is NULL");
  const size_t bytes = (size_t)nvox * c * elem_size(dtype);
  if (y != z && overlap(y, bytes, z, bytes))
    return fail(CF_ERR_ALIAS, "bias_lrelu_fwd: y partially overlaps z");
  if (overlap(y, bytes, bias, (size_t)c * 4)) return fail(CF_ERR_ALIAS, "bias_lrelu_fwd: y overlaps bias");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_bias_lrelu_fwd(nvox, c, dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32, z, bias,
                                          alpha, y, st),
                st, "cf_bias_lrelu_fwd");
}

size_t cf_bias_lrelu_bwd_workspace_size(int64_t nvox, int32_t c) {
  if (nvox <= 0 || c <= 0) return 0;
  return cf::bias_lrelu_bwd_workspace(nvox, c);
}

cf_status cf_bias_lrelu_bwd(int64_t nvox, int32_t c, int32_t dtype, const void *dy, const void *y,
                            float alpha, void *dz, float *db, void *ws, size_t ws_bytes,
                            void *stream) {
  if (nvox < 0) return fail(CF_ERR_INVALID_ARG, "nvox must be >= 0");
  if (c <= 0) return fail(CF_ERR_INVALID_ARG, "channels must be > 0");
  if (c > 2048) return fail(CF_ERR_UNSUPPORTED, "bias_lrelu_bwd: more than 2048 channels");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  if (!std::isfinite(alpha)) return fail(CF_ERR_INVALID_ARG, "alpha must be finite");
  hipStream_t st = (hipStream_t)stream;
  const int dt = dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32;
  if (nvox == 0) {
    if (!db) return ok();
    if (!aligned16(db)) return fail(CF_ERR_ALIGNMENT, "db not 16-byte aligned");
    return finish(cf::launch_bias_lrelu_bwd(0, c, dt, nullptr, nullptr, alpha, nullptr, db, nullptr, st),
                  st, "cf_bias_lrelu_bwd");
  }
  cf_status r;
  if ((r = check_ptrs({dy, y, dz})) != CF_OK) return r;
  const size_t bytes = (size_t)nvox * c * elem_size(dtype);
  if (dz != dy && overlap(dz, bytes, dy, bytes))
    return fail(CF_ERR_ALIAS, "bias_lrelu_bwd: dz partially overlaps dy");
  if (overlap(dz, bytes, y, bytes)) return fail(CF_ERR_ALIAS, "bias_lrelu_bwd: dz overlaps y");
  if (db) {
    if (!aligned16(db)) return fail(CF_ERR_ALIGNMENT, "db not 16-byte aligned");
    const size_t need = cf::bias_lrelu_bwd_workspace(nvox, c);
    if (!ws || ws_bytes < need)
      return fail(CF_ERR_WORKSPACE, "bias_lrelu_bwd: workspace smaller than cf_bias_lrelu_bwd_workspace_size()");
    if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
    if (overlap(db, (size_t)c * 4, dz, bytes) || overlap(ws, need, dz, bytes) ||
        overlap(ws, need, dy, bytes) || overlap(ws, need, y, bytes) || overlap(ws, need, db, (size_t)c * 4))
      return fail(CF_ERR_ALIAS, "bias_lrelu_bwd: db or workspace overlaps a tensor");
  }
  return finish(cf::launch_bias_lrelu_bwd(nvox, c, dt, dy, y, alpha, dz, db, ws, st), st,
                "cf_bias_lrelu_bwd");
}

size_t cf_avgpool3d_lrelu_bwd_workspace_size(int32_t n, int32_t d, int32_t h, int32_t w, int32_t c) {
  if (n <= 0 || d <= 0 || h <= 0 || w <= 0 || c <= 0) return 0;
  return cf::pool_lrelu_bwd_workspace((int64_t)n * d * h * w, c);
}

cf_status cf_avgpool3d_lrelu_bwd(int32_t n, int32_t d, int32_t h, int32_t w, int32_t c, int32_t dtype,
                                 const void *dp, const void *mask, float alpha, void *dz, float *db, void *ws,
                                 size_t ws_bytes, void *stream) {
  if (n < 0) return fail(CF_ERR_INVALID_ARG, "batch n must be >= 0");
  if (d <= 0 || h <= 0 || w <= 0 || c <= 0) return fail(CF_ERR_INVALID_ARG, "extents and channels must be > 0");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  if (!std::isfinite(alpha) || alpha < 0.f) return fail(CF_ERR_INVALID_ARG, "alpha must be finite and >= 0");
  const int dt = dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32;
  const int64_t nvox = (int64_t)n * d * h * w;
  if (!cf::pool_lrelu_bwd_supported(nvox, c, dt))
    return fail(CF_ERR_UNSUPPORTED, "avgpool3d_lrelu_bwd: channels must be a power-of-two multiple (at most 64) of "
                                    "the 16-byte vector, at most 256, and the tensor below 2^31 elements");
  hipStream_t st = (hipStream_t)stream;
  if (nvox == 0) {
    if (!db) return ok();
    if (!aligned16(db)) return fail(CF_ERR_ALIGNMENT, "db not 16-byte aligned");
    return finish(cf::launch_pool_lrelu_bwd(0, d, h, w, c, dt, nullptr, nullptr, alpha, nullptr, db, nullptr, st), st,
                  "cf_avgpool3d_lrelu_bwd");
  }
  cf_status r;
  if ((r = check_ptrs({dp, mask, dz})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  const size_t bz = (size_t)nvox * c * es, bp = (size_t)n * (d / 2) * (h / 2) * (w / 2) * c * es;
  const size_t bm = ((size_t)nvox * c + 31) / 32 * 4;
  if (overlap(dz, bz, dp, bp) || overlap(dz, bz, mask, bm))
    return fail(CF_ERR_ALIAS, "avgpool3d_lrelu_bwd: dz overlaps an input");
  if (db) {
    if (!aligned16(db)) return fail(CF_ERR_ALIGNMENT, "db not 16-byte aligned");
    const size_t need = cf::pool_lrelu_bwd_workspace(nvox, c);
    if (!ws || ws_bytes < need)
      return fail(CF_ERR_WORKSPACE, "avgpool3d_lrelu_bwd: workspace smaller than the size query");
    if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
    if (overlap(db, (size_t)c * 4, dz, bz) || overlap(ws, need, dz, bz) || overlap(ws, need, dp, bp) ||
        overlap(ws, need, mask, bm) || overlap(ws, need, db, (size_t)c * 4) || overlap(db, (size_t)c * 4, dp, bp) ||
        overlap(db, (size_t)c * 4, mask, bm))
      return fail(CF_ERR_ALIAS, "avgpool3d_lrelu_bwd: db or workspace overlaps a tensor");
  }
  return finish(cf::launch_pool_lrelu_bwd(n, d, h, w, c, dt, dp, mask, alpha, dz, db, ws, st), st,
                "cf_avgpool3d_lrelu_bwd");
}

static cf_status pool_check(int32_t n, int32_t d, int32_t h, int32_t w, int32_t c, int32_t k,
                            int32_t s, int32_t dtype) {
  if (n < 0) return fail(CF_ERR_INVALID_ARG, "batch n must be >= 0");
  if (d <= 0 || h <= 0 || w <= 0 || c <= 0) return fail(CF_ERR_INVALID_ARG, "extents and channels must be > 0");
  if (k <= 0 || s <= 0) return fail(CF_ERR_INVALID_ARG, "window and stride must be > 0");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  if (k != s) return fail(CF_ERR_UNSUPPORTED, "avgpool3d: only non-overlapping windows (k == s)");
  if (d < k || h < k || w < k) return fail(CF_ERR_INVALID_ARG, "avgpool3d: window larger than input");
  if ((long long)n * d * h * w >= kMaxRows) return fail(CF_ERR_INVALID_ARG, "too many voxels (>= 2^31)");
  return CF_OK;
}

cf_status cf_avgpool3d_fwd(int32_t n, int32_t d, int32_t h, int32_t w, int32_t c, int32_t k, int32_t s,
                           int32_t dtype, const void *y, void *p, void *stream) {
  cf_status r = pool_check(n, d, h, w, c, k, s, dtype);
  if (r != CF_OK) return r;
  if (n == 0) return ok();
  if ((r = check_ptrs({y, p})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  const size_t by = (size_t)n * d * h * w * c * es;
  const size_t bp = (size_t)n * ((d - k) / s + 1) * ((h - k) / s + 1) * ((w - k) / s + 1) * c * es;
  if (overlap(y, by, p, bp)) return fail(CF_ERR_ALIAS, "avgpool3d_fwd: p overlaps y");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_avgpool_fwd(n, d, h, w, c, k, dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32, y, p, st),
                st, "cf_avgpool3d_fwd");
}

cf_status cf_avgpool3d_bwd(int32_t n, int32_t d, int32_t h, int32_t w, int32_t c, int32_t k, int32_t s,
                           int32_t dtype, const void *dp, void *dy, void *stream) {
  cf_status r = pool_check(n, d, h, w, c, k, s, dtype);
  if (r != CF_OK) return r;
  if (n == 0) return ok();
  if ((r = check_ptrs({dp, dy})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  const size_t by = (size_t)n * d * h * w * c * es;
  const size_t bp = (size_t)n * ((d - k) / s + 1) * ((h - k) / s + 1) * ((w - k) / s + 1) * c * es;
  if (overlap(dy, by, dp, bp)) return fail(CF_ERR_ALIAS, "avgpool3d_bwd: dy overlaps dp");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_avgpool_bwd(n, d, h, w, c, k, dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32, dp, dy, st),
                st, "cf_avgpool3d_bwd");
}

// ---------------------------------------------------------------------------
// Fused layer variants
// ---------------------------------------------------------------------------

static int32_t fused_mask(const cf::ConvShape &s, uint32_t flags) {
  int32_t m = 0;
  if (flags & ~(CF_FUSE_POOL2 | CF_FUSE_MASK)) return 0;
  // the mask flag only asks the forward for the mask; with the pool it is implied
  const bool ymode = flags == 0;  // unpooled backward from (dy, y)
  if (flags & CF_FUSE_POOL2) flags = CF_FUSE_POOL2;
  if (flags == CF_FUSE_POOL2) {
    if (cf::smallc_supported(s, true)) m |= 1;
    if (cf::smallc_wgrad_fused_supported(s) || cf::c16_wgrad_supported(s)) m |= 2;
  }
  if (cf::c16_fwd_supported(s)) m |= 1;  // with or without the pool
  if ((flags == 0 || flags == CF_FUSE_MASK) && (cf::direct_supported(s, true) || cf::f32conv_supported(s, true)))
    m |= 1;
  if (ymode && cf::f32wgrad_supported(s)) m |= 2 | 8;
  if (ymode && cf::f32conv_supported(s, false)) m |= 4;
  if (flags == CF_FUSE_POOL2 && cf::f32conv_pool_supported(s)) m |= 1;
  if (flags == CF_FUSE_POOL2 && cf::c16_bwd_supported(s)) m |= 4;
  if (flags == CF_FUSE_POOL2 && cf::c16_wgrad_supported(s) && !cf::smallc_wgrad_fused_supported(s)) m |= 8;
  if (flags == CF_FUSE_POOL2 && cf::f32wgrad_fused_supported(s) && !cf::smallc_wgrad_fused_supported(s)) m |= 2 | 8;
  // bf16 deep layers: pooled forward, and both backward kernels forming dz from
  // (pooled gradient, mask) or (dy, y) as they load it (no dz output)
  if (flags == CF_FUSE_POOL2 && cf::direct_pool_supported(s)) m |= 1;
  if ((flags == CF_FUSE_POOL2 || ymode) && s.dtype == cf::DT_BF16 && cf::direct_wgrad_supported(s)) m |= 2;
  if ((flags == CF_FUSE_POOL2 || ymode) && cf::direct_supported(s, false)) m |= 4;
  return m;
}

int32_t cf_conv3d_fused_supported(const cf_conv3d_desc *desc, uint32_t flags) {
  cf::ConvShape s;
  std::string keep = g_last_error;
  if (resolve(desc, &s) != CF_OK) {
    g_last_error = keep;
    return 0;
  }
  return fused_mask(s, flags);
}

static size_t mask_bytes(const cf::ConvShape &s) {
  const size_t bits = (size_t)s.n * s.od * s.oh * s.ow * s.co;
  return (bits + 31) / 32 * 4;
}

static size_t fused_wgrad_workspace(const cf::ConvShape &s, uint32_t flags) {
  const bool deep16 = s.dtype == cf::DT_BF16 && cf::direct_wgrad_supported(s);
  if (!(flags & CF_FUSE_POOL2))  // (dy, y)
    return deep16 ? cf::direct_wgrad_workspace(s, true) : cf::f32wgrad_workspace(s, 3);
  if (cf::smallc_wgrad_fused_supported(s)) return cf::smallc_wgrad_fused_workspace(s);
  if (cf::f32wgrad_fused_supported(s)) return cf::f32wgrad_workspace(s, 1);
  if (deep16) return cf::direct_wgrad_workspace(s, true);
  return cf::c16_wgrad_workspace(s);
}

// bytes of the 2^3 stride-2 pooled conv output (floor extents)
static size_t pooled_bytes(const cf::ConvShape &s) {
  const size_t es = s.dtype == cf::DT_BF16 ? 2 : 4;
  return (size_t)s.n * (s.od / 2) * (s.oh / 2) * (s.ow / 2) * s.co * es;
}

size_t cf_conv3d_mask_bytes(const cf_conv3d_desc *desc) {
  cf::ConvShape s;
  std::string keep = g_last_error;
  if (resolve(desc, &s) != CF_OK) {
    g_last_error = keep;
    return 0;
  }
  return mask_bytes(s);
}

cf_status cf_conv3d_fwd_fused(const cf_conv3d_desc *desc, const void *x, const void *w, const float *bias,
                              float alpha, uint32_t flags, void *out, void *mask, void *stream) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  if (!std::isfinite(alpha) || alpha < 0.f) return fail(CF_ERR_INVALID_ARG, "alpha must be finite and >= 0");
  if (flags & ~(CF_FUSE_POOL2 | CF_FUSE_MASK)) return fail(CF_ERR_INVALID_ARG, "unknown flags");
  if (!(fused_mask(s, flags) & 1))
    return fail(CF_ERR_UNSUPPORTED, "conv3d_fwd_fused: no fused kernel for this layer shape / flags");
  if (s.n == 0) return ok();
  const bool pool = (flags & CF_FUSE_POOL2) != 0;
  if ((r = check_ptrs({x, w, out})) != CF_OK) return r;
  if (pool && !mask) return fail(CF_ERR_INVALID_ARG, "conv3d_fwd_fused: the pooled variant needs the mask");
  if ((flags & CF_FUSE_MASK) && !mask) return fail(CF_ERR_INVALID_ARG, "conv3d_fwd_fused: CF_FUSE_MASK needs the mask");
  if (mask && !aligned16(mask)) return fail(CF_ERR_ALIGNMENT, "mask not 16-byte aligned");
  if (!bias) return fail(CF_ERR_INVALID_ARG, "bias is NULL");
  Sizes b = conv_bytes(s);
  const size_t ob = pool ? pooled_bytes(s) : b.z;
  const size_t mb = mask_bytes(s);
  if (overlap(out, ob, x, b.x) || overlap(out, ob, w, b.w) || overlap(mask, mb, x, b.x) ||
      overlap(mask, mb, w, b.w) || overlap(mask, mb, out, ob) || overlap(bias, (size_t)s.co * 4, out, ob) ||
      overlap(bias, (size_t)s.co * 4, mask, mb))
    return fail(CF_ERR_ALIAS, "conv3d_fwd_fused: an output overlaps an input");
  hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  if (pool && cf::l1pair_supported(s))
    e = cf::launch_l1pair_fwd(s, x, w, bias, alpha, out, (uint16_t *)mask, st);
  else if (pool && cf::smallc_supported(s, true) && cf::l1c4_supported(s))
    e = cf::launch_conv_fwd_l1c4(s, x, w, bias, alpha, out, (uint16_t *)mask, true, st);
  else if (pool && cf::smallc_supported(s, true))
    e = cf::launch_conv_fwd_smallc(s, x, w, bias, alpha, out, (uint16_t *)mask, true, st);
  else if (cf::f32conv_supported(s, true) && !cf::c16_fwd_supported(s))
    e = cf::launch_conv_fwd_f32(s, (const float *)x, (const float *)w, bias, alpha, (float *)out, (uint8_t *)mask,
                                pool ? 2 : 1, st);
  else if (!pool && !cf::c16_fwd_supported(s))
    e = cf::launch_conv_fwd_direct(s, x, w, bias, alpha, out, mask, true, st);
  else if (pool && cf::direct_pool_supported(s))
    e = cf::launch_conv_fwd_direct_pool(s, x, w, bias, alpha, out, mask, st);
  else
    e = cf::launch_conv_fwd_c16(s, x, w, bias, alpha, out, (uint32_t *)mask, pool ? 2 : 1, st);
  return finish(e, st, "cf_conv3d_fwd_fused");
}

size_t cf_conv3d_bwd_weight_fused_workspace_size(const cf_conv3d_desc *desc, uint32_t flags) {
  cf::ConvShape s;
  std::string keep = g_last_error;
  if (resolve(desc, &s) != CF_OK || !(fused_mask(s, flags) & 2) || s.n == 0) {
    g_last_error = keep;
    return 0;
  }
  return fused_wgrad_workspace(s, flags);
}

// check_only: validate every argument and return without launching
static cf_status bwd_weight_fused(const char *name, const cf_conv3d_desc *desc, const void *x, const void *g,
                                  const void *mask, float alpha, uint32_t flags, float *dw, float *db, void *dz,
                                  void *ws, size_t ws_bytes, void *stream, bool check_only = false) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  if (!std::isfinite(alpha) || alpha < 0.f) return fail(CF_ERR_INVALID_ARG, "alpha must be finite and >= 0");
  if (flags & ~(CF_FUSE_POOL2 | CF_FUSE_MASK)) return fail(CF_ERR_INVALID_ARG, "unknown flags");
  if (!(fused_mask(s, flags) & (dz ? 8 : 2)))
    return fail(CF_ERR_UNSUPPORTED, std::string(name) + ": no fused kernel for this layer shape / flags");
  const bool pool = (flags & CF_FUSE_POOL2) != 0;
  hipStream_t st = (hipStream_t)stream;
  const size_t dw_bytes = (size_t)s.kd * s.kh * s.kw * s.ci * s.co * sizeof(float);
  if (s.n == 0) {
    if ((r = check_ptrs({dw, db})) != CF_OK) return r;
    if (check_only) return CF_OK;
    hipError_t e = cf::launch_fill_zero(dw, (long long)(dw_bytes / 4), st);
    if (e == hipSuccess) e = cf::launch_fill_zero(db, s.co, st);
    return finish(e, st, name);
  }
  if ((r = check_ptrs({x, g, mask, dw, db})) != CF_OK) return r;
  if (dz && (r = check_ptrs({dz})) != CF_OK) return r;
  const size_t need = fused_wgrad_workspace(s, flags);
  if (!ws || ws_bytes < need) return fail(CF_ERR_WORKSPACE, std::string(name) + ": workspace smaller than the size query");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  Sizes b = conv_bytes(s);
  // pooled: g = pooled-output gradient, mask = slope mask; else g = dy, mask = y
  const size_t gb = pool ? pooled_bytes(s) : b.z, mb = pool ? mask_bytes(s) : b.z, dbb = (size_t)s.co * 4;
  const void *ins[3] = {x, g, mask};
  const size_t insz[3] = {b.x, gb, mb};
  for (int i = 0; i < 3; ++i)
    if (overlap(dw, dw_bytes, ins[i], insz[i]) || overlap(db, dbb, ins[i], insz[i]) ||
        overlap(ws, need, ins[i], insz[i]) || (dz && overlap(dz, b.z, ins[i], insz[i])))
      return fail(CF_ERR_ALIAS, std::string(name) + ": an output or the workspace overlaps an input");
  if (overlap(dw, dw_bytes, db, dbb) || overlap(ws, need, dw, dw_bytes) || overlap(ws, need, db, dbb))
    return fail(CF_ERR_ALIAS, std::string(name) + ": outputs / workspace overlap");
  if (dz && (overlap(dz, b.z, dw, dw_bytes) || overlap(dz, b.z, db, dbb) || overlap(dz, b.z, ws, need)))
    return fail(CF_ERR_ALIAS, std::string(name) + ": dz overlaps another output or the workspace");
  if (check_only) return CF_OK;
  hipError_t e;
  const bool deep16 = s.dtype == cf::DT_BF16 && cf::direct_wgrad_supported(s);
  if (!pool && deep16)
    e = cf::launch_conv_bwd_weight_direct(s, x, g, mask, cf::DWG_DYY, alpha, dw, db, ws, st);
  else if (!pool)
    e = cf::launch_conv_bwd_weight_f32(s, (const float *)x, (const float *)g, mask, alpha, dw, db, ws, 3, (float *)dz,
                                       st);
  else if (cf::smallc_wgrad_fused_supported(s))
    e = cf::launch_smallc_wgrad_fused(s, x, g, (const uint16_t *)mask, alpha, dw, db, ws, st);
  else if (cf::f32wgrad_fused_supported(s))
    e = cf::launch_conv_bwd_weight_f32(s, (const float *)x, (const float *)g, mask, alpha, dw, db, ws, 1, (float *)dz,
                                       st);
  else if (deep16)
    e = cf::launch_conv_bwd_weight_direct(s, x, g, mask, cf::DWG_POOL, alpha, dw, db, ws, st);
  else
    e = cf::launch_conv_bwd_weight_c16(s, x, g, (const uint32_t *)mask, alpha, dw, db, ws, true, dz, st);
  return finish(e, st, name);
}

cf_status cf_conv3d_bwd_weight_fused(const cf_conv3d_desc *desc, const void *x, const void *g, const void *mask,
                                     float alpha, uint32_t flags, float *dw, float *db, void *ws, size_t ws_bytes,
                                     void *stream) {
  return bwd_weight_fused("cf_conv3d_bwd_weight_fused", desc, x, g, mask, alpha, flags, dw, db, nullptr, ws,
                          ws_bytes, stream);
}

cf_status cf_conv3d_bwd_weight_fused_dz(const cf_conv3d_desc *desc, const void *x, const void *g, const void *mask,
                                        float alpha, uint32_t flags, float *dw, float *db, void *dz, void *ws,
                                        size_t ws_bytes, void *stream) {
  if (!dz && desc && desc->n > 0) return fail(CF_ERR_INVALID_ARG, "cf_conv3d_bwd_weight_fused_dz: dz is NULL");
  return bwd_weight_fused("cf_conv3d_bwd_weight_fused_dz", desc, x, g, mask, alpha, flags, dw, db, dz, ws,
                          ws_bytes, stream);
}

static cf_status bwd_data_fused(const cf_conv3d_desc *desc, const void *g, const void *mask, const void *w,
                                float alpha, uint32_t flags, void *dx, void *stream, bool check_only) {
  cf::ConvShape s;
  cf_status r = resolve(desc, &s);
  if (r != CF_OK) return r;
  if (!std::isfinite(alpha) || alpha < 0.f) return fail(CF_ERR_INVALID_ARG, "alpha must be finite and >= 0");
  if (flags & ~(CF_FUSE_POOL2 | CF_FUSE_MASK)) return fail(CF_ERR_INVALID_ARG, "unknown flags");
  if (!(fused_mask(s, flags) & 4))
    return fail(CF_ERR_UNSUPPORTED, "conv3d_bwd_data_fused: no fused kernel for this layer shape / flags");
  if (s.n == 0) return ok();
  if ((r = check_ptrs({g, mask, w, dx})) != CF_OK) return r;
  Sizes b = conv_bytes(s);
  const bool pool = (flags & CF_FUSE_POOL2) != 0;
  const size_t gb = pool ? pooled_bytes(s) : b.z, mb = pool ? mask_bytes(s) : b.z;
  if (overlap(dx, b.x, g, gb) || overlap(dx, b.x, mask, mb) || overlap(dx, b.x, w, b.w))
    return fail(CF_ERR_ALIAS, "conv3d_bwd_data_fused: dx overlaps an input");
  if (check_only) return CF_OK;
  hipStream_t st = (hipStream_t)stream;
  hipError_t e;
  if (pool && cf::c16_bwd_supported(s))
    e = cf::launch_conv_bwd_data_c16(s, g, (const uint32_t *)mask, w, alpha, dx, true, st);
  else if (cf::direct_supported(s, false))  // bf16 deep layers
    e = cf::launch_conv_bwd_data_direct_fused(s, g, mask, pool ? cf::DWG_POOL : cf::DWG_DYY, alpha, w, dx, st);
  else
    e = cf::launch_conv_bwd_data_f32(s, (const float *)g, (const float *)w, (float *)dx, st, (const float *)mask,
                                     alpha);
  return finish(e, st, "cf_conv3d_bwd_data_fused");
}

cf_status cf_conv3d_bwd_data_fused(const cf_conv3d_desc *desc, const void *g, const void *mask, const void *w,
                                   float alpha, uint32_t flags, void *dx, void *stream) {
  return bwd_data_fused(desc, g, mask, w, alpha, flags, dx, stream, false);
}

cf_status cf_conv3d_bwd_fused(const cf_conv3d_desc *desc, const void *x, const void *g, const void *mask,
                              const void *w, float alpha, uint32_t flags, float *dw, float *db, void *dx, void *ws,
                              size_t ws_bytes, void *stream) {
  const char *name = "cf_conv3d_bwd_fused";
  cf_status r = bwd_weight_fused(name, desc, x, g, mask, alpha, flags, dw, db, nullptr, ws, ws_bytes, stream, true);
  if (r != CF_OK) return r;
  if ((r = bwd_data_fused(desc, g, mask, w, alpha, flags, dx, stream, true)) != CF_OK) return r;
  cf::ConvShape s;
  resolve(desc, &s);
  if (s.n > 0) {
    const size_t dxb = conv_bytes(s).x, dwb = (size_t)s.kd * s.kh * s.kw * s.ci * s.co * sizeof(float);
    if (overlap(dx, dxb, dw, dwb) || overlap(dx, dxb, db, (size_t)s.co * 4) ||
        overlap(dx, dxb, ws, fused_wgrad_workspace(s, flags)))
      return fail(CF_ERR_ALIAS, "cf_conv3d_bwd_fused: dx overlaps dW, db or the workspace");
  }
  // fp32 unpooled layers: both products from (dy, y) in one launch where the
  // kernels allow; everything else is the two calls in sequence
  if (s.n > 0 && s.dtype == cf::DT_F32 && !(flags & CF_FUSE_POOL2)) {
    hipStream_t st = (hipStream_t)stream;
    return finish(cf::launch_conv_bwd_fused_f32(s, (const float *)x, (const float *)g, (const float *)mask,
                                                (const float *)w, alpha, dw, db, (float *)dx, ws, st),
                  st, name);
  }
  if ((r = bwd_weight_fused(name, desc, x, g, mask, alpha, flags, dw, db, nullptr, ws, ws_bytes, stream)) != CF_OK)
    return r;
  return bwd_data_fused(desc, g, mask, w, alpha, flags, dx, stream, false);
}

// ---------------------------------------------------------------------------
// Deferred gradient sums
// ---------------------------------------------------------------------------


cf_status cf_reduce_partials(int32_t n, const cf_reduction *jobs, void *stream) {
  if (n < 0) return fail(CF_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return ok();
  if (!jobs) return fail(CF_ERR_INVALID_ARG, "jobs is NULL");
  std::vector<cf::SumJob> v;
  v.reserve(n);
  for (int32_t i = 0; i < n; ++i) {
    const cf_reduction &j = jobs[i];
    if (j.rows < 0 || j.cols < 0) return fail(CF_ERR_INVALID_ARG, "reduction with negative rows or cols");
    if (j.cols == 0) continue;
    if (!j.out || (j.rows > 0 && !j.part)) return fail(CF_ERR_INVALID_ARG, "reduction with a NULL pointer");
    if (((uintptr_t)j.out & 3) || ((uintptr_t)j.part & 3))
      return fail(CF_ERR_ALIGNMENT, "reduction pointers must be 4-byte aligned");
    if (overlap(j.out, (size_t)j.cols * 4, j.part, (size_t)j.rows * j.cols * 4))
      return fail(CF_ERR_ALIAS, "reduction output overlaps its partials");
    v.push_back(cf::SumJob{j.part, j.out, j.rows, j.cols});
  }
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_sum_batch(v.data(), (int)v.size(), st), st, "cf_reduce_partials");
}

cf_status cf_conv3d_bwd_weight_deferred(const cf_conv3d_desc *desc, const void *x, const void *dz, float *dw,
                                        void *ws, size_t ws_bytes, cf_reduction *pending, int32_t *npending,
                                        void *stream) {
  return deferred(pending, npending, [&] { return cf_conv3d_bwd_weight(desc, x, dz, dw, ws, ws_bytes, stream); });
}

cf_status cf_bias_lrelu_bwd_deferred(int64_t nvox, int32_t c, int32_t dtype, const void *dy, const void *y,
                                     float alpha, void *dz, float *db, void *ws, size_t ws_bytes,
                                     cf_reduction *pending, int32_t *npending, void *stream) {
  return deferred(pending, npending, [&] {
    return cf_bias_lrelu_bwd(nvox, c, dtype, dy, y, alpha, dz, db, ws, ws_bytes, stream);
  });
}

cf_status cf_avgpool3d_lrelu_bwd_deferred(int32_t n, int32_t d, int32_t h, int32_t w, int32_t c, int32_t dtype,
                                          const void *dp, const void *mask, float alpha, void *dz, float *db,
                                          void *ws, size_t ws_bytes, cf_reduction *pending, int32_t *npending,
                                          void *stream) {
  return deferred(pending, npending, [&] {
    return cf_avgpool3d_lrelu_bwd(n, d, h, w, c, dtype, dp, mask, alpha, dz, db, ws, ws_bytes, stream);
  });
}

cf_status cf_conv3d_bwd_weight_fused_deferred(const cf_conv3d_desc *desc, const void *x, const void *g,
                                              const void *mask, float alpha, uint32_t flags, float *dw, float *db,
                                              void *dz, void *ws, size_t ws_bytes, cf_reduction *pending,
                                              int32_t *npending, void *stream) {
  return deferred(pending, npending, [&] {
    return bwd_weight_fused(dz ? "cf_conv3d_bwd_weight_fused_dz" : "cf_conv3d_bwd_weight_fused", desc, x, g, mask,
                            alpha, flags, dw, db, dz, ws, ws_bytes, stream);
  });
}

cf_status cf_conv3d_bwd_deferred(const cf_conv3d_desc *desc, const void *x, const void *dz, const void *w,
                                 float *dw, void *dx, void *ws, size_t ws_bytes, cf_reduction *pending,
                                 int32_t *npending, void *stream) {
  return deferred(pending, npending, [&] { return cf_conv3d_bwd(desc, x, dz, w, dw, dx, ws, ws_bytes, stream); });
}

cf_status cf_conv3d_bwd_fused_deferred(const cf_conv3d_desc *desc, const void *x, const void *g, const void *mask,
                                       const void *w, float alpha, uint32_t flags, float *dw, float *db, void *dx,
                                       void *ws, size_t ws_bytes, cf_reduction *pending, int32_t *npending,
                                       void *stream) {
  return deferred(pending, npending, [&] {
    return cf_conv3d_bwd_fused(desc, x, g, mask, w, alpha, flags, dw, db, dx, ws, ws_bytes, stream);
  });
}


size_t cf_adam_larc_workspace_size(int32_t ngroups, const int64_t *offsets) {
  std::string keep = g_last_error;
  cf::OptGroups G;
  int chunks = 0;
  if (adam_plan(ngroups, offsets, &G, &chunks) != CF_OK) {
    g_last_error = keep;
    return 0;
  }
  return (size_t)chunks * 2 * sizeof(double);
}

cf_status cf_adam_larc_step(int32_t ngroups, const int64_t *offsets, int64_t t, const cf_adam_larc_hparams *hp,
                            float *v, const float *g, float *m, float *s, void *v16, void *ws, size_t ws_bytes,
                            void *stream) {
  cf::OptGroups G;
  int chunks = 0;
  cf_status r = adam_plan(ngroups, offsets, &G, &chunks);
  if (r != CF_OK) return r;
  if (!hp) return fail(CF_ERR_INVALID_ARG, "adam_larc: hp is NULL");
  if (t < 0) return fail(CF_ERR_INVALID_ARG, "adam_larc: t must be >= 0");
  if (hp->t_decay <= 0) return fail(CF_ERR_INVALID_ARG, "adam_larc: t_decay must be > 0");
  const double vals[] = {hp->eta0, hp->eta_min, hp->beta1, hp->beta2, hp->eps_hat,
                         hp->larc_coef, hp->larc_fallback, hp->larc_clip};
  for (double x : vals)
    if (!std::isfinite(x)) return fail(CF_ERR_INVALID_ARG, "adam_larc: hyperparameters must be finite");
  if (hp->beta1 < 0.0 || hp->beta1 >= 1.0 || hp->beta2 < 0.0 || hp->beta2 >= 1.0)
    return fail(CF_ERR_INVALID_ARG, "adam_larc: beta1 and beta2 must lie in [0, 1)");
  if (hp->eps_hat < 0.0) return fail(CF_ERR_INVALID_ARG, "adam_larc: eps_hat must be >= 0");
  if (chunks == 0) return ok();
  if ((r = check_ptrs({v, g, m, s})) != CF_OK) return r;
  if (v16 && !aligned16(v16)) return fail(CF_ERR_ALIGNMENT, "adam_larc: v16 not 16-byte aligned");
  const size_t need = (size_t)chunks * 2 * sizeof(double);
  if (!ws || ws_bytes < need)
    return fail(CF_ERR_WORKSPACE, "adam_larc: workspace smaller than cf_adam_larc_workspace_size()");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  const size_t nb = (size_t)offsets[ngroups] * 4;
  const void *bufs[] = {v, g, m, s, v16, ws};
  const size_t lens[] = {nb, nb, nb, nb, nb / 2, need};
  for (int a = 0; a < 6; ++a)
    for (int b = a + 1; b < 6; ++b)
      if (overlap(bufs[a], lens[a], bufs[b], lens[b]))
        return fail(CF_ERR_ALIAS, "adam_larc: v, g, m, s, v16 and the workspace must not overlap");
  cf::OptHparams h{hp->eta0,  hp->eta_min,   hp->t_decay,       hp->beta1,    hp->beta2,
                   hp->eps_hat, hp->larc_coef, hp->larc_fallback, hp->larc_clip};
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_adam_larc(G, chunks, h, (long long)t, v, g, m, s, (uint16_t *)v16, (double *)ws, st),
                st, "cf_adam_larc_step");
}

}  // extern "C"

// ---- fully-connected head and loss -------------------------------------------

namespace {
cf_status fc_check(int32_t m, int32_t k, int32_t n, int32_t dtype, const char *who) {
  if (m < 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": m must be >= 0");
  if (k <= 0 || n <= 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": k and n must be > 0");
  if (n > 65536) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": more than 65536 outputs");
  if ((long long)k * n >= (1LL << 40)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": k * n too large");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  return CF_OK;
}
int kdt(int32_t dtype) { return dtype == CF_BF16 ? cf::DT_BF16 : cf::DT_F32; }
}  // namespace

size_t cf_fc_fwd_workspace_size(int32_t m, int32_t k, int32_t n) {
  if (m <= 0 || k <= 0 || n <= 0 || n > 65536 || (long long)k * n >= (1LL << 40)) return 0;
  return cf::fc_fwd_workspace(m, k, n);
}

cf_status cf_fc_fwd(int32_t m, int32_t k, int32_t n, int32_t dtype, const void *x, const void *w, void *z,
                    void *ws, size_t ws_bytes, void *stream) {
  cf_status r = fc_check(m, k, n, dtype, "fc_fwd");
  if (r != CF_OK) return r;
  if (m == 0) return ok();
  if ((r = check_ptrs({x, w, z})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  const size_t bx = (size_t)m * k * es, bw = (size_t)k * n * es, bz = (size_t)m * n * es;
  const size_t need = cf::fc_fwd_workspace(m, k, n);
  if (!ws || ws_bytes < need) return fail(CF_ERR_WORKSPACE, "fc_fwd: workspace smaller than cf_fc_fwd_workspace_size()");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  if (overlap(z, bz, x, bx) || overlap(z, bz, w, bw)) return fail(CF_ERR_ALIAS, "fc_fwd: z overlaps x or W");
  if (overlap(ws, need, x, bx) || overlap(ws, need, w, bw) || overlap(ws, need, z, bz))
    return fail(CF_ERR_ALIAS, "fc_fwd: workspace overlaps a tensor");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_fc_fwd(m, k, n, kdt(dtype), x, w, z, ws, st), st, "cf_fc_fwd");
}

cf_status cf_fc_bwd_data(int32_t m, int32_t k, int32_t n, int32_t dtype, const void *dz, const void *w, void *dx,
                         void *stream) {
  cf_status r = fc_check(m, k, n, dtype, "fc_bwd_data");
  if (r != CF_OK) return r;
  if (m == 0) return ok();
  if ((r = check_ptrs({dz, w, dx})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  const size_t bx = (size_t)m * k * es, bw = (size_t)k * n * es, bz = (size_t)m * n * es;
  if (overlap(dx, bx, dz, bz) || overlap(dx, bx, w, bw)) return fail(CF_ERR_ALIAS, "fc_bwd_data: dx overlaps dz or W");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_fc_bwd_data(m, k, n, kdt(dtype), dz, w, dx, st), st, "cf_fc_bwd_data");
}

cf_status cf_fc_bwd_weight(int32_t m, int32_t k, int32_t n, int32_t dtype, const void *x, const void *dz, float *dw,
                           void *stream) {
  cf_status r = fc_check(m, k, n, dtype, "fc_bwd_weight");
  if (r != CF_OK) return r;
  hipStream_t st = (hipStream_t)stream;
  if (m == 0) {
    if ((r = check_ptrs({dw})) != CF_OK) return r;
    return finish(cf::launch_fill_zero(dw, (long long)k * n, st), st, "cf_fc_bwd_weight");
  }
  if ((r = check_ptrs({x, dz, dw})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  const size_t bx = (size_t)m * k * es, bz = (size_t)m * n * es, bw = (size_t)k * n * 4;
  if (overlap(dw, bw, x, bx) || overlap(dw, bw, dz, bz)) return fail(CF_ERR_ALIAS, "fc_bwd_weight: dW overlaps x or dz");
  return finish(cf::launch_fc_bwd_weight(m, k, n, kdt(dtype), x, dz, dw, st), st, "cf_fc_bwd_weight");
}

size_t cf_fc_head_workspace_size(int32_t m, int32_t nlayers, const int32_t *dims) {
  if (!dims || nlayers < 2 || nlayers > 4 || m < 1) return 0;
  int d[5];
  for (int i = 0; i <= nlayers; ++i) {
    if (dims[i] < 1) return 0;
    d[i] = dims[i];
  }
  return cf::fc_head_workspace(m, nlayers, d);
}

cf_status cf_fc_head(int32_t m, int32_t nlayers, const int32_t *dims, int32_t dtype, const void *x,
                     const void *const *w, const float *const *b, float alpha, const float *target, void *const *y,
                     void *const *dz, void *const *dx, float *const *dw, float *const *db, float *loss, void *ws,
                     size_t ws_bytes, void *stream) {
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  if (!dims || !w || !b || !y || !dz || !dx || !dw || !db)
    return fail(CF_ERR_INVALID_ARG, "fc_head: NULL dims or pointer array");
  if (nlayers < 2 || nlayers > 4) return fail(CF_ERR_UNSUPPORTED, "fc_head: 2 to 4 layers");
  if (m < 1 || m > 8) return fail(CF_ERR_UNSUPPORTED, "fc_head: 1 to 8 batch rows");
  int d[5];
  for (int i = 0; i <= nlayers; ++i) {
    if (dims[i] < 1) return fail(CF_ERR_INVALID_ARG, "fc_head: every width must be > 0");
    d[i] = dims[i];
  }
  if (!cf::fc_head_supported(m, nlayers, d, kdt(dtype)))
    return fail(CF_ERR_UNSUPPORTED, "fc_head: widths outside the fused head's limits (see cf_fc_head)");
  cf_status r;
  if ((r = check_ptrs({x, target, loss, ws})) != CF_OK) return r;
  const size_t es = elem_size(dtype);
  // (pointer, bytes) of every input and every output
  std::vector<std::pair<const void *, size_t>> in, out;
  in.push_back({x, (size_t)m * d[0] * es});
  in.push_back({target, (size_t)m * d[nlayers] * 4});
  for (int i = 0; i < nlayers; ++i) {
    if ((r = check_ptrs({w[i], b[i], y[i], dz[i], dx[i], dw[i], db[i]})) != CF_OK) return r;
    const size_t kn = (size_t)d[i] * d[i + 1];
    in.push_back({w[i], kn * es});
    in.push_back({b[i], (size_t)d[i + 1] * 4});
    out.push_back({y[i], (size_t)m * d[i + 1] * es});
    out.push_back({dz[i], (size_t)m * d[i + 1] * es});
    out.push_back({dx[i], (size_t)m * d[i] * es});
    out.push_back({dw[i], kn * 4});
    out.push_back({db[i], (size_t)d[i + 1] * 4});
  }
  out.push_back({loss, 4});
  const size_t need = cf::fc_head_workspace(m, nlayers, d);
  if (ws_bytes < need) return fail(CF_ERR_WORKSPACE, "fc_head: workspace smaller than cf_fc_head_workspace_size()");
  out.push_back({ws, need});
  for (size_t i = 0; i < out.size(); ++i) {
    for (const auto &t : in)
      if (overlap(out[i].first, out[i].second, t.first, t.second))
        return fail(CF_ERR_ALIAS, "fc_head: an output or the workspace overlaps an input");
    for (size_t j = i + 1; j < out.size(); ++j)
      if (overlap(out[i].first, out[i].second, out[j].first, out[j].second))
        return fail(CF_ERR_ALIAS, "fc_head: two outputs overlap");
  }
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_fc_head(m, nlayers, d, kdt(dtype), x, w, b, alpha, target, y, dz, dx, dw, db, loss, ws, st),
                st, "cf_fc_head");
}

cf_status cf_mse_loss(int32_t m, int32_t n, int32_t dtype, const void *p, const float *t, float *loss, void *dp,
                      void *stream) {
  if (m <= 0 || n <= 0) return fail(CF_ERR_INVALID_ARG, "mse_loss: m and n must be > 0");
  if ((long long)m * n >= (1LL << 31)) return fail(CF_ERR_UNSUPPORTED, "mse_loss: m * n too large");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  cf_status r;
  if ((r = check_ptrs({p, t, loss})) != CF_OK) return r;
  if (dp && !aligned16(dp)) return fail(CF_ERR_ALIGNMENT, "dp not 16-byte aligned");
  const long long cnt = (long long)m * n;
  const size_t es = elem_size(dtype);
  if (overlap(loss, 4, p, cnt * es) || overlap(loss, 4, t, cnt * 4) || overlap(loss, 4, dp, dp ? cnt * es : 0))
    return fail(CF_ERR_ALIAS, "mse_loss: loss overlaps a tensor");
  if (dp && (overlap(dp, cnt * es, p, cnt * es) || overlap(dp, cnt * es, t, cnt * 4)))
    return fail(CF_ERR_ALIAS, "mse_loss: dp overlaps p or t");
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_mse_loss(cnt, kdt(dtype), p, t, loss, dp, (float)(1.0 / (double)cnt), st), st,
                "cf_mse_loss");
}

// ---- layer normalisation -------------------------------------------------------

namespace {
cf_status norm_check(int64_t rows, int32_t c, int32_t dtype, const char *who) {
  if (rows < 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": rows must be >= 0");
  if (c <= 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": c must be > 0");
  if (c > (1 << 30)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": more than 2^30 values a row");
  if (rows >= (1LL << 40) / c) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": rows * c too large");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  return CF_OK;
}

typedef std::pair<const void *, size_t> Span;

// an output may be one of `same` exactly; otherwise no output overlaps an input or another output
cf_status norm_alias(std::initializer_list<Span> in, std::initializer_list<Span> out, const void *first_out,
                     std::initializer_list<const void *> same, const char *who) {
  for (const Span *o = out.begin(); o != out.end(); ++o) {
    for (const Span &i : in) {
      bool exact = false;
      for (const void *p : same) exact = exact || (o->first == first_out && o->first == i.first && p == i.first);
      if (!exact && overlap(o->first, o->second, i.first, i.second))
        return fail(CF_ERR_ALIAS, std::string(who) + ": an output or the workspace overlaps an input");
    }
    for (const Span *q = o + 1; q != out.end(); ++q)
      if (overlap(o->first, o->second, q->first, q->second))
        return fail(CF_ERR_ALIAS, std::string(who) + ": two outputs overlap");
  }
  return CF_OK;
}
}  // namespace

extern "C" {

size_t cf_layernorm_fwd_workspace_size(int64_t rows, int32_t c, int32_t dtype) {
  const std::string keep = g_last_error;
  const bool bad = norm_check(rows, c, dtype, "layernorm") != CF_OK;
  g_last_error = keep;
  return bad || rows == 0 ? 0 : cf::layernorm_fwd_workspace(rows, c, kdt(dtype));
}

cf_status cf_layernorm_fwd(int64_t rows, int32_t c, int32_t dtype, const void *x, const float *gamma,
                           const float *beta, float eps, void *y, float *mean, float *rstd, void *ws,
                           size_t ws_bytes, void *stream) {
  cf_status r = norm_check(rows, c, dtype, "layernorm_fwd");
  if (r != CF_OK) return r;
  if (!std::isfinite(eps) || eps < 0.f) return fail(CF_ERR_INVALID_ARG, "layernorm_fwd: eps must be finite and >= 0");
  if (rows == 0) return ok();
  if ((r = check_ptrs({x, gamma, beta, y, mean, rstd})) != CF_OK) return r;
  const size_t need = cf::layernorm_fwd_workspace(rows, c, kdt(dtype));
  if (need && (!ws || ws_bytes < need))
    return fail(CF_ERR_WORKSPACE, "layernorm_fwd: workspace smaller than cf_layernorm_fwd_workspace_size()");
  if (need && !aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  const size_t nx = (size_t)rows * c * elem_size(dtype), nc = (size_t)c * 4, nr = (size_t)rows * 4;
  if ((r = norm_alias({{x, nx}, {gamma, nc}, {beta, nc}}, {{y, nx}, {mean, nr}, {rstd, nr}, {ws, need}}, y, {x},
                      "layernorm_fwd")) != CF_OK)
    return r;
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_layernorm_fwd(rows, c, kdt(dtype), x, gamma, beta, eps, y, mean, rstd, ws, st), st,
                "cf_layernorm_fwd");
}

size_t cf_layernorm_bwd_workspace_size(int64_t rows, int32_t c, int32_t dtype) {
  const std::string keep = g_last_error;
  const bool bad = norm_check(rows, c, dtype, "layernorm") != CF_OK;
  g_last_error = keep;
  return bad || rows == 0 ? 0 : cf::layernorm_bwd_workspace(rows, c, kdt(dtype));
}

cf_status cf_layernorm_bwd(int64_t rows, int32_t c, int32_t dtype, const void *dy, const void *x,
                           const float *gamma, const float *mean, const float *rstd, void *dx, float *dgamma,
                           float *dbeta, void *ws, size_t ws_bytes, void *stream) {
  cf_status r = norm_check(rows, c, dtype, "layernorm_bwd");
  if (r != CF_OK) return r;
  hipStream_t st = (hipStream_t)stream;
  const size_t nc = (size_t)c * 4;
  if (rows == 0) {
    if ((r = check_ptrs({dgamma, dbeta})) != CF_OK) return r;
    if (overlap(dgamma, nc, dbeta, nc)) return fail(CF_ERR_ALIAS, "layernorm_bwd: two outputs overlap");
    hipError_t e = cf::launch_fill_zero(dgamma, c, st);
    if (e == hipSuccess) e = cf::launch_fill_zero(dbeta, c, st);
    return finish(e, st, "cf_layernorm_bwd");
  }
  if ((r = check_ptrs({dy, x, gamma, mean, rstd, dx, dgamma, dbeta})) != CF_OK) return r;
  const size_t need = cf::layernorm_bwd_workspace(rows, c, kdt(dtype));
  if (!ws || ws_bytes < need)
    return fail(CF_ERR_WORKSPACE, "layernorm_bwd: workspace smaller than cf_layernorm_bwd_workspace_size()");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  const size_t nx = (size_t)rows * c * elem_size(dtype), nr = (size_t)rows * 4;
  if ((r = norm_alias({{dy, nx}, {x, nx}, {gamma, nc}, {mean, nr}, {rstd, nr}},
                      {{dx, nx}, {dgamma, nc}, {dbeta, nc}, {ws, need}}, dx, {dy, x}, "layernorm_bwd")) != CF_OK)
    return r;
  return finish(cf::launch_layernorm_bwd(rows, c, kdt(dtype), dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, st), st,
                "cf_layernorm_bwd");
}

}  // extern "C"

// ---- orthogonalised updates -----------------------------------------------------

namespace {
constexpr int32_t kMaxMats = 1 << 16;

// validates the matrices; end = elements from the arrays' start to the last matrix's end
cf_status mats_check(int32_t nmat, const cf_matrix *mats, int64_t *end, const char *who) {
  *end = 0;
  if (nmat < 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": nmat must be >= 0");
  if (nmat > kMaxMats) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": more than 65536 matrices");
  if (nmat > 0 && !mats) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": mats is NULL");
  for (int32_t l = 0; l < nmat; ++l) {
    const cf_matrix &M = mats[l];
    if (M.offset < 0 || M.rows < 0 || M.cols < 0)
      return fail(CF_ERR_INVALID_ARG, std::string(who) + ": negative offset, rows or cols");
    if (M.offset % 8 != 0) return fail(CF_ERR_ALIGNMENT, std::string(who) + ": a matrix's offset is not a multiple of 8");
    if (M.rows == 0 || M.cols == 0) continue;
    const int32_t lo = M.rows < M.cols ? M.rows : M.cols, hi = M.rows < M.cols ? M.cols : M.rows;
    if (lo > 16384 || hi > (1 << 24))
      return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": a side longer than 16384 (shorter) or 2^24 (longer)");
    if (M.offset >= (1LL << 40)) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": offset too large");
    if (M.offset < *end) return fail(CF_ERR_ALIAS, std::string(who) + ": matrices overlap or are not in ascending order");
    *end = M.offset + (int64_t)M.rows * M.cols;
  }
  return CF_OK;
}

cf_status ns_check(const cf_ns_hparams &hp, cf::NsSteps *S, const char *who) {
  for (double x : {hp.a, hp.b, hp.c, hp.eps})
    if (!std::isfinite(x)) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": coefficients and eps must be finite");
  if (hp.eps < 0.0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": eps must be >= 0");
  if (hp.steps < 1 || hp.steps > CF_NS_MAX_STEPS)
    return fail(CF_ERR_INVALID_ARG, std::string(who) + ": steps must be 1 to CF_NS_MAX_STEPS");
  static_assert(cf::kNsMaxSteps == CF_NS_MAX_STEPS, "stage table size");
  S->eps = hp.eps;
  if (!cf::ns_scales(hp.a, hp.b, hp.c, hp.steps, S))
    return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": the iteration can grow past its factors' range with these coefficients");
  return CF_OK;
}

// calls f(table, workspace bytes) for the non-empty matrices, a table at a time
template <class F> cf_status mats_tables(int32_t nmat, const cf_matrix *mats, int32_t dtype, bool momentum, F f) {
  int32_t l = 0;
  while (l < nmat) {
    long long off[cf::kNsTable];
    int rows[cf::kNsTable], cols[cf::kNsTable], n = 0;
    for (; l < nmat && n < cf::kNsTable; ++l) {
      if (mats[l].rows == 0 || mats[l].cols == 0) continue;
      off[n] = mats[l].offset;
      rows[n] = mats[l].rows;
      cols[n++] = mats[l].cols;
    }
    if (n == 0) break;
    cf::NsTable T;
    const size_t need = cf::ns_plan(n, off, rows, cols, kdt(dtype), momentum, &T);
    const cf_status r = f(T, rows, cols, need);
    if (r != CF_OK) return r;
  }
  return CF_OK;
}

size_t mats_workspace(int32_t nmat, const cf_matrix *mats, int32_t dtype, bool momentum) {
  size_t most = 0;
  mats_tables(nmat, mats, dtype, momentum, [&](cf::NsTable &, const int *, const int *, size_t need) {
    most = need > most ? need : most;
    return CF_OK;
  });
  return most;
}
}  // namespace

extern "C" {

size_t cf_newton_schulz_workspace_size(int32_t nmat, const cf_matrix *mats, int32_t dtype) {
  const std::string keep = g_last_error;
  int64_t end;
  const bool bad = mats_check(nmat, mats, &end, "newton_schulz") != CF_OK || (dtype != CF_F32 && dtype != CF_BF16);
  g_last_error = keep;
  return bad ? 0 : mats_workspace(nmat, mats, dtype, false);
}

cf_status cf_newton_schulz(int32_t nmat, const cf_matrix *mats, int32_t dtype, const cf_ns_hparams *hp,
                           const void *g, void *o, void *ws, size_t ws_bytes, void *stream) {
  int64_t end;
  cf_status r = mats_check(nmat, mats, &end, "newton_schulz");
  if (r != CF_OK) return r;
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  if (!hp) return fail(CF_ERR_INVALID_ARG, "newton_schulz: hp is NULL");
  cf::NsSteps S;
  if ((r = ns_check(*hp, &S, "newton_schulz")) != CF_OK) return r;
  if (end == 0) return ok();
  if ((r = check_ptrs({g, o})) != CF_OK) return r;
  const size_t need = mats_workspace(nmat, mats, dtype, false), nb = (size_t)end * elem_size(dtype);
  if (!ws || ws_bytes < need)
    return fail(CF_ERR_WORKSPACE, "newton_schulz: workspace smaller than cf_newton_schulz_workspace_size()");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  if ((g != o && overlap(g, nb, o, nb)) || overlap(ws, need, g, nb) || overlap(ws, need, o, nb))
    return fail(CF_ERR_ALIAS, "newton_schulz: g, o and the workspace must not overlap (o may be g)");
  hipStream_t st = (hipStream_t)stream;
  return mats_tables(nmat, mats, dtype, false, [&](cf::NsTable &T, const int *, const int *, size_t) {
    return finish(cf::launch_newton_schulz(T, S, kdt(dtype), g, nullptr, nullptr, nullptr, o, nullptr, ws, st), st,
                  "cf_newton_schulz");
  });
}

size_t cf_muon_workspace_size(int32_t nmat, const cf_matrix *mats) {
  const std::string keep = g_last_error;
  int64_t end;
  const bool bad = mats_check(nmat, mats, &end, "muon") != CF_OK;
  g_last_error = keep;
  return bad ? 0 : mats_workspace(nmat, mats, CF_F32, true);
}

cf_status cf_muon_step(int32_t nmat, const cf_matrix *mats, int64_t t, const cf_muon_hparams *hp, float *v,
                       const float *g, float *m, void *v16, void *ws, size_t ws_bytes, void *stream) {
  int64_t end;
  cf_status r = mats_check(nmat, mats, &end, "muon");
  if (r != CF_OK) return r;
  if (!hp) return fail(CF_ERR_INVALID_ARG, "muon: hp is NULL");
  if (t < 0) return fail(CF_ERR_INVALID_ARG, "muon: t must be >= 0");
  if (hp->t_decay <= 0) return fail(CF_ERR_INVALID_ARG, "muon: t_decay must be > 0");
  for (double x : {hp->eta0, hp->eta_min, hp->mu, hp->weight_decay})
    if (!std::isfinite(x)) return fail(CF_ERR_INVALID_ARG, "muon: hyperparameters must be finite");
  if (hp->mu < 0.0 || hp->mu >= 1.0) return fail(CF_ERR_INVALID_ARG, "muon: mu must lie in [0, 1)");
  if (hp->weight_decay < 0.0) return fail(CF_ERR_INVALID_ARG, "muon: weight_decay must be >= 0");
  if (hp->nesterov != 0 && hp->nesterov != 1) return fail(CF_ERR_INVALID_ARG, "muon: nesterov must be 0 or 1");
  if (hp->scale != CF_MUON_SCALE_SHAPE && hp->scale != CF_MUON_SCALE_RMS)
    return fail(CF_ERR_INVALID_ARG, "muon: unknown scale");
  cf::NsSteps S;
  if ((r = ns_check(hp->ns, &S, "muon")) != CF_OK) return r;
  if (end == 0) return ok();
  if ((r = check_ptrs({v, g, m})) != CF_OK) return r;
  if (v16 && !aligned16(v16)) return fail(CF_ERR_ALIGNMENT, "muon: v16 not 16-byte aligned");
  const size_t need = mats_workspace(nmat, mats, CF_F32, true);
  if (!ws || ws_bytes < need) return fail(CF_ERR_WORKSPACE, "muon: workspace smaller than cf_muon_workspace_size()");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  const size_t nb = (size_t)end * 4;
  const void *bufs[] = {v, g, m, v16, ws};
  const size_t lens[] = {nb, nb, nb, nb / 2, need};
  for (int a = 0; a < 5; ++a)
    for (int b = a + 1; b < 5; ++b)
      if (overlap(bufs[a], lens[a], bufs[b], lens[b]))
        return fail(CF_ERR_ALIAS, "muon: v, g, m, v16 and the workspace must not overlap");
  const double tc = (double)(t < hp->t_decay ? t : hp->t_decay);
  const cf::NsMomentum mom{hp->mu, 1.0 - hp->mu, hp->nesterov};
  const cf::NsUpdate up{(float)((hp->eta0 - hp->eta_min) * (1.0 - tc / (double)hp->t_decay) + hp->eta_min),
                        (float)hp->weight_decay};
  hipStream_t st = (hipStream_t)stream;
  return mats_tables(nmat, mats, CF_F32, true, [&](cf::NsTable &T, const int *rows, const int *cols, size_t) {
    for (int l = 0; l < T.count; ++l) {
      const double R = rows[l], C = cols[l];
      T.mat[l].gain = (float)(hp->scale == CF_MUON_SCALE_RMS ? 0.2 * std::sqrt(R > C ? R : C)
                                                             : std::sqrt(C > R ? C / R : 1.0));
    }
    return finish(cf::launch_newton_schulz(T, S, cf::DT_F32, g, &mom, m, &up, v, (uint16_t *)v16, ws, st), st,
                  "cf_muon_step");
  });
}

}  // extern "C"

// ---- group normalisation ----------------------------------------------------------

namespace {
cf_status act_check(int32_t act, float alpha, const char *who) {
  if (act < CF_ACT_NONE || act > CF_ACT_GELU) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": unknown activation");
  if (act == CF_ACT_LRELU && !std::isfinite(alpha))
    return fail(CF_ERR_INVALID_ARG, std::string(who) + ": alpha must be finite");
  return CF_OK;
}
static_assert((int)CF_ACT_LRELU == (int)cf::ACT_LRELU && (int)CF_ACT_SILU == (int)cf::ACT_SILU &&
                  (int)CF_ACT_GELU == (int)cf::ACT_GELU && (int)CF_ACT_NONE == (int)cf::ACT_NONE,
              "activation codes");

cf_status gn_check(int32_t n, int64_t vox, int32_t c, int32_t groups, int32_t dtype, const char *who) {
  if (n < 0 || vox < 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": n and vox must be >= 0");
  if (c <= 0 || groups <= 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": c and groups must be > 0");
  if (c % groups != 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": c is not a multiple of groups");
  if (vox >= (1LL << 31)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": more than 2^31 voxels a sample");
  if ((int64_t)(n > 0 ? n : 1) * c >= (1LL << 24)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": n * c too large");
  if ((int64_t)n * c * vox >= (1LL << 40)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": n * vox * c too large");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  return CF_OK;
}

// bytes of a workspace query: 0 for what `bad` rejects, the last error as it was
template <class Bad, class Size> size_t workspace_query(Bad bad, Size size) {
  const std::string keep = g_last_error;
  const bool b = bad() != CF_OK;
  g_last_error = keep;
  return b ? 0 : size();
}

cf_status workspace_check(const void *ws, size_t ws_bytes, size_t need, const char *who) {
  if (!need) return CF_OK;
  if (!ws || ws_bytes < need) return fail(CF_ERR_WORKSPACE, std::string(who) + ": workspace missing or smaller than its size query returns");
  if (!aligned16(ws)) return fail(CF_ERR_ALIGNMENT, "workspace not 16-byte aligned");
  return CF_OK;
}
}  // namespace

extern "C" {

size_t cf_groupnorm_fwd_workspace_size(int32_t n, int64_t vox, int32_t c, int32_t groups, int32_t dtype) {
  return workspace_query([&] { return gn_check(n, vox, c, groups, dtype, "groupnorm"); },
                         [&] { return n == 0 || vox == 0 ? 0 : cf::groupnorm_fwd_workspace(n, vox, c, groups, kdt(dtype)); });
}

cf_status cf_groupnorm_fwd(int32_t n, int64_t vox, int32_t c, int32_t groups, int32_t dtype, const void *x,
                           const float *gamma, const float *beta, float eps, int32_t act, float alpha, void *y,
                           float *mean, float *rstd, void *ws, size_t ws_bytes, void *stream) {
  const char *who = "groupnorm_fwd";
  cf_status r = gn_check(n, vox, c, groups, dtype, who);
  if (r != CF_OK || (r = act_check(act, alpha, who)) != CF_OK) return r;
  if (!std::isfinite(eps) || eps < 0.f) return fail(CF_ERR_INVALID_ARG, "groupnorm_fwd: eps must be finite and >= 0");
  if (n == 0 || vox == 0) return ok();
  if ((r = check_ptrs({x, gamma, beta, y, mean, rstd})) != CF_OK) return r;
  const size_t need = cf::groupnorm_fwd_workspace(n, vox, c, groups, kdt(dtype));
  if ((r = workspace_check(ws, ws_bytes, need, who)) != CF_OK) return r;
  const size_t nx = (size_t)n * vox * c * elem_size(dtype), nc = (size_t)c * 4, ng = (size_t)n * groups * 4;
  if ((r = norm_alias({{x, nx}, {gamma, nc}, {beta, nc}}, {{y, nx}, {mean, ng}, {rstd, ng}, {ws, need}}, y, {x}, who)) != CF_OK)
    return r;
  hipStream_t st = (hipStream_t)stream;
  return finish(cf::launch_groupnorm_fwd(n, vox, c, groups, kdt(dtype), x, gamma, beta, eps, act, alpha, y, mean, rstd, ws, st),
                st, "cf_groupnorm_fwd");
}

size_t cf_groupnorm_bwd_workspace_size(int32_t n, int64_t vox, int32_t c, int32_t groups, int32_t dtype) {
  return workspace_query([&] { return gn_check(n, vox, c, groups, dtype, "groupnorm"); },
                         [&] { return n == 0 || vox == 0 ? 0 : cf::groupnorm_bwd_workspace(n, vox, c, groups, kdt(dtype)); });
}

cf_status cf_groupnorm_bwd(int32_t n, int64_t vox, int32_t c, int32_t groups, int32_t dtype, const void *dy,
                           const void *x, const float *gamma, const float *beta, const float *mean, const float *rstd,
                           int32_t act, float alpha, void *dx, float *dgamma, float *dbeta, void *ws, size_t ws_bytes,
                           void *stream) {
  const char *who = "groupnorm_bwd";
  cf_status r = gn_check(n, vox, c, groups, dtype, who);
  if (r != CF_OK || (r = act_check(act, alpha, who)) != CF_OK) return r;
  hipStream_t st = (hipStream_t)stream;
  const size_t nc = (size_t)c * 4;
  if (n == 0 || vox == 0) {
    if ((r = check_ptrs({dgamma, dbeta})) != CF_OK) return r;
    if (overlap(dgamma, nc, dbeta, nc)) return fail(CF_ERR_ALIAS, "groupnorm_bwd: two outputs overlap");
    hipError_t e = cf::launch_fill_zero(dgamma, c, st);
    if (e == hipSuccess) e = cf::launch_fill_zero(dbeta, c, st);
    return finish(e, st, "cf_groupnorm_bwd");
  }
  if ((r = check_ptrs({dy, x, gamma, beta, mean, rstd, dx, dgamma, dbeta})) != CF_OK) return r;
  const size_t need = cf::groupnorm_bwd_workspace(n, vox, c, groups, kdt(dtype));
  if ((r = workspace_check(ws, ws_bytes, need, who)) != CF_OK) return r;
  const size_t nx = (size_t)n * vox * c * elem_size(dtype), ng = (size_t)n * groups * 4;
  if ((r = norm_alias({{dy, nx}, {x, nx}, {gamma, nc}, {beta, nc}, {mean, ng}, {rstd, ng}},
                      {{dx, nx}, {dgamma, nc}, {dbeta, nc}, {ws, need}}, dx, {dy, x}, who)) != CF_OK)
    return r;
  return finish(cf::launch_groupnorm_bwd(n, vox, c, groups, kdt(dtype), dy, x, gamma, beta, mean, rstd, act, alpha, dx,
                                         dgamma, dbeta, ws, st),
                st, "cf_groupnorm_bwd");
}

}  // extern "C"

// ---- matrix products with an epilogue -----------------------------------------------

namespace {
cf_status linear_check(int32_t m, int32_t k, int32_t n, int32_t dtype, const char *who) {
  if (m < 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": m must be >= 0");
  if (k <= 0 || n <= 0) return fail(CF_ERR_INVALID_ARG, std::string(who) + ": k and n must be > 0");
  if (k > (1 << 24) || n > (1 << 24)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": k or n past 2^24");
  for (int64_t p : {(int64_t)m * k, (int64_t)m * n, (int64_t)k * n})
    if (p >= (1LL << 40)) return fail(CF_ERR_UNSUPPORTED, std::string(who) + ": a matrix of 2^40 values or more");
  if (dtype != CF_F32 && dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "unknown dtype");
  return CF_OK;
}
cf_status optional_ptr(const void *p, const char *who) {
  return p && !aligned16(p) ? fail(CF_ERR_ALIGNMENT, std::string(who) + ": tensor pointer not 16-byte aligned") : CF_OK;
}
}  // namespace

extern "C" {

size_t cf_linear_fwd_workspace_size(int32_t m, int32_t k, int32_t n, int32_t dtype) {
  return workspace_query([&] { return linear_check(m, k, n, dtype, "linear"); },
                         [&] { return m == 0 ? 0 : cf::linear_fwd_workspace(m, k, n, kdt(dtype)); });
}
size_t cf_linear_bwd_data_workspace_size(int32_t m, int32_t k, int32_t n, int32_t dtype) {
  return workspace_query([&] { return linear_check(m, k, n, dtype, "linear"); },
                         [&] { return m == 0 ? 0 : cf::linear_bwd_data_workspace(m, k, n, kdt(dtype)); });
}
size_t cf_linear_bwd_weight_workspace_size(int32_t m, int32_t k, int32_t n, int32_t dtype) {
  return workspace_query([&] { return linear_check(m, k, n, dtype, "linear"); },
                         [&] { return m == 0 ? 0 : cf::linear_bwd_weight_workspace(m, k, n, kdt(dtype)); });
}

cf_status cf_linear_fwd(int32_t m, int32_t k, int32_t n, int32_t dtype, const void *x, const void *w, const float *bias,
                        int32_t act, float alpha, const void *residual, void *y, void *z, void *ws, size_t ws_bytes,
                        void *stream) {
  const char *who = "linear_fwd";
  cf_status r = linear_check(m, k, n, dtype, who);
  if (r != CF_OK || (r = act_check(act, alpha, who)) != CF_OK) return r;
  if (m == 0) return ok();
  if ((r = check_ptrs({x, w, y})) != CF_OK) return r;
  for (const void *p : {(const void *)bias, residual, (const void *)z})
    if ((r = optional_ptr(p, who)) != CF_OK) return r;
  const size_t need = cf::linear_fwd_workspace(m, k, n, kdt(dtype)), es = elem_size(dtype);
  if ((r = workspace_check(ws, ws_bytes, need, who)) != CF_OK) return r;
  const size_t ny = (size_t)m * n * es;
  if ((r = norm_alias({{x, (size_t)m * k * es}, {w, (size_t)k * n * es}, {bias, (size_t)n * 4}, {residual, ny}},
                      {{y, ny}, {z, ny}, {ws, need}}, y, {residual}, who)) != CF_OK)
    return r;
  hipStream_t st = (hipStream_t)stream;
  const cf::LinearEpilogue e{bias, residual, z, nullptr, act, alpha};
  return finish(cf::launch_linear_fwd(m, k, n, kdt(dtype), x, w, e, y, ws, st), st, "cf_linear_fwd");
}

cf_status cf_linear_bwd_data(int32_t m, int32_t k, int32_t n, int32_t dtype, const void *dz, const void *w,
                             const void *residual, const void *z, int32_t act, float alpha, void *dx, void *ws,
                             size_t ws_bytes, void *stream) {
  const char *who = "linear_bwd_data";
  cf_status r = linear_check(m, k, n, dtype, who);
  if (r != CF_OK || (r = act_check(act, alpha, who)) != CF_OK) return r;
  if (m == 0) return ok();
  if ((r = check_ptrs({dz, w, dx})) != CF_OK) return r;
  if (act != CF_ACT_NONE && !z) return fail(CF_ERR_INVALID_ARG, "linear_bwd_data: an activation needs z");
  if (act == CF_ACT_NONE) z = nullptr;
  for (const void *p : {residual, z})
    if ((r = optional_ptr(p, who)) != CF_OK) return r;
  const size_t need = cf::linear_bwd_data_workspace(m, k, n, kdt(dtype)), es = elem_size(dtype);
  if ((r = workspace_check(ws, ws_bytes, need, who)) != CF_OK) return r;
  const size_t nx = (size_t)m * k * es;
  if ((r = norm_alias({{dz, (size_t)m * n * es}, {w, (size_t)k * n * es}, {residual, nx}, {z, nx}}, {{dx, nx}, {ws, need}}, dx,
                      {residual, z}, who)) != CF_OK)
    return r;
  hipStream_t st = (hipStream_t)stream;
  const cf::LinearEpilogue e{nullptr, residual, nullptr, z, act, alpha};
  return finish(cf::launch_linear_bwd_data(m, k, n, kdt(dtype), dz, w, e, dx, ws, st), st, "cf_linear_bwd_data");
}

cf_status cf_linear_bwd_weight(int32_t m, int32_t k, int32_t n, int32_t dtype, const void *x, const void *dz, float *dw,
                               float *db, void *ws, size_t ws_bytes, void *stream) {
  const char *who = "linear_bwd_weight";
  cf_status r = linear_check(m, k, n, dtype, who);
  if (r != CF_OK) return r;
  hipStream_t st = (hipStream_t)stream;
  const size_t nw = (size_t)k * n * 4, nb = (size_t)n * 4;
  if ((r = check_ptrs({dw})) != CF_OK || (r = optional_ptr(db, who)) != CF_OK) return r;
  if (overlap(dw, nw, db, nb)) return fail(CF_ERR_ALIAS, "linear_bwd_weight: two outputs overlap");
  if (m == 0) {
    hipError_t e = cf::launch_fill_zero(dw, (long long)k * n, st);
    if (e == hipSuccess && db) e = cf::launch_fill_zero(db, n, st);
    return finish(e, st, "cf_linear_bwd_weight");
  }
  if ((r = check_ptrs({x, dz})) != CF_OK) return r;
  const size_t need = cf::linear_bwd_weight_workspace(m, k, n, kdt(dtype)), es = elem_size(dtype);
  if ((r = workspace_check(ws, ws_bytes, need, who)) != CF_OK) return r;
  if ((r = norm_alias({{x, (size_t)m * k * es}, {dz, (size_t)m * n * es}}, {{dw, nw}, {db, nb}, {ws, need}}, nullptr, {},
                      who)) != CF_OK)
    return r;
  return finish(cf::launch_linear_bwd_weight(m, k, n, kdt(dtype), x, dz, dw, db, ws, st), st, "cf_linear_bwd_weight");
}

}  // extern "C"

// ---- AdamW ------------------------------------------------------------------------

namespace {
constexpr int32_t kMaxTensors = 1 << 16;
constexpr int64_t kAdamwPiece = 1LL << 30;  // values of one table entry: a launch stays below 2^24 workgroups

struct Extent {
  uintptr_t beg, end;
  bool written;
};

// whether something written overlaps anything else (the extents of each role are mostly
// in ascending order already)
bool any_overlap(std::vector<Extent> &v) {
  std::sort(v.begin(), v.end(), [](const Extent &a, const Extent &b) { return a.beg < b.beg; });
  uintptr_t read_end = 0, write_end = 0;
  for (const Extent &e : v) {
    if (e.beg < write_end || (e.written && e.beg < read_end)) return true;
    uintptr_t &end = e.written ? write_end : read_end;
    end = std::max(end, e.end);
  }
  return false;
}

cf_status adamw_check(int32_t ntensors, const cf_adamw_tensor *tensors) {
  if (ntensors < 0) return fail(CF_ERR_INVALID_ARG, "adamw: ntensors must be >= 0");
  if (ntensors > kMaxTensors) return fail(CF_ERR_UNSUPPORTED, "adamw: more than 65536 tensors");
  if (ntensors > 0 && !tensors) return fail(CF_ERR_INVALID_ARG, "adamw: tensors is NULL");
  std::vector<Extent> ext;
  try {
    ext.reserve((size_t)ntensors * 7);  // (nothing further on allocates)
  } catch (const std::bad_alloc &) {
    return fail(CF_ERR_UNSUPPORTED, "adamw: no host memory for the tensors' extents");
  }
  for (int32_t l = 0; l < ntensors; ++l) {
    const cf_adamw_tensor &A = tensors[l];
    if (A.count < 0 || A.count >= (1LL << 40)) return fail(CF_ERR_INVALID_ARG, "adamw: a count is negative or past 2^40");
    if (A.g_dtype != CF_F32 && A.g_dtype != CF_BF16) return fail(CF_ERR_INVALID_ARG, "adamw: unknown g_dtype");
    if (!std::isfinite(A.weight_decay) || A.weight_decay < 0.f)
      return fail(CF_ERR_INVALID_ARG, "adamw: weight_decay must be finite and >= 0");
    if (!A.m_scale != !A.v_scale) return fail(CF_ERR_INVALID_ARG, "adamw: m_scale and v_scale must both be given or both be NULL");
    if (A.count == 0) continue;
    cf_status r;
    if ((r = check_ptrs({A.p, A.g, A.m, A.v})) != CF_OK) return r;
    const size_t n = (size_t)A.count, state = A.m_scale ? n : 4 * n, scales = (n + CF_ADAMW_BLOCK - 1) / CF_ADAMW_BLOCK * 4;
    auto add = [&](const void *p, size_t bytes, bool written) {
      if (p) ext.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written});
    };
    if ((r = optional_ptr(A.p16, "adamw")) != CF_OK) return r;
    if (((uintptr_t)A.m_scale | (uintptr_t)A.v_scale) & 3u) return fail(CF_ERR_ALIGNMENT, "adamw: scales not 4-byte aligned");
    add(A.p, 4 * n, true);
    add(A.g, n * elem_size(A.g_dtype), false);
    add(A.m, state, true);
    add(A.v, state, true);
    add(A.m_scale, scales, true);
    add(A.v_scale, scales, true);
    add(A.p16, 2 * n, true);
  }
  if (any_overlap(ext)) return fail(CF_ERR_ALIAS, "adamw: what is updated overlaps something else of the call");
  return CF_OK;
}
}  // namespace

extern "C" {

cf_status cf_adamw_step(int32_t ntensors, const cf_adamw_tensor *tensors, int64_t t, const cf_adamw_hparams *hp,
                        void *stream) {
  if (!hp) return fail(CF_ERR_INVALID_ARG, "adamw: hp is NULL");
  if (t < 0) return fail(CF_ERR_INVALID_ARG, "adamw: t must be >= 0");
  if (hp->t_decay <= 0) return fail(CF_ERR_INVALID_ARG, "adamw: t_decay must be > 0");
  for (double x : {hp->eta0, hp->eta_min, hp->beta1, hp->beta2, hp->eps})
    if (!std::isfinite(x)) return fail(CF_ERR_INVALID_ARG, "adamw: hyperparameters must be finite");
  if (hp->beta1 < 0.0 || hp->beta1 >= 1.0 || hp->beta2 < 0.0 || hp->beta2 >= 1.0)
    return fail(CF_ERR_INVALID_ARG, "adamw: beta1 and beta2 must lie in [0, 1)");
  if (hp->eps < 0.0) return fail(CF_ERR_INVALID_ARG, "adamw: eps must be >= 0");
  cf_status r = adamw_check(ntensors, tensors);
  if (r != CF_OK) return r;
  const double tc = (double)(t < hp->t_decay ? t : hp->t_decay), k = (double)t + 1.0;
  const double eta = (hp->eta0 - hp->eta_min) * (1.0 - tc / (double)hp->t_decay) + hp->eta_min;
  const cf::AdamwStep step{(float)hp->beta1, (float)(1.0 - hp->beta1), (float)hp->beta2, (float)(1.0 - hp->beta2),
                           (float)(1.0 / std::sqrt(1.0 - std::pow(hp->beta2, k))), (float)hp->eps,
                           (float)(eta / (1.0 - std::pow(hp->beta1, k)))};
  hipStream_t st = (hipStream_t)stream;
  cf::AdamwTable T;
  T.count = 0;
  int64_t total = 0;
  auto flush = [&] {
    const hipError_t e = T.count ? cf::launch_adamw(T, step, st) : hipSuccess;
    T.count = 0;
    total = 0;
    return finish(e, st, "cf_adamw_step");
  };
  for (int32_t l = 0; l < ntensors; ++l) {
    const cf_adamw_tensor &A = tensors[l];
    const int es = (int)elem_size(A.g_dtype), ss = A.m_scale ? 1 : 4;
    const uint32_t key = cf::adamw_key(hp->seed, t, l);
    const volatile float decayed = (float)eta * A.weight_decay;  // rounded by itself
    for (int64_t at = 0; at < A.count; at += kAdamwPiece) {
      const int64_t n = std::min(kAdamwPiece, A.count - at);
      if (T.count == cf::kAdamwTable || total + n > 4 * kAdamwPiece)
        if ((r = flush()) != CF_OK) return r;
      cf::AdamwTensor &B = T.t[T.count++];
      total += n;
      B.p = A.p + at;
      B.g = (const char *)A.g + at * es;
      B.m = (char *)A.m + at * ss;
      B.v = (char *)A.v + at * ss;
      B.ms = A.m_scale ? A.m_scale + at / CF_ADAMW_BLOCK : nullptr;
      B.vs = A.v_scale ? A.v_scale + at / CF_ADAMW_BLOCK : nullptr;
      B.p16 = A.p16 ? (uint16_t *)A.p16 + at : nullptr;
      B.count = n;
      B.key = key + (uint32_t)at * 0x9E3779B9u;
      B.keep = 1.f - decayed;
      B.first = 0;
      B.g16 = A.g_dtype == CF_BF16;
    }
  }
  return flush();
}

}  // extern "C"
