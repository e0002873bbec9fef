// Single-operation entry points of the C ABI: thin argument checks around the kernel
// launchers, for per-layer parity tests and roofline measurements.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <new>
#include <vector>

#include "../../include/accudnn.h"
#include "kernels.h"
#include "dtype.h"

using namespace acc;

namespace {
inline size_t al256(size_t b) { return (b + 255) & ~(size_t)255; }
inline int out_dim(int in, int r, int stride, int pad) { return (in + 2 * pad - r) / stride + 1; }
inline bool conv_ok(int n, int h, int w, int cin, int cout, int r, int s, int stride, int pad) {
  return n > 0 && h > 0 && w > 0 && cin > 0 && cout > 0 && r > 0 && s == r && stride > 0 && pad >= 0 && pad < r &&
         h + 2 * pad >= r && w + 2 * pad >= s;
}
inline bool dtype_ok(int dt) { return dt == ACC_F32 || dt == ACC_BF16; }
// the kernels move 16 bytes at a time: null is let through here (checked where it matters)
inline bool al16(std::initializer_list<const void*> ps) {
  for (const void* p : ps) if (reinterpret_cast<uintptr_t>(p) & 15) return false;
  return true;
}
inline int status(hipError_t e) { return e == hipSuccess ? ACC_OK : (e == hipErrorInvalidValue ? ACC_EINVAL : ACC_EHIP); }
}  // namespace

extern "C" size_t acc_op_conv_workspace(int n, int h, int w, int cin, int cout, int r, int s, int stride, int pad) {
  if (!conv_ok(n, h, w, cin, cout, r, s, stride, pad)) return 0;
  const int ho = out_dim(h, r, stride, pad), wo = out_dim(w, s, stride, pad);
  // the sub-filters of a strided data gradient are aligned one by one
  return al256(wgrad_workspace_bytes(n, ho, wo, cin, cout, r, s, -1)) + al256((size_t)cout * cin * r * s * sizeof(float)) +
         (stride > 1 ? kMaxDgradParts * 256 : 0);
}

namespace {
int conv_fwd(const void* x, const void* w, void* y, int n, int h, int wd, int cin, int cout, int r, int s, int stride, int pad,
             int dtype, hipStream_t st, LaunchProbe* probe) {
  if (!x || !w || !y || !dtype_ok(dtype) || !conv_ok(n, h, wd, cin, cout, r, s, stride, pad)) return ACC_EINVAL;
  if (!al16({x, w, y})) return ACC_EINVAL;
  ConvGeom g{};
  g.in = x; g.w = w; g.out = y; g.dtype = dtype;
  g.n_img = n; g.h = h; g.wd = wd; g.c = cin;
  g.p = out_dim(h, r, stride, pad); g.q = out_dim(wd, s, stride, pad); g.n_out = cout;
  g.r = r; g.s = s; g.stride = stride; g.pad = pad;
  g.out_h = g.p; g.out_w = g.q; g.out_stride = 1;
  return status(conv_igemm(g, st, probe));
}

int conv_dgrad(const void* dy, const void* w, void* dx, int n, int h, int wd, int cin, int cout, int r, int s, int stride, int pad,
               int accumulate, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st, LaunchProbe* probe) {
  if (!dy || !w || !dx || !dtype_ok(dtype) || !conv_ok(n, h, wd, cin, cout, r, s, stride, pad)) return ACC_EINVAL;
  if (!al16({dy, w, dx, workspace})) return ACC_EINVAL;
  const bool dry = probe && probe->dry;
  const int ho = out_dim(h, r, stride, pad), wo = out_dim(wd, s, stride, pad);
  hipError_t e;
  if (stride > 1 && (r > 1 || pad > 0)) {
    // one stride-1 convolution per residue class of the dx position
    DgradPart parts[kMaxDgradParts];
    bool covers_all = false;
    size_t wt_bytes = 0;
    const int np = dgrad_split(h, wd, cin, cout, r, s, stride, pad, (int)dt_size(dtype), parts, &covers_all, &wt_bytes);
    if (np < 0 || !workspace || workspace_bytes < wt_bytes) return ACC_EINVAL;
    if (!covers_all && !accumulate) {
      const size_t bytes = (size_t)n * h * wd * cin * dt_size(dtype);
      if (bytes % 4) return ACC_EINVAL;
      if (!dry && (e = fill_zero((float*)dx, bytes / 4, st)) != hipSuccess) return status(e);
    }
    if (np == 0) return ACC_OK;      // no position of dx has a tap
    const DgradSplit split{w, cout, cin, r, s, stride, parts, np};
    ConvGeom g{};
    g.in = dy; g.w = workspace; g.out = dx; g.dtype = dtype;
    g.n_img = n; g.h = ho; g.wd = wo; g.c = cout; g.n_out = cin;
    g.out_h = h; g.out_w = wd; g.accumulate = accumulate;
    g.split = &split;
    return status(conv_igemm(g, st, probe));
  }
  const size_t filt = al256((size_t)cout * cin * r * s * sizeof(float));
  if (!workspace || workspace_bytes < filt) return ACC_EINVAL;
  void* wt = workspace;
  ConvGeom g{};
  g.in = dy; g.out = dx; g.dtype = dtype;
  g.n_img = n; g.h = ho; g.wd = wo; g.c = cout; g.n_out = cin;
  g.r = r; g.s = s; g.stride = 1; g.accumulate = accumulate;
  g.out_h = h; g.out_w = wd;
  if (stride == 1) {
    g.p = h; g.q = wd; g.pad = r - 1 - pad; g.out_stride = 1;
  } else {
    g.p = ho; g.q = wo; g.pad = 0; g.out_stride = stride;
    if (!accumulate) {
      const size_t bytes = (size_t)n * h * wd * cin * dt_size(dtype);
      if (bytes % 4) return ACC_EINVAL;
      if (!dry && (e = fill_zero((float*)dx, bytes / 4, st)) != hipSuccess) return status(e);
    }
  }
  g.w_kn = w;
  if (dtype == DT_BF16 && conv_igemm_bf16_takes(g, (long)n * g.p * g.q, (long)r * s * cout)) return status(conv_igemm(g, st, probe));   // reads the filter as it lies
  if (r != 1) g.w_kn = nullptr;
  if (!g.w_kn || !conv_igemm_rows_takes(g, (long)n * g.p * g.q, cout)) {     // that kernel reads the filter as it lies
    g.w = wt;
    g.w_kn = nullptr;
    if (!dry && (e = filter_flip_transpose(w, wt, cout, cin, r, s, dtype, st)) != hipSuccess) return status(e);
  }
  return status(conv_igemm(g, st, probe));
}

int conv_wgrad_op(const void* x, const void* dy, float* dw, int n, int h, int wd, int cin, int cout, int r, int s, int stride, int pad,
                  void* workspace, size_t workspace_bytes, int dtype, hipStream_t st, LaunchProbe* probe) {
  if (!x || !dy || !dw || !dtype_ok(dtype) || !conv_ok(n, h, wd, cin, cout, r, s, stride, pad)) return ACC_EINVAL;
  if (!al16({x, dy, dw, workspace})) return ACC_EINVAL;
  const int ho = out_dim(h, r, stride, pad), wo = out_dim(wd, s, stride, pad);
  const size_t need = wgrad_workspace_least(n, ho, wo, cin, cout, r, s, dtype);
  if (need && (!workspace || workspace_bytes < need)) return ACC_EINVAL;
  WgradGeom g{};
  g.x = x; g.dy = dy; g.dw = dw; g.dtype = dtype;
  g.n_img = n; g.h = h; g.wd = wd; g.cin = cin; g.p = ho; g.q = wo; g.cout = cout;
  g.r = r; g.s = s; g.stride = stride; g.pad = pad; g.workspace = (float*)workspace; g.workspace_bytes = workspace ? workspace_bytes : 0;
  return status(conv_wgrad(g, st, probe));
}
}  // namespace

extern "C" int acc_op_conv_fwd(const void* x, const void* w, void* y, int n, int h, int wd, int cin, int cout,
                               int r, int s, int stride, int pad, int dtype, void* stream) {
  return conv_fwd(x, w, y, n, h, wd, cin, cout, r, s, stride, pad, dtype, (hipStream_t)stream, nullptr);
}

extern "C" int acc_op_conv_dgrad(const void* dy, const void* w, void* dx, int n, int h, int wd, int cin, int cout,
                                 int r, int s, int stride, int pad, int accumulate, void* workspace,
                                 size_t workspace_bytes, int dtype, void* stream) {
  return conv_dgrad(dy, w, dx, n, h, wd, cin, cout, r, s, stride, pad, accumulate, workspace, workspace_bytes, dtype,
                    (hipStream_t)stream, nullptr);
}

extern "C" int acc_op_conv_wgrad(const void* x, const void* dy, float* dw, int n, int h, int wd, int cin, int cout,
                                 int r, int s, int stride, int pad, void* workspace, size_t workspace_bytes,
                                 int dtype, void* stream) {
  return conv_wgrad_op(x, dy, dw, n, h, wd, cin, cout, r, s, stride, pad, workspace, workspace_bytes, dtype,
                       (hipStream_t)stream, nullptr);
}

extern "C" const char* acc_op_conv_kernel(int role, int n, int h, int wd, int cin, int cout, int r, int s, int stride, int pad,
                                          int dtype) {
  LaunchProbe probe;
  probe.dry = true;
  float* const p = reinterpret_cast<float*>((uintptr_t)4096);      // any aligned address: nothing reads it
  const size_t all = ~(size_t)0;
  const int rc = role == 0 ? conv_fwd(p, p, p, n, h, wd, cin, cout, r, s, stride, pad, dtype, nullptr, &probe)
                 : role == 1 ? conv_dgrad(p, p, p, n, h, wd, cin, cout, r, s, stride, pad, 0, p, all, dtype, nullptr, &probe)
                 : role == 2 ? conv_wgrad_op(p, p, p, n, h, wd, cin, cout, r, s, stride, pad, p, all, dtype, nullptr, &probe)
                             : ACC_EINVAL;
  return rc != ACC_OK ? nullptr : probe.kernel ? probe.kernel : "none";
}


extern "C" size_t acc_op_bn_workspace(int c) { return c > 0 ? al256(bn_workspace_bytes(c)) : 0; }

extern "C" int acc_op_bn_fwd(const void* x, const float* gamma, const float* beta, const void* res, void* y,
                             float* mean, float* istd, int rows, int c, int relu, float eps, void* workspace,
                             int dtype, void* stream) {
  if (!dtype_ok(dtype) || !al16({x, gamma, beta, res, y, mean, istd, workspace})) return ACC_EINVAL;
  return status(bn_forward(x, gamma, beta, res, y, mean, istd, rows, c, relu, eps, workspace, dtype,
                           (hipStream_t)stream));
}

extern "C" int acc_op_bn_bwd(const void* x, const void* dy, const void* y, const float* gamma, const float* mean,
                             const float* istd, void* dx, float* dgamma, float* dbeta, void* g_out, int rows, int c,
                             void* workspace, int dtype, void* stream) {
  if (!dtype_ok(dtype) || !al16({x, dy, y, gamma, mean, istd, dx, dgamma, dbeta, g_out, workspace})) return ACC_EINVAL;
  return status(bn_backward(x, dy, y, gamma, mean, istd, dx, dgamma, dbeta, g_out, rows, c, workspace, dtype,
                            (hipStream_t)stream));
}

extern "C" int acc_op_maxpool_fwd(const void* x, void* y, int n, int h, int wd, int c, int r, int stride, int pad,
                                  int dtype, void* stream) {
  if (!x || !y || !dtype_ok(dtype) || !al16({x, y})) return ACC_EINVAL;
  return status(maxpool_forward(x, y, n, h, wd, c, r, r, stride, pad, dtype, (hipStream_t)stream));
}

extern "C" int acc_op_maxpool_bwd(const void* x, const void* dy, void* dx, int n, int h, int wd, int c, int r,
                                  int stride, int pad, int accumulate, int dtype, void* stream) {
  if (!x || !dy || !dx || !dtype_ok(dtype) || !al16({x, dy, dx})) return ACC_EINVAL;
  return status(maxpool_backward(x, dy, dx, n, h, wd, c, r, r, stride, pad, accumulate, dtype, (hipStream_t)stream));
}

extern "C" int acc_op_gap_fwd(const void* x, void* y, int n, int hw, int c, int dtype, void* stream) {
  if (!x || !y || !dtype_ok(dtype)) return ACC_EINVAL;
  return status(gap_forward(x, y, n, hw, c, dtype, (hipStream_t)stream));
}

extern "C" int acc_op_gap_bwd(const void* dy, void* dx, int n, int hw, int c, int accumulate, int dtype, void* stream) {
  if (!dy || !dx || !dtype_ok(dtype)) return ACC_EINVAL;
  return status(gap_backward(dy, dx, n, hw, c, accumulate, dtype, (hipStream_t)stream));
}

extern "C" int acc_op_softmax_ce(const void* z, const int32_t* labels, float* loss_rows, float* loss, void* dz, int n,
                                 int classes, int dtype, void* stream) {
  if (!z || !labels || !dtype_ok(dtype) || n <= 0 || classes <= 0 || (!loss_rows && !dz) || (loss_rows && !loss))
    return ACC_EINVAL;
  return status(softmax_ce(z, labels, loss_rows, loss, dz, n, classes, dtype, (hipStream_t)stream));
}

// The text of a refusal for acc_last_error(NULL).
static int refuse(const char* text) {
  set_thread_error(text);
  return ACC_EINVAL;
}
static int told(hipError_t e, const char* text) {
  if (e == hipSuccess) return ACC_OK;
  set_thread_error(e == hipErrorInvalidValue ? text : hipGetErrorString(e));
  return status(e);
}

// What a call writes must not overlap anything else that it is given, but for tensors of the same kind that begin at the same address where a value is read
// by the thread that writes it (`over`).  Null: not given.
struct Given {
  const void* p;
  size_t bytes;
  const void* over[2];
};
static bool clash(std::initializer_list<Given> written, std::initializer_list<Given> read) {
  auto meet = [](const Given& a, const Given& b) {
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return x && y && x < y + b.bytes && y < x + a.bytes;
  };
  for (const Given* w = written.begin(); w != written.end(); ++w) {
    for (const Given* v = w + 1; v != written.end(); ++v)
      if (meet(*w, *v)) return true;
    for (const Given& r : read)
      if (meet(*w, r) && !(w->p == r.p && w->bytes == r.bytes && (w->over[0] == r.p || w->over[1] == r.p))) return true;
  }
  return false;
}
// sizes that the launchers look at (and may refuse) anyway: here only that the products below don't overflow
static bool sizes_ok(int a, int b, int c) { return a > 0 && b > 0 && c > 0 && (double)a * b * c < 1e15; }

extern "C" size_t acc_op_gn_workspace(int n, int hw, int c, int groups) { return al256(gn_workspace_bytes(n, hw, c, groups)); }

extern "C" int acc_op_gn_fwd(const void* x, const float* gamma, const float* beta, const void* res, void* y, float* mean, float* istd, int n, int hw,
                             int c, int groups, int act, float eps, void* workspace, size_t workspace_bytes, int dtype, void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_gn_fwd: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({x, gamma, beta, res, y, mean, istd, workspace})) return refuse("acc_op_gn_fwd: pointers must be 16-byte aligned");
  if (sizes_ok(n, hw, c) && groups > 0) {
    const size_t map = (size_t)n * hw * c * dt_size(dtype), row = (size_t)c * 4, stats = (size_t)n * groups * 4;
    if (clash({{y, map, {x, res}}, {mean, stats, {}}, {istd, stats, {}}, {workspace, workspace_bytes, {}}},
              {{x, map, {}}, {res, map, {}}, {gamma, row, {}}, {beta, row, {}}}))
      return refuse("acc_op_gn_fwd: what is written overlaps another argument (y may be x or res)");
  }
  return told(gn_forward(x, gamma, beta, res, y, mean, istd, n, hw, c, groups, act, eps, workspace, workspace_bytes, dtype, (hipStream_t)stream),
              "acc_op_gn_fwd: null pointer, sizes that are not positive or too large, groups that do not divide c, unknown act, eps < 0 or a workspace "
              "smaller than acc_op_gn_workspace()");
}

extern "C" int acc_op_gn_bwd(const void* x, const void* dy, const void* y, const void* res, const float* gamma, const float* beta, const float* mean,
                             const float* istd, void* dx, float* dgamma, float* dbeta, void* dres, int n, int hw, int c, int groups, int act,
                             void* workspace, size_t workspace_bytes, int dtype, void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_gn_bwd: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({x, dy, y, res, gamma, beta, mean, istd, dx, dgamma, dbeta, dres, workspace})) return refuse("acc_op_gn_bwd: pointers must be 16-byte aligned");
  if (sizes_ok(n, hw, c) && groups > 0) {
    const size_t map = (size_t)n * hw * c * dt_size(dtype), row = (size_t)c * 4, stats = (size_t)n * groups * 4;
    if (clash({{dx, map, {x, dy}}, {dres, map, {dy}}, {dgamma, row, {}}, {dbeta, row, {}}, {workspace, workspace_bytes, {}}},
              {{x, map, {}}, {dy, map, {}}, {act == ACC_ACT_RELU ? y : nullptr, map, {}}, {act == ACC_ACT_SILU ? res : nullptr, map, {}}, {gamma, row, {}},
               {beta, row, {}}, {mean, stats, {}}, {istd, stats, {}}}))
      return refuse("acc_op_gn_bwd: what is written overlaps another argument (dx may be x or dy, dres may be dy)");
  }
  return told(gn_backward(x, dy, y, res, gamma, beta, mean, istd, dx, dgamma, dbeta, dres, n, hw, c, groups, act, workspace, workspace_bytes, dtype,
                          (hipStream_t)stream),
              "acc_op_gn_bwd: null pointer (y is needed with ACC_ACT_RELU), sizes that are not positive or too large, groups that do not divide c, "
              "unknown act or a workspace smaller than acc_op_gn_workspace()");
}

extern "C" size_t acc_op_linear_ce_workspace(int n, int d, int classes, int gradients, int dtype) {
  return linear_ce_workspace_bytes(n, d, classes, gradients, dtype);
}

extern "C" int acc_op_linear_ce(const void* x, const void* w, const float* bias, const int32_t* labels, int ignore, float* loss_rows, float* loss,
                                void* dx, float* dw, float* db, int n, int d, int classes, void* workspace, size_t workspace_bytes, int dtype,
                                void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_linear_ce: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({x, w, bias, labels, loss_rows, loss, dx, dw, db, workspace})) return refuse("acc_op_linear_ce: pointers must be 16-byte aligned");
  if (sizes_ok(n, d, classes)) {
    const size_t es = dt_size(dtype), nx = (size_t)n * d, nw = (size_t)classes * d;
    if (clash({{loss_rows, (size_t)n * 4, {}}, {loss, 4, {}}, {dx, nx * es, {}}, {dw, nw * 4, {}}, {db, (size_t)classes * 4, {}}, {workspace, workspace_bytes, {}}},
              {{x, nx * es, {}}, {w, nw * es, {}}, {bias, (size_t)classes * 4, {}}, {labels, (size_t)n * 4, {}}}))
      return refuse("acc_op_linear_ce: what is written overlaps another argument");
  }
  return told(linear_ce(x, w, bias, labels, ignore, loss_rows, loss, dx, dw, db, n, d, classes, workspace, workspace_bytes, dtype, (hipStream_t)stream),
              "acc_op_linear_ce: null pointer, no result asked for, sizes that are not positive or too large, or a workspace smaller than "
              "acc_op_linear_ce_workspace()");
}

extern "C" size_t acc_op_glu_workspace(int rows, int d, int f, int backward, int dtype) { return glu_workspace_bytes(rows, d, f, backward, dtype); }

extern "C" int acc_op_glu_fwd(const void* x, const void* w, const float* bias, void* h, void* ab, int rows, int d, int f, int act, void* workspace,
                              size_t workspace_bytes, int dtype, void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_glu_fwd: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({x, w, bias, h, ab, workspace})) return refuse("acc_op_glu_fwd: pointers must be 16-byte aligned");
  if (sizes_ok(rows, d, 1) && sizes_ok(rows, f, 1)) {
    const size_t es = dt_size(dtype), nh = (size_t)rows * f * es;
    if (clash({{h, nh, {}}, {ab, 2 * nh, {}}, {workspace, workspace_bytes, {}}},
              {{x, (size_t)rows * d * es, {}}, {w, 2 * (size_t)f * d * es, {}}, {bias, 2 * (size_t)f * 4, {}}}))
      return refuse("acc_op_glu_fwd: what is written overlaps another argument");
  }
  return told(glu_forward(x, w, bias, h, ab, rows, d, f, act, workspace, workspace_bytes, dtype, (hipStream_t)stream),
              "acc_op_glu_fwd: null pointer, sizes that are not positive or too large, unknown act or a workspace smaller than acc_op_glu_workspace()");
}

extern "C" int acc_op_glu_bwd(const void* x, const void* w, const float* bias, const void* ab, const void* dh, void* dx, float* dw, float* db, int rows, int d,
                              int f, int act, void* workspace, size_t workspace_bytes, int dtype, void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_glu_bwd: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({x, w, bias, ab, dh, dx, dw, db, workspace})) return refuse("acc_op_glu_bwd: pointers must be 16-byte aligned");
  if (sizes_ok(rows, d, 1) && sizes_ok(rows, f, 1)) {
    const size_t es = dt_size(dtype), nx = (size_t)rows * d * es, nh = (size_t)rows * f * es, nw = 2 * (size_t)f * d, nb = 2 * (size_t)f * 4;
    if (clash({{dx, nx, {}}, {dw, nw * 4, {}}, {db, nb, {}}, {workspace, workspace_bytes, {}}},
              {{x, nx, {}}, {w, nw * es, {}}, {ab ? nullptr : bias, nb, {}}, {ab, 2 * nh, {}}, {dh, nh, {}}}))
      return refuse("acc_op_glu_bwd: what is written overlaps another argument");
  }
  return told(glu_backward(x, w, bias, ab, dh, dx, dw, db, rows, d, f, act, workspace, workspace_bytes, dtype, (hipStream_t)stream),
              "acc_op_glu_bwd: null pointer, no result asked for, sizes that are not positive or too large, unknown act or a workspace smaller than "
              "acc_op_glu_workspace()");
}

extern "C" size_t acc_op_top_logits_workspace(int n, int classes, int k, int dtype) { return top_logits_workspace_bytes(n, classes, k, dtype); }

extern "C" int acc_op_top_logits(const void* z, int32_t* index, float* top, int n, int classes, int k, void* workspace, size_t workspace_bytes, int dtype,
                                 void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_top_logits: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({z, index, top, workspace})) return refuse("acc_op_top_logits: pointers must be 16-byte aligned");
  if (sizes_ok(n, classes, 1) && k > 0) {
    const size_t list = (size_t)n * k * 4;
    if (clash({{index, list, {}}, {top, list, {}}, {workspace, workspace_bytes, {}}}, {{z, (size_t)n * classes * dt_size(dtype), {}}}))
      return refuse("acc_op_top_logits: what is written overlaps another argument");
  }
  return told(top_logits(z, index, top, n, classes, k, workspace, workspace_bytes, dtype, (hipStream_t)stream),
              "acc_op_top_logits: null pointer, sizes that are not positive or too large, more entries than classes or a workspace smaller than "
              "acc_op_top_logits_workspace()");
}

extern "C" size_t acc_op_distill_workspace(int n, int classes, int k, int dtype) { return distill_workspace_bytes(n, classes, k, dtype); }

extern "C" int acc_op_distill(const void* z, const int32_t* index, const float* top, const int32_t* labels, int ignore, float temperature, float alpha,
                              float* loss_rows, float* loss, void* dz, int n, int classes, int k, void* workspace, size_t workspace_bytes, int dtype,
                              void* stream) {
  if (!dtype_ok(dtype)) return refuse("acc_op_distill: dtype must be ACC_F32 or ACC_BF16");
  if (!al16({z, index, top, labels, loss_rows, loss, dz, workspace})) return refuse("acc_op_distill: pointers must be 16-byte aligned");
  if (!(temperature >= 1e-18f && temperature <= 1e18f)) return refuse("acc_op_distill: the temperature must lie in [1e-18, 1e18]");      // (its square is a fp32 number)
  if (!(alpha > 0.f && alpha <= 1.f) || (!labels && alpha != 1.f)) return refuse("acc_op_distill: alpha must lie in (0, 1], and be 1 without labels");
  if (sizes_ok(n, classes, 1) && k > 0) {
    const size_t list = (size_t)n * k * 4, rows = (size_t)n * 4, map = (size_t)n * classes * dt_size(dtype);
    if (clash({{loss_rows, rows, {}}, {loss, 4, {}}, {dz, map, {z}}, {workspace, workspace_bytes, {}}},
              {{z, map, {}}, {index, list, {}}, {top, list, {}}, {labels, rows, {}}}))
      return refuse("acc_op_distill: what is written overlaps another argument (dz may be z)");
  }
  return told(distill(z, index, top, labels, ignore, temperature, alpha, loss_rows, loss, dz, n, classes, k, workspace, workspace_bytes, dtype,
                      (hipStream_t)stream),
              "acc_op_distill: null pointer, no result asked for, sizes that are not positive or too large, or a workspace smaller than "
              "acc_op_distill_workspace()");
}

extern "C" size_t acc_op_tensor_list_bytes(const size_t* counts, int n) {
  if (!counts || n <= 0) return 0;
  const size_t b = tensor_list_bytes(counts, n);
  return b ? al256(b) : 0;
}

extern "C" int acc_op_tensor_list(const void* const* src, void* const* dst, const size_t* counts, const int32_t* dtypes, int n, void* list,
                                  size_t list_bytes, void* stream) {
  if (!src || !counts || !dtypes || n <= 0 || !list) return refuse("acc_op_tensor_list: null pointer or no tensors");
  if (!al16({list})) return refuse("acc_op_tensor_list: the list must be 16-byte aligned");
  const size_t need = acc_op_tensor_list_bytes(counts, n);
  if (!need || list_bytes < need) return refuse("acc_op_tensor_list: the list is smaller than acc_op_tensor_list_bytes(), or too long");
  try {
    // what is written must not overlap what another tensor of the list reads or writes: pieces run at once
    struct Span { uintptr_t lo, hi; int tensor; bool written; };
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)n + 1);
    spans.push_back(Span{(uintptr_t)list, (uintptr_t)list + need, -1, true});      // the list itself
    for (int i = 0; i < n; ++i) {
      if (!dtype_ok(dtypes[i])) return refuse("acc_op_tensor_list: dtypes must be ACC_F32 or ACC_BF16");
      if (!counts[i]) continue;
      const uintptr_t es = dt_size(dtypes[i]), from = (uintptr_t)src[i], to = dst ? (uintptr_t)dst[i] : from;
      if (!from || !to || from % es || to % es) return refuse("acc_op_tensor_list: null or misaligned tensor");
      spans.push_back(Span{to, to + counts[i] * es, i, true});
      if (from != to) spans.push_back(Span{from, from + counts[i] * es, i, false});
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    uintptr_t end = 0, end_written = 0;              // the furthest end so far, of all and of what is written
    for (const Span& s : spans) {
      if (s.written ? s.lo < end : s.lo < end_written) return refuse("acc_op_tensor_list: tensors overlap one another (or the same one is listed twice) or the list's memory");
      end = std::max(end, s.hi);
      if (s.written) end_written = std::max(end_written, s.hi);
    }
  } catch (const std::bad_alloc&) {
    set_thread_error("acc_op_tensor_list: out of host memory");
    return ACC_EHOSTMEM;
  }
  return told(tensor_list(src, dst, counts, dtypes, n, list, (hipStream_t)stream), "acc_op_tensor_list: too long");
}

extern "C" int acc_set_grad_clip(acc_ctx* ctx, float max_norm) {
  if (!ctx) return refuse("acc_set_grad_clip: no context");
  if (!(max_norm >= 0.f)) return refuse("acc_set_grad_clip: max_norm negative or no number");
  return set_clipped_update(ctx, max_norm > 0.f ? sgd_update_clipped : nullptr, max_norm);
}

extern "C" size_t acc_op_grad_norm_workspace(void) { return grad_norm_workspace_bytes(); }

extern "C" int acc_op_grad_norm(const void* list, size_t list_bytes, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (!al16({list, norm, workspace})) return refuse("acc_op_grad_norm: pointers must be 16-byte aligned");
  if (workspace_bytes < grad_norm_workspace_bytes()) return refuse("acc_op_grad_norm: workspace smaller than acc_op_grad_norm_workspace()");
  if (clash({{norm, 4, {}}, {workspace, workspace_bytes, {}}}, {{list, list_bytes, {}}})) return refuse("acc_op_grad_norm: list, norm and workspace overlap");
  return told(grad_norm(list, list_bytes, norm, workspace, (hipStream_t)stream), "acc_op_grad_norm: null pointer or no list");
}

extern "C" int acc_op_grad_clip(const void* list, size_t list_bytes, float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (!al16({list, norm, workspace})) return refuse("acc_op_grad_clip: pointers must be 16-byte aligned");
  if (workspace_bytes < grad_norm_workspace_bytes()) return refuse("acc_op_grad_clip: workspace smaller than acc_op_grad_norm_workspace()");
  if (clash({{norm, 4, {}}, {workspace, workspace_bytes, {}}}, {{list, list_bytes, {}}})) return refuse("acc_op_grad_clip: list, norm and workspace overlap");
  return told(grad_clip(list, list_bytes, max_norm, norm, workspace, (hipStream_t)stream), "acc_op_grad_clip: null pointer, no list, or max_norm negative or no number");
}
