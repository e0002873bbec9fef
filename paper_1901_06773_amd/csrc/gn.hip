// Group normalisation of an NHWC tensor, fused with the residual add and the activation that follow it.
//
//   x[n][hw][c], groups of `per` = c / groups channels, m = hw * per values of one image each:
//   mu = sum x / m,  istd = (sum (x - mu)^2 / m + eps)^(-1/2),  z = gamma * (x - mu) * istd + beta (+ res),  y = act(z)
//   backward: g = dy * act'(z); dbeta = sum g, dgamma = sum g * xhat over images and map; with a = g * gamma and the means A of a and
//   B of a * xhat over a group of an image: dx = istd * (a - A - xhat * B), and the residual's gradient is g.
//   The mask of a ReLU comes from the stored output, the derivative of a SiLU from z, worked out again from x (and res).
//
// Bound by memory.  A sum over rows is a sum per channel first, in a fixed order, then over the channels of a group: no atomics.
#include "kernels.h"
#include "dtype.h"

namespace acc {
namespace {

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2 };

// V neighbouring values: sixteen bytes, eight, or one at a time where rows do not start on such an address.
template <class T, int V> struct Vec;
template <class T> struct Vec<T, 1> {
  T raw;
  __device__ __forceinline__ void load(const T* p) { raw = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = raw; }
  __device__ __forceinline__ float get(int) const { return Elem<T>::load(&raw); }
  __device__ __forceinline__ void set(const float (&v)[1]) { Elem<T>::store(&raw, v[0]); }
};
template <> struct Vec<float, 4> {
  float4 raw;
  __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = raw; }
  __device__ __forceinline__ float get(int i) const { return i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w; }
  __device__ __forceinline__ void set(const float (&v)[4]) { raw = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<bf16_t, 8> {
  uint4 raw;
  __device__ __forceinline__ void load(const bf16_t* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<uint4*>(p) = raw; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? raw.x : i < 4 ? raw.y : i < 6 ? raw.z : raw.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)float_to_bf16(v[2 * i]) | ((uint32_t)float_to_bf16(v[2 * i + 1]) << 16);
    raw = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
template <int ACT> __device__ __forceinline__ float act(float z) {
  if (ACT == ACT_RELU) return z < 0.f ? 0.f : z;       // (a value that is no number stays none)
  if (ACT == ACT_SILU) return z * sigmoid(z);
  return z;
}
__device__ __forceinline__ float silu_slope(float z) {
  const float s = sigmoid(z);
  return s * (1.f + z * (1.f - s));
}

// ---------------------------------------------------------------------------------- any size: sums, finish, apply
//
// The rows of an image are cut into slabs; a workgroup adds up, per channel, the rows of one slab for up to THREADS groups of V
// channels, in fp64 (the square of a mean is subtracted from the mean of squares), and leaves part[image][slab][2][c].
constexpr int THREADS = 256;
constexpr int U = 4;                                   // rows of a thread in flight

struct Cover {
  int hw, c, groups, per;
  int tpr, rpi, slices;                                // threads across a row of one slice, rows per trip, slices of channels
  int slabs, rows_per_slab;
};

template <int ACT, class T, int V>
__device__ __forceinline__ float slope_times(float dy, float y, float x, float mu, float istd, float ga, float be, float res) {
  if (ACT == ACT_RELU) return y > 0.f ? dy : 0.f;
  if (ACT == ACT_SILU) return dy * silu_slope(fmaf((x - mu) * istd, ga, be) + res);
  return dy;
}

// BWD 0: (x, x*x).  BWD 1: (g, g * xhat).  side: the stored output (ReLU) or the residual (SiLU; may be null).
template <int BWD, int ACT, class T, int V>
__global__ __launch_bounds__(THREADS) void gn_sums_kernel(const T* __restrict__ x, const T* __restrict__ dy, const T* __restrict__ side,
                                                          const float* __restrict__ gamma, const float* __restrict__ beta,
                                                          const float* __restrict__ mean, const float* __restrict__ istd,
                                                          double* __restrict__ part, Cover cv) {
  __shared__ double red[2][THREADS][V];
  const int tid = threadIdx.x, lane_r = tid / cv.tpr, lane_c = tid - lane_r * cv.tpr;
  const int slice = blockIdx.x % cv.slices, rest = blockIdx.x / cv.slices, slab = rest % cv.slabs, img = rest / cv.slabs;
  const int ch = (slice * cv.tpr + lane_c) * V;
  const bool active = lane_r < cv.rpi && ch < cv.c;
  double s0[V], s1[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.0;
  if (active) {
    float mu[V], is[V], ga[V], be[V];
    if (BWD) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int g = (ch + j) / cv.per;
        mu[j] = mean[(size_t)img * cv.groups + g];
        is[j] = istd[(size_t)img * cv.groups + g];
        ga[j] = ACT == ACT_SILU ? gamma[ch + j] : 0.f;
        be[j] = ACT == ACT_SILU ? beta[ch + j] : 0.f;
      }
    }
    const int lo = slab * cv.rows_per_slab, hi = min(lo + cv.rows_per_slab, cv.hw);
    const size_t base = (size_t)img * cv.hw * cv.c + ch;
    auto add = [&](const Vec<T, V>& xv, const Vec<T, V>& dv, const Vec<T, V>& sv) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!BWD) {
          const double d = (double)xv.get(j);
          s0[j] += d;
          s1[j] += d * d;
        } else {
          const float xs = xv.get(j);
          const float g = slope_times<ACT, T, V>(dv.get(j), ACT == ACT_RELU ? sv.get(j) : 0.f, xs, mu[j], is[j], ga[j], be[j],
                                                 ACT == ACT_SILU && side ? sv.get(j) : 0.f);
          s0[j] += (double)g;
          s1[j] += (double)g * (double)((xs - mu[j]) * is[j]);
        }
      }
    };
    int r = lo + lane_r;
    for (; r + (U - 1) * cv.rpi < hi; r += U * cv.rpi) {
      Vec<T, V> xv[U], dv[U], sv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t at = base + (size_t)(r + u * cv.rpi) * cv.c;
        xv[u].load(x + at);
        if (BWD) dv[u].load(dy + at);
        if (BWD && ACT != ACT_NONE && side) sv[u].load(side + at);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) add(xv[u], dv[u], sv[u]);
    }
    for (; r < hi; r += cv.rpi) {
      Vec<T, V> xv, dv, sv;
      const size_t at = base + (size_t)r * cv.c;
      xv.load(x + at);
      if (BWD) dv.load(dy + at);
      if (BWD && ACT != ACT_NONE && side) sv.load(side + at);
      add(xv, dv, sv);
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) { red[0][tid][j] = s0[j]; red[1][tid][j] = s1[j]; }
  __syncthreads();
  if (lane_r == 0 && active) {
    for (int rr = 1; rr < cv.rpi; ++rr)
#pragma unroll
      for (int j = 0; j < V; ++j) { s0[j] += red[0][rr * cv.tpr + lane_c][j]; s1[j] += red[1][rr * cv.tpr + lane_c][j]; }
    double* p = part + ((size_t)img * cv.slabs + slab) * 2 * cv.c + ch;
#pragma unroll
    for (int j = 0; j < V; ++j) { p[j] = s0[j]; p[cv.c + j] = s1[j]; }
  }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// One wave per group of an image.  Forward: mean and 1/std.
__global__ __launch_bounds__(THREADS) void gn_fwd_finish_kernel(const double* __restrict__ part, float* __restrict__ mean, float* __restrict__ istd,
                                                                Cover cv, int all, float eps) {
  const int at = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (at >= all) return;
  const int img = at / cv.groups, g = at - img * cv.groups;
  double s = 0.0, ss = 0.0;
  for (int i = lane; i < cv.per * cv.slabs; i += 64) {
    const int slab = i / cv.per, j = i - slab * cv.per;
    const double* p = part + ((size_t)img * cv.slabs + slab) * 2 * cv.c + g * cv.per + j;
    s += p[0];
    ss += p[cv.c];
  }
  s = wave_sum(s);
  ss = wave_sum(ss);
  if (lane) return;
  const double m = (double)cv.per * cv.hw, mu = s / m;
  double var = ss / m - mu * mu;
  if (var < 0.0) var = 0.0;
  mean[at] = (float)mu;
  istd[at] = (float)(1.0 / sqrt(var + (double)eps));
}

// Backward: per channel of the image the sums of g and g * xhat (chan[image][2][c]), per group A and B (coef[image * groups + g][2]).
__global__ __launch_bounds__(THREADS) void gn_bwd_finish_kernel(const double* __restrict__ part, const float* __restrict__ gamma,
                                                                float* __restrict__ chan, float* __restrict__ coef, Cover cv, int all) {
  const int at = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (at >= all) return;
  const int img = at / cv.groups, g = at - img * cv.groups;
  double a = 0.0, b = 0.0;
  for (int j = lane; j < cv.per; j += 64) {
    const int ch = g * cv.per + j;
    const double* p = part + (size_t)img * cv.slabs * 2 * cv.c + ch;
    double s0 = 0.0, s1 = 0.0;
    for (int k = 0; k < cv.slabs; ++k) { s0 += p[(size_t)k * 2 * cv.c]; s1 += p[(size_t)k * 2 * cv.c + cv.c]; }
    chan[(size_t)img * 2 * cv.c + ch] = (float)s0;
    chan[(size_t)img * 2 * cv.c + cv.c + ch] = (float)s1;
    const double ga = (double)gamma[ch];
    a += ga * s0;
    b += ga * s1;
  }
  a = wave_sum(a);
  b = wave_sum(b);
  if (lane) return;
  const double m = (double)cv.per * cv.hw;
  coef[2 * (size_t)at] = (float)(a / m);
  coef[2 * (size_t)at + 1] = (float)(b / m);
}

// dbeta and dgamma: the images' sums in order, a wave of lanes per channel column
__global__ __launch_bounds__(THREADS) void gn_params_kernel(const float* __restrict__ chan, float* __restrict__ dgamma, float* __restrict__ dbeta, int n,
                                                            int c) {
  __shared__ double red[THREADS];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;      // 8 parts of the images
  double s = 0.0;
  if (col < 2 * c)
    for (int i = part; i < n; i += THREADS / 32) s += (double)chan[(size_t)i * 2 * c + col];
  red[threadIdx.x] = s;
  __syncthreads();
  if (part || col >= 2 * c) return;
#pragma unroll
  for (int k = 1; k < THREADS / 32; ++k) s += red[threadIdx.x + 32 * k];
  if (col < c) dbeta[col] = (float)s; else dgamma[col - c] = (float)s;
}

template <int ACT, class T, int V>
__global__ __launch_bounds__(THREADS) void gn_apply_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                           const T* __restrict__ res, const float* __restrict__ mean, const float* __restrict__ istd,
                                                           T* __restrict__ y, Cover cv) {
  const int tid = threadIdx.x, lane_r = tid / cv.tpr, lane_c = tid - lane_r * cv.tpr;
  const int slice = blockIdx.x % cv.slices, rest = blockIdx.x / cv.slices, slab = rest % cv.slabs, img = rest / cv.slabs;
  const int ch = (slice * cv.tpr + lane_c) * V;
  if (lane_r >= cv.rpi || ch >= cv.c) return;
  float mu[V], is[V], ga[V], be[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const size_t g = (size_t)img * cv.groups + (ch + j) / cv.per;
    mu[j] = mean[g]; is[j] = istd[g]; ga[j] = gamma[ch + j]; be[j] = beta[ch + j];
  }
  const int lo = slab * cv.rows_per_slab, hi = min(lo + cv.rows_per_slab, cv.hw);
  const size_t base = (size_t)img * cv.hw * cv.c + ch;
  for (int r = lo + lane_r; r < hi; r += cv.rpi) {
    const size_t at = base + (size_t)r * cv.c;
    Vec<T, V> xv, rv;
    xv.load(x + at);
    if (res) rv.load(res + at);
    float o[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float z = fmaf((xv.get(j) - mu[j]) * is[j], ga[j], be[j]);
      if (res) z += rv.get(j);
      o[j] = act<ACT>(z);
    }
    xv.set(o);
    xv.store(y + at);
  }
}

template <int ACT, class T, int V>
__global__ __launch_bounds__(THREADS) void gn_bwd_apply_kernel(const T* x, const T* dy, const T* __restrict__ side,
                                                               const float* __restrict__ gamma, const float* __restrict__ beta,
                                                               const float* __restrict__ mean, const float* __restrict__ istd,
                                                               const float* __restrict__ coef, T* dx, T* dres, Cover cv) {
  const int tid = threadIdx.x, lane_r = tid / cv.tpr, lane_c = tid - lane_r * cv.tpr;
  const int slice = blockIdx.x % cv.slices, rest = blockIdx.x / cv.slices, slab = rest % cv.slabs, img = rest / cv.slabs;
  const int ch = (slice * cv.tpr + lane_c) * V;
  if (lane_r >= cv.rpi || ch >= cv.c) return;
  float mu[V], is[V], ga[V], be[V], ca[V], cb[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const size_t g = (size_t)img * cv.groups + (ch + j) / cv.per;
    mu[j] = mean[g]; is[j] = istd[g]; ga[j] = gamma[ch + j]; be[j] = ACT == ACT_SILU ? beta[ch + j] : 0.f;
    ca[j] = coef[2 * g]; cb[j] = coef[2 * g + 1];
  }
  const int lo = slab * cv.rows_per_slab, hi = min(lo + cv.rows_per_slab, cv.hw);
  const size_t base = (size_t)img * cv.hw * cv.c + ch;
  for (int r = lo + lane_r; r < hi; r += cv.rpi) {
    const size_t at = base + (size_t)r * cv.c;
    Vec<T, V> xv, dv, sv;
    xv.load(x + at);
    dv.load(dy + at);
    if (ACT != ACT_NONE && side) sv.load(side + at);
    float o[V], gv[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float xs = xv.get(j), xh = (xs - mu[j]) * is[j];
      gv[j] = slope_times<ACT, T, V>(dv.get(j), ACT == ACT_RELU ? sv.get(j) : 0.f, xs, mu[j], is[j], ga[j], be[j],
                                     ACT == ACT_SILU && side ? sv.get(j) : 0.f);
      o[j] = is[j] * (gv[j] * ga[j] - ca[j] - xh * cb[j]);
    }
    xv.set(o);
    xv.store(dx + at);
    if (dres) {
      xv.set(gv);
      xv.store(dres + at);
    }
  }
}

// `images` x slabs workgroups, about four per compute unit, at least 4 trips of U rows each
Cover cover(int n, int hw, int c, int groups, int v, long target) {
  Cover cv{};
  cv.hw = hw; cv.c = c; cv.groups = groups; cv.per = c / groups;
  const int cols = (c + v - 1) / v;
  cv.slices = (cols + THREADS - 1) / THREADS;
  cv.tpr = (cols + cv.slices - 1) / cv.slices;
  cv.rpi = THREADS / cv.tpr;
  long slabs = (target + (long)n * cv.slices - 1) / ((long)n * cv.slices);
  const long most = ((long)hw + (long)cv.rpi * U - 1) / ((long)cv.rpi * U);
  if (slabs > most) slabs = most;
  if (slabs > kGnMaxSlabs) slabs = kGnMaxSlabs;
  if (slabs < 1) slabs = 1;
  cv.rows_per_slab = (int)((hw + slabs - 1) / slabs);
  cv.slabs = (hw + cv.rows_per_slab - 1) / cv.rows_per_slab;
  return cv;
}
constexpr long kSumGroups = 1024, kApplyGroups = 4096;

struct GnArgs {
  const void *x, *dy, *side;
  const float *gamma, *beta;
  const float *mean_in, *istd_in;
  float *mean, *istd;
  void *out, *dres;
  float *dgamma, *dbeta;
  int n, hw, c, groups;
  float eps;
  void* workspace;
  hipStream_t st;
};

template <int ACT, class T, int V>
void forward_any(const GnArgs& a) {
  const Cover cv = cover(a.n, a.hw, a.c, a.groups, V, kSumGroups), ca = cover(a.n, a.hw, a.c, a.groups, V, kApplyGroups);
  double* part = static_cast<double*>(a.workspace);
  const int all = a.n * a.groups;
  hipLaunchKernelGGL((gn_sums_kernel<0, ACT_NONE, T, V>), dim3((unsigned)(a.n * cv.slabs * cv.slices)), dim3(THREADS), 0, a.st, (const T*)a.x,
                     (const T*)nullptr, (const T*)nullptr, nullptr, nullptr, nullptr, nullptr, part, cv);
  hipLaunchKernelGGL(gn_fwd_finish_kernel, dim3((all + THREADS / 64 - 1) / (THREADS / 64)), dim3(THREADS), 0, a.st, part, a.mean, a.istd, cv, all, a.eps);
  hipLaunchKernelGGL((gn_apply_kernel<ACT, T, V>), dim3((unsigned)(a.n * ca.slabs * ca.slices)), dim3(THREADS), 0, a.st, (const T*)a.x, a.gamma, a.beta,
                     (const T*)a.side, a.mean, a.istd, (T*)a.out, ca);
}

template <int ACT, class T, int V>
void backward_any(const GnArgs& a) {
  const Cover cv = cover(a.n, a.hw, a.c, a.groups, V, kSumGroups), ca = cover(a.n, a.hw, a.c, a.groups, V, kApplyGroups);
  float* chan = static_cast<float*>(a.workspace);
  const int all = a.n * a.groups;
  float* coef = chan + 2 * (size_t)a.n * a.c;
  double* part = reinterpret_cast<double*>(chan + ((2 * (size_t)a.n * a.c + 2 * (size_t)all + 3) & ~(size_t)3));
  hipLaunchKernelGGL((gn_sums_kernel<1, ACT, T, V>), dim3((unsigned)(a.n * cv.slabs * cv.slices)), dim3(THREADS), 0, a.st, (const T*)a.x,
                     (const T*)a.dy, (const T*)a.side, a.gamma, a.beta, a.mean_in, a.istd_in, part, cv);
  hipLaunchKernelGGL(gn_bwd_finish_kernel, dim3((all + THREADS / 64 - 1) / (THREADS / 64)), dim3(THREADS), 0, a.st, part, a.gamma, chan, coef, cv, all);
  hipLaunchKernelGGL((gn_bwd_apply_kernel<ACT, T, V>), dim3((unsigned)(a.n * ca.slabs * ca.slices)), dim3(THREADS), 0, a.st, (const T*)a.x,
                     (const T*)a.dy, (const T*)a.side, a.gamma, a.beta, a.mean_in, a.istd_in, coef, (T*)a.out, (T*)a.dres, ca);
  hipLaunchKernelGGL(gn_params_kernel, dim3((2 * a.c + 31) / 32), dim3(THREADS), 0, a.st, chan, a.dgamma, a.dbeta, a.n, a.c);
}

#define ACC_GN_ACT(F, T, V)                        \
  switch (act) {                                   \
    case ACT_NONE: F<ACT_NONE, T, V>(a); break;    \
    case ACT_RELU: F<ACT_RELU, T, V>(a); break;    \
    default: F<ACT_SILU, T, V>(a); break;          \
  }
#define ACC_GN(F)                                                                                             \
  do {                                                                                                        \
    if (dtype == DT_F32) { if (a.c % 4 == 0) ACC_GN_ACT(F, float, 4) else ACC_GN_ACT(F, float, 1) }            \
    else { if (a.c % 8 == 0) ACC_GN_ACT(F, bf16_t, 8) else ACC_GN_ACT(F, bf16_t, 1) }                          \
  } while (0)

bool shape_ok(int n, int hw, int c, int groups, int act, int dtype) {
  if (n <= 0 || hw <= 0 || c <= 0 || groups <= 0 || c % groups != 0 || act < ACT_NONE || act > ACT_SILU) return false;
  if (dtype != DT_F32 && dtype != DT_BF16) return false;
  // a launch has fewer than 2^32 threads (beyond an image each, the workgroups are at most kApplyGroups), a thread counts its rows in 31 bits
  const long slices = ((long)c + THREADS - 1) / THREADS;
  return (long)n * groups < (1L << 26) && n * slices + kApplyGroups < (1L << 24) && hw < (1 << 30) && c < (1 << 24);
}

}  // namespace

size_t gn_workspace_bytes(int n, int hw, int c, int groups) {
  if (!shape_ok(n, hw, c, groups, ACT_NONE, DT_F32)) return 0;
  // the sums of the backward pass, whichever width a thread has: per image and slab 2 c doubles, per image 2 c floats, two per group
  int slabs = 0;
  for (int v : {1, 4, 8}) {
    const int s = cover(n, hw, c, groups, v, kSumGroups).slabs;
    if (s > slabs) slabs = s;
  }
  return (size_t)n * slabs * 2 * c * sizeof(double) + (((size_t)2 * n * c + (size_t)2 * n * groups + 3) & ~(size_t)3) * sizeof(float);
}

hipError_t gn_forward(const void* x, const float* gamma, const float* beta, const void* res, void* y, float* mean, float* istd, int n, int hw, int c,
                      int groups, int act, float eps, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!x || !gamma || !beta || !y || !mean || !istd || !workspace || !(eps >= 0.f)) return hipErrorInvalidValue;
  if (!shape_ok(n, hw, c, groups, act, dtype) || workspace_bytes < gn_workspace_bytes(n, hw, c, groups)) return hipErrorInvalidValue;
  GnArgs a{};
  a.x = x; a.gamma = gamma; a.beta = beta; a.side = res; a.out = y; a.mean = mean; a.istd = istd;
  a.n = n; a.hw = hw; a.c = c; a.groups = groups; a.eps = eps; a.workspace = workspace; a.st = st;
  ACC_GN(forward_any);
  return hipGetLastError();
}

hipError_t gn_backward(const void* x, const void* dy, const void* y, const void* res, const float* gamma, const float* beta, const float* mean,
                       const float* istd, void* dx, float* dgamma, float* dbeta, void* dres, int n, int hw, int c, int groups, int act, void* workspace,
                       size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!x || !dy || !gamma || !beta || !mean || !istd || !dx || !dgamma || !dbeta || !workspace) return hipErrorInvalidValue;
  if (!shape_ok(n, hw, c, groups, act, dtype) || workspace_bytes < gn_workspace_bytes(n, hw, c, groups)) return hipErrorInvalidValue;
  if (act == ACT_RELU && !y) return hipErrorInvalidValue;
  GnArgs a{};
  a.x = x; a.dy = dy; a.side = act == ACT_RELU ? y : act == ACT_SILU ? res : nullptr; a.gamma = gamma; a.beta = beta; a.mean_in = mean; a.istd_in = istd;
  a.out = dx; a.dgamma = dgamma; a.dbeta = dbeta; a.dres = dres;
  a.n = n; a.hw = hw; a.c = c; a.groups = groups; a.workspace = workspace; a.st = st;
  ACC_GN(backward_any);
  return hipGetLastError();
}

}  // namespace acc
