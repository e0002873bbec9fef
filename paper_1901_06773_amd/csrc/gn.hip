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

// ---------------------------------------------------------------------------------- small images: one read, the values stay in registers
//
// A workgroup takes all rows of a few neighbouring groups of one image, 64 bytes of channels or more, and keeps them: thread t has V channels of the rows
// t / tpr, t / tpr + rpi, ...  Forward: mean, then the squares of the deviations from it, both in fp32 (a thread adds at most R values one behind
// the other, the rest in a tree).  The XCD-wise order of workgroups lets neighbouring slices of a row meet in one L2.
struct Slice {
  int hw, c, groups, per;
  int k, s, slices;                                    // groups and channels of a slice, slices of an image
  int tpr, rpi;
  int all;                                             // slices of all images
};

// sums over a wave; the first lane's order is fixed
__device__ __forceinline__ float wave_sum_f(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Values of the threads, added up per group: val[NV] of a thread belong to NV parts of its channels.  red: NT * NV floats, out: one per group, finish() of the sum.
template <int NT, int NV, class F>
__device__ __forceinline__ void group_sums(const float (&val)[NV], float* red, float* out, const Slice& sl, bool active, F finish) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
#pragma unroll
  for (int j = 0; j < NV; ++j) red[tid * NV + j] = active ? val[j] : 0.f;
  __syncthreads();
  // a row of red: tpr * NV parts, of which each group has `parts` neighbouring ones
  const int width = sl.tpr * NV, parts = width / sl.k, count = parts * sl.rpi;
  for (int g = wave; g < sl.k; g += NT / 64) {
    float t = 0.f;
    for (int i = lane; i < count; i += 64) {
      const int r = i / parts, j = i - r * parts;
      t += red[r * width + g * parts + j];
    }
    t = wave_sum_f(t);
    if (lane == 0) out[g] = finish(t);
  }
  __syncthreads();
}

// V values added up in pairs
template <int V> __device__ __forceinline__ float pairs(float (&v)[V]) {
#pragma unroll
  for (int o = V / 2; o > 0; o >>= 1)
#pragma unroll
    for (int j = 0; j < o; ++j) v[j] += v[j + o];
  return v[0];
}

// Keeps the compiler from working on more than a few rows of many at a time, which would not fit the registers.
__device__ __forceinline__ void fence() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_sched_barrier(0);
#endif
}
// a value that the compiler takes for a new one: what follows from it is worked out again, not kept in registers
__device__ __forceinline__ uint32_t anew(uint32_t v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
  return v;
}
template <int R> __device__ __forceinline__ void pause(int u) {
  if (R > 4 && (u & 1)) fence();
}

constexpr int kMaxSliceGroups = 256;

// PERCH: a thread's channels may belong to several groups
template <class T, int V, int R, int NT, bool PERCH>
__global__ __launch_bounds__(NT) void gn_fwd_slice_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, const T* res,
                                                          float* __restrict__ mean, float* __restrict__ istd, T* y, int act_kind, float eps, Slice sl, int blocks) {
  constexpr int NV = PERCH ? V : 1;
  __shared__ float red[NT * NV];
  __shared__ float mu_sh[kMaxSliceGroups], is_sh[kMaxSliceGroups];
  const int at = (blockIdx.x & 7) * (blocks >> 3) + (blockIdx.x >> 3);
  if (at >= sl.all) return;
  const int img = at / sl.slices, slice = at - img * sl.slices, tid = threadIdx.x, row0 = tid / sl.tpr, col = tid - row0 * sl.tpr;
  const int ch = slice * sl.s + col * V;
  const bool active = row0 < sl.rpi;
  const int rows = active && row0 < sl.hw ? (sl.hw - 1 - row0) / sl.rpi + 1 : 0;       // of this thread
  // (an image is less than 4 GiB: byte offsets of 32 bits beside addresses that the workgroup shares, worked out anew for every pass)
  const size_t base = (size_t)img * sl.hw * sl.c + (size_t)slice * sl.s;
  const uint32_t off0 = rows > 0 ? ((uint32_t)row0 * (uint32_t)sl.c + (uint32_t)(col * V)) * (uint32_t)sizeof(T) : 0u;
  const uint32_t step = (uint32_t)sl.rpi * (uint32_t)sl.c * (uint32_t)sizeof(T);
  const char *const xb = (const char*)(x + base), *const rb = res ? (const char*)(res + base) : nullptr;
  char* const yb = (char*)(y + base);
  Vec<T, V> xv[R];
  uint32_t to = anew(off0);
#pragma unroll
  for (int u = 0; u < R; ++u) {
    xv[u].load((const T*)(xb + (u < rows ? to : 0u)));
    to += step;
  }
  float ga[V], be[V];
#pragma unroll
  for (int j = 0; j < V; ++j) { ga[j] = active ? gamma[ch + j] : 0.f; be[j] = active ? beta[ch + j] : 0.f; }
  const float m = (float)sl.hw * (float)sl.per;
  float val[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) val[j] = 0.f;
  auto add = [&](float (&v)[V]) {
    if constexpr (PERCH) {
#pragma unroll
      for (int j = 0; j < V; ++j) val[j] += v[j];
    } else {
      val[0] += pairs<V>(v);
    }
  };
#pragma unroll
  for (int u = 0; u < R; ++u)
    if (u < rows) {
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = xv[u].get(j);
      add(v);
      pause<R>(u);
    }
  group_sums<NT, NV>(val, red, mu_sh, sl, active, [&](float t) { return t / m; });
  int g[NV];
  float mu[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    g[j] = active ? (col * V + j) / sl.per : 0;
    mu[j] = mu_sh[g[j]];
    val[j] = 0.f;
  }
#pragma unroll
  for (int u = 0; u < R; ++u)
    if (u < rows) {
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = xv[u].get(j) - mu[PERCH ? j : 0];
        v[j] = d * d;
      }
      add(v);
      pause<R>(u);
    }
  group_sums<NT, NV>(val, red, is_sh, sl, active, [&](float t) { return (float)(1.0 / sqrt((double)(t / m) + (double)eps)); });
  for (int i = tid; i < sl.k; i += NT) {
    const size_t to = (size_t)img * sl.groups + slice * sl.k + i;
    mean[to] = mu_sh[i];
    istd[to] = is_sh[i];
  }
  if (!active) return;
  float is[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) is[j] = is_sh[g[j]];
  to = anew(off0);
#pragma unroll
  for (int u = 0; u < R; ++u)
    if (u < rows) {
      Vec<T, V> rv;
      if (res) rv.load((const T*)(rb + to));
      float o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int q = PERCH ? j : 0;
        o[j] = fmaf((xv[u].get(j) - mu[q]) * is[q], ga[j], be[j]);
        if (res) o[j] += rv.get(j);
      }
      if (act_kind == ACT_RELU) {
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = act<ACT_RELU>(o[j]);
      } else if (act_kind == ACT_SILU) {
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = act<ACT_SILU>(o[j]);
      }
      rv.set(o);
      rv.store((T*)(yb + to));
      to += step;
      pause<R>(u);
    }
}

// Backward: x and g in registers (SiLU: x and dy, g worked out twice); per channel the sums of g and g * xhat, left in chan[image][2][c] for
// gn_params_kernel and added up to A and B here.
template <class T, int V, int R, int NT, bool PERCH>
__global__ __launch_bounds__(NT) void gn_bwd_slice_kernel(const T* x, const T* dy, const T* side, const float* __restrict__ gamma,
                                                          const float* __restrict__ beta, const float* __restrict__ mean, const float* __restrict__ istd,
                                                          T* dx, T* dres, float* __restrict__ chan, int act_kind, Slice sl, int blocks) {
  constexpr int NV = PERCH ? V : 1;
  extern __shared__ float dyn[];                       // [rpi][2][s] sums of the threads, then [parts][2 s], then tot[2 s]
  __shared__ float coef[2 * kMaxSliceGroups];
  const int at = (blockIdx.x & 7) * (blocks >> 3) + (blockIdx.x >> 3);
  if (at >= sl.all) return;
  const int img = at / sl.slices, slice = at - img * sl.slices, tid = threadIdx.x, row0 = tid / sl.tpr, col = tid - row0 * sl.tpr;
  const int ch = slice * sl.s + col * V;
  const bool active = row0 < sl.rpi;
  const int rows = active && row0 < sl.hw ? (sl.hw - 1 - row0) / sl.rpi + 1 : 0;
  const size_t base = (size_t)img * sl.hw * sl.c + (size_t)slice * sl.s;
  const uint32_t off0 = rows > 0 ? ((uint32_t)row0 * (uint32_t)sl.c + (uint32_t)(col * V)) * (uint32_t)sizeof(T) : 0u;
  const uint32_t step = (uint32_t)sl.rpi * (uint32_t)sl.c * (uint32_t)sizeof(T);
  const char *const xb = (const char*)(x + base), *const db = (const char*)(dy + base), *const sb = side ? (const char*)(side + base) : nullptr;
  char *const dxb = (char*)(dx + base), *const drb = dres ? (char*)(dres + base) : nullptr;
  Vec<T, V> xv[R], gv[R];
  uint32_t to = anew(off0);
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const uint32_t from = u < rows ? to : 0u;
    xv[u].load((const T*)(xb + from));
    gv[u].load((const T*)(db + from));
    to += step;
  }
  float ga[V], be[V], mu[NV], is[NV];
  int g[NV];
#pragma unroll
  for (int j = 0; j < V; ++j) { ga[j] = active ? gamma[ch + j] : 0.f; be[j] = active && act_kind == ACT_SILU ? beta[ch + j] : 0.f; }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    g[j] = active ? (col * V + j) / sl.per : 0;
    mu[j] = mean[(size_t)img * sl.groups + slice * sl.k + g[j]];
    is[j] = istd[(size_t)img * sl.groups + slice * sl.k + g[j]];
  }
  if (act_kind == ACT_RELU) {
    to = anew(off0);
#pragma unroll
    for (int u = 0; u < R; ++u) {
      Vec<T, V> yv;
      yv.load((const T*)(sb + (u < rows ? to : 0u)));
      to += step;
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = yv.get(j) > 0.f ? gv[u].get(j) : 0.f;
      gv[u].set(v);                                    // (a value or zero: exact)
      if (R > 4 && (u & 3) == 3) fence();
    }
  }
  auto slope = [&](int u, float (&v)[V]) {             // g of one row
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = gv[u].get(j);
    if (act_kind == ACT_SILU) {
      Vec<T, V> rv;
      if (side) rv.load((const T*)(sb + to));
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int q = PERCH ? j : 0;
        float z = fmaf((xv[u].get(j) - mu[q]) * is[q], ga[j], be[j]);
        if (side) z += rv.get(j);
        v[j] *= silu_slope(z);
      }
    }
  };
  float s0[V], s1[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.f;
  to = anew(off0);
#pragma unroll
  for (int u = 0; u < R; ++u)
    if (u < rows) {
      float v[V];
      slope(u, v);
      to += step;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        s0[j] += v[j];
        s1[j] = fmaf(v[j], (xv[u].get(j) - mu[PERCH ? j : 0]) * is[PERCH ? j : 0], s1[j]);
      }
      pause<R>(u);
    }
  const int s2 = 2 * sl.s;
  if (active) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      dyn[row0 * s2 + col * V + j] = s0[j];
      dyn[row0 * s2 + sl.s + col * V + j] = s1[j];
    }
  }
  __syncthreads();
  // columns: `parts` threads each, then one
  const int parts = NT / s2 > 0 ? NT / s2 : 1;
  float* const sub = dyn + sl.rpi * s2;
  for (int i = tid; i < parts * s2; i += NT) {
    const int part = i / s2, cl = i - part * s2;
    float t = 0.f;
    for (int r = part; r < sl.rpi; r += parts) t += dyn[r * s2 + cl];
    sub[i] = t;
  }
  __syncthreads();
  float* const tot = sub + parts * s2;
  for (int i = tid; i < s2; i += NT) {
    float t = 0.f;
    for (int q = 0; q < parts; ++q) t += sub[q * s2 + i];
    tot[i] = t;
    const int which = i >= sl.s, cl = i - which * sl.s;
    chan[(size_t)img * 2 * sl.c + which * sl.c + slice * sl.s + cl] = t;
  }
  __syncthreads();
  const float inv_m = 1.f / ((float)sl.hw * (float)sl.per);
  for (int w = tid >> 6; w < 2 * sl.k; w += NT / 64) {
    const int which = w >= sl.k, gg = w - which * sl.k;
    float t = 0.f;
    for (int j = tid & 63; j < sl.per; j += 64) t += gamma[slice * sl.s + gg * sl.per + j] * tot[which * sl.s + gg * sl.per + j];
    t = wave_sum_f(t);
    if ((tid & 63) == 0) coef[w] = t * inv_m;
  }
  __syncthreads();
  to = anew(off0);
#pragma unroll
  for (int u = 0; u < R; ++u)
    if (u < rows) {
      float v[V], o[V];
      slope(u, v);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int q = PERCH ? j : 0;
        const float xh = (xv[u].get(j) - mu[q]) * is[q];
        o[j] = is[q] * (v[j] * ga[j] - coef[g[q]] - xh * coef[sl.k + g[q]]);
      }
      xv[u].set(o);
      xv[u].store((T*)(dxb + to));
      if (dres) {
        xv[u].set(v);
        xv[u].store((T*)(drb + to));
      }
      to += step;
      pause<R>(u);
    }
}

// The slices of a tensor, if they fit: 64 bytes of channels (a line of memory is then read by two workgroups at most) or as many groups as it takes for
// whole threads; 32 where 64 do not fit.  Threads and rows of a workgroup: the fewest threads whose registers hold a slice.
struct SliceCfg {
  Slice sl;
  int nt, r;                                           // 0: does not fit
};
// rows of a thread of 1024 that fit 128 registers beside what else it needs
constexpr int slice_rows(int v, bool perch, bool backward) { return !backward ? 20 : v == 4 ? (perch ? 8 : 10) : (perch ? 6 : 8); }
SliceCfg slice_cfg(int n, int hw, int c, int groups, int v, int es, bool backward) {
  SliceCfg f{};
  const int per = c / groups;
  if ((long)hw * c * es >= 1L << 32) return f;
  auto fits = [&](int k) {
    const int tpr = k * per / v;
    if (tpr > 256) return false;
    auto rows = [&](int nt) { return (int)(((long)hw + nt / tpr - 1) / (nt / tpr)); };
    const int nt = rows(256) <= (backward ? 4 : 8) ? 256 : rows(512) <= (backward ? 8 : 16) ? 512 : rows(1024) <= slice_rows(v, per % v != 0, backward) ? 1024 : 0;
    if (!nt || (long)n * (groups / k) * nt >= (1L << 32) - 8192) return false;         // (a launch has fewer than 2^32 threads)
    f.nt = nt;
    f.r = rows(nt);
    f.sl = Slice{hw, c, groups, per, k, k * per, groups / k, tpr, nt / tpr, n * (groups / k)};
    return true;
  };
  int narrow = 0;                                      // the widest slice of 32 bytes or more that is narrower than 64
  for (int k = 1; k <= groups && k <= kMaxSliceGroups; ++k) {
    if (groups % k != 0 || (long)k * per % v != 0) continue;
    const long bytes = (long)k * per * es;
    if (bytes < 64 && k < groups) {
      if (bytes >= 32) narrow = k;
      continue;
    }
    if (!fits(k) && narrow) fits(narrow);
    return f;
  }
  return f;
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

template <class T, int V, int R, int NT, bool PERCH>
void launch_fwd_slice(const GnArgs& a, const Slice& sl, int act) {
  const int blocks = (sl.all + 7) / 8 * 8;
  hipLaunchKernelGGL((gn_fwd_slice_kernel<T, V, R, NT, PERCH>), dim3(blocks), dim3(NT), 0, a.st, (const T*)a.x, a.gamma, a.beta, (const T*)a.side, a.mean,
                     a.istd, (T*)a.out, act, a.eps, sl, blocks);
}
template <class T, int V, int R, int NT, bool PERCH>
void launch_bwd_slice(const GnArgs& a, const Slice& sl, int act) {
  const int blocks = (sl.all + 7) / 8 * 8, s2 = 2 * sl.s, parts = NT / s2 > 0 ? NT / s2 : 1;
  const size_t lds = ((size_t)sl.rpi * s2 + (size_t)parts * s2 + s2) * sizeof(float);
  float* chan = static_cast<float*>(a.workspace);
  hipLaunchKernelGGL((gn_bwd_slice_kernel<T, V, R, NT, PERCH>), dim3(blocks), dim3(NT), lds, a.st, (const T*)a.x, (const T*)a.dy, (const T*)a.side, a.gamma,
                     a.beta, a.mean_in, a.istd_in, (T*)a.out, (T*)a.dres, chan, act, sl, blocks);
  hipLaunchKernelGGL(gn_params_kernel, dim3((2 * a.c + 31) / 32), dim3(THREADS), 0, a.st, chan, a.dgamma, a.dbeta, a.n, a.c);
}
template <class T, int V, bool PERCH>
bool forward_slices(const GnArgs& a, int act) {
  const SliceCfg f = slice_cfg(a.n, a.hw, a.c, a.groups, V, (int)sizeof(T), false);
  if (!f.nt) return false;
#define ACC_CASE(NT, ROWS) if (constexpr int R = ROWS; f.nt == NT && f.r <= R) { launch_fwd_slice<T, V, R, NT, PERCH>(a, f.sl, act); return true; }
  ACC_CASE(256, 1) ACC_CASE(256, 2) ACC_CASE(256, 4) ACC_CASE(256, 8) ACC_CASE(512, 8) ACC_CASE(512, 16) ACC_CASE(1024, 16) ACC_CASE(1024, slice_rows(V, PERCH, false))
#undef ACC_CASE
  return false;
}
template <class T, int V, bool PERCH>
bool backward_slices(const GnArgs& a, int act) {
  const SliceCfg f = slice_cfg(a.n, a.hw, a.c, a.groups, V, (int)sizeof(T), true);
  if (!f.nt) return false;
#define ACC_CASE(NT, ROWS) if (constexpr int R = ROWS; f.nt == NT && f.r <= R) { launch_bwd_slice<T, V, R, NT, PERCH>(a, f.sl, act); return true; }
  ACC_CASE(256, 1) ACC_CASE(256, 2) ACC_CASE(256, 4) ACC_CASE(512, 4) ACC_CASE(512, 8) ACC_CASE(1024, slice_rows(V, PERCH, true))
#undef ACC_CASE
  return false;
}
template <class T, int V>
bool slices(const GnArgs& a, int act, bool backward) {
  const bool perch = (a.c / a.groups) % V != 0;
  if (backward) return perch ? backward_slices<T, V, true>(a, act) : backward_slices<T, V, false>(a, act);
  return perch ? forward_slices<T, V, true>(a, act) : forward_slices<T, V, false>(a, act);
}
// whether the tensor's slices fit a workgroup, which then has been launched
bool by_slices(const GnArgs& a, int act, int dtype, bool backward) {
  if (dtype == DT_F32) return a.c % 4 == 0 && slices<float, 4>(a, act, backward);
  return a.c % 8 == 0 && slices<bf16_t, 8>(a, act, backward);
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
  if (by_slices(a, act, dtype, false)) return hipGetLastError();
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
  if (by_slices(a, act, dtype, true)) return hipGetLastError();
  ACC_GN(backward_any);
  return hipGetLastError();
}

}  // namespace acc
