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
#include "gn_shape.h"

namespace acc {
namespace {

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2 };

// V neighbouring values: sixteen bytes, eight, or one at a time where rows do not start on such an address.
template <class T, int V> struct Vec;
template <class T> struct Vec<T, 1> {
  T raw;
  __device__ __forceinline__ void load(const T* p) { raw = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = raw; }
  __device__ __forceinline__ void store_past(T* p) const { *p = raw; }
  __device__ __forceinline__ float get(int) const { return Elem<T>::load(&raw); }
  __device__ __forceinline__ void set(const float (&v)[1]) { Elem<T>::store(&raw, v[0]); }
};
template <> struct Vec<float, 4> {
  float4 raw;
  __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = raw; }
  __device__ __forceinline__ void store_past(float* p) const {        // past the caches
    typedef float words __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(words{raw.x, raw.y, raw.z, raw.w}, reinterpret_cast<words*>(p));
  }
  __device__ __forceinline__ float get(int i) const { return i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w; }
  __device__ __forceinline__ void set(const float (&v)[4]) { raw = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<bf16_t, 8> {
  uint4 raw;
  __device__ __forceinline__ void load(const bf16_t* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<uint4*>(p) = raw; }
  __device__ __forceinline__ void store_past(bf16_t* p) const {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(words{raw.x, raw.y, raw.z, raw.w}, reinterpret_cast<words*>(p));
  }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? raw.x : i < 4 ? raw.y : i < 6 ? raw.z : raw.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    raw = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
};

// 1 / (1 + e^-z) by the base-two exponential and the reciprocal of the hardware, a rounding or two each; the rounding of z * log2 e makes e^-z wrong by
// |z| / 1.4 of them more, which is little beside 1 where z is positive and where z is negative leaves a value of at most 1 / 4 of z's size (an exact expf
// and a division took the kernels from memory to arithmetic: 8 images of 56x56, 64 channels, bf16 forward 39 us)
__device__ __forceinline__ float sigmoid(float z) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
#else
  return z;
#endif
}
template <int ACT> __device__ __forceinline__ float act(float z) {
  if (ACT == ACT_RELU) return z < 0.f ? 0.f : z;       // (a value that is no number stays none)
  if (ACT == ACT_SILU) return z * sigmoid(z);
  return z;
}
__device__ __forceinline__ float silu_slope(float z) {
  const float s = sigmoid(z);
  return s * (1.f + z * (1.f - s));
}

// V neighbouring fp32 parameters
template <int V> __device__ __forceinline__ void load_params(const float* p, float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      const float4 q = *reinterpret_cast<const float4*>(p + j);
      v[j] = q.x; v[j + 1] = q.y; v[j + 2] = q.z; v[j + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = p[j];
  }
}

// ---------------------------------------------------------------------------------- any size: sums, then apply
//
// The rows of an image are cut into slabs, its channels into slices of whole groups (or a group into several slices, where it is wider than a workgroup).
// A workgroup adds up one slab of one slice, per channel and then per group, and leaves one pair of sums per group; every workgroup of the second
// launch joins the slabs of its own groups, while its first rows are on their way, and works on its rows.  A thread adds a few rows in fp32 and these
// in fp64.
constexpr int THREADS = 256;
template <int BWD, int V> struct Rows { static constexpr int U = BWD && V == 8 ? 2 : 4; };      // rows of a thread on their way, twice

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

struct Cover {
  int hw, c, groups, per;
  int slices, width;                                   // slices of a row, channels of a slice (the last of a row or group may have fewer)
  int k, s;                                            // groups of a slice, slices of a group: one of them is 1
  int tpr, rpi;                                        // threads across a slice, rows per trip
  int slabs, rows_per_slab;                            // of the sums
  int cuts, rows_per_cut;                              // of the second launch
  int past;                                            // results are written past the caches
  // first channel of a slice, and the end of its channels
  __host__ __device__ int first(int slice) const { return s > 1 ? slice / s * per + slice % s * width : slice * width; }
  __host__ __device__ int end(int slice) const {
    const int all = s > 1 ? (slice / s + 1) * per : c, e = first(slice) + width;
    return e < all ? e : all;
  }
  // pairs of sums per image and slab: one per group, or one per slice
  __host__ __device__ int slots() const { return s > 1 ? slices : groups; }
};

template <int ACT, class T, int V>
__device__ __forceinline__ float slope_times(float dy, float y, float x, float mu, float istd, float ga, float be, float res) {
  if (ACT == ACT_RELU) return y > 0.f ? dy : 0.f;
  if (ACT == ACT_SILU) return dy * silu_slope(fmaf((x - mu) * istd, ga, be) + res);
  return dy;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// BWD 0: sums of x and x * x, taken from x - p and its square with p the slab's first row (fp32 sums of these lose nothing to a mean that is far from
// zero); pairs[image][slab][slot][2].  BWD 1: of g and g * xhat, per channel chan[image][slab][2][c], per group with gamma as a factor in pairs.
// side: the stored output (ReLU) or the residual (SiLU; may be null).  Memory, and in small tensors one trip to it behind another: bf16, 13 images of 51x51, 120
// channels 7.7 us (8.1 MB), backward fp32, 19 images of 55x55, 128 channels 14 us (58.8 MB, 4.2 TB/s).
template <int BWD, int ACT, class T, int V>
__global__ __launch_bounds__(THREADS) void gn_sums_kernel(const T* __restrict__ x, const T* __restrict__ dy, const T* __restrict__ side,
                                                          const float* __restrict__ gamma, const float* __restrict__ beta,
                                                          const float* __restrict__ mean, const float* __restrict__ istd,
                                                          double* __restrict__ pairs, float* __restrict__ chan, Cover cv) {
  constexpr int U = Rows<BWD, V>::U;
  __shared__ double red[2][THREADS * V];
  const int tid = threadIdx.x, lane_r = tid / cv.tpr, lane_c = tid - lane_r * cv.tpr;
  const int slice = blockIdx.x % cv.slices, rest = blockIdx.x / cv.slices, slab = rest % cv.slabs, img = rest / cv.slabs;
  const int ch0 = cv.first(slice), ch1 = cv.end(slice), ch = ch0 + lane_c * V;
  const bool active = lane_r < cv.rpi && ch < ch1;
  const int lo = slab * cv.rows_per_slab, hi = min(lo + cv.rows_per_slab, cv.hw);
  double s0[V], s1[V];
  float p[V], mu[V], is[V], ga[V], be[V];
#pragma unroll
  for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.0;
  if (active) {
    const size_t base = (size_t)img * cv.hw * cv.c + ch;
    if (BWD) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int g = (ch + j) / cv.per;
        mu[j] = mean[(size_t)img * cv.groups + g];
        is[j] = istd[(size_t)img * cv.groups + g];
        ga[j] = ACT == ACT_SILU ? gamma[ch + j] : 0.f;
        be[j] = ACT == ACT_SILU ? beta[ch + j] : 0.f;
      }
    } else {
      Vec<T, V> first;
      first.load(x + base + (size_t)lo * cv.c);
#pragma unroll
      for (int j = 0; j < V; ++j) p[j] = first.get(j);
    }
    float t0[V], t1[V];
    auto add = [&](const Vec<T, V>& xv, const Vec<T, V>& dv, const Vec<T, V>& sv) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!BWD) {
          const float d = xv.get(j) - p[j];
          t0[j] += d;
          t1[j] = fmaf(d, d, t1[j]);
        } else {
          const float xs = xv.get(j);
          const float g = slope_times<ACT, T, V>(dv.get(j), ACT == ACT_RELU ? sv.get(j) : 0.f, xs, mu[j], is[j], ga[j], be[j],
                                                 ACT == ACT_SILU && side ? sv.get(j) : 0.f);
          t0[j] += g;
          t1[j] = fmaf(g, (xs - mu[j]) * is[j], t1[j]);
        }
      }
    };
    // the next rows are asked for before these are added
    Vec<T, V> xv[2][U], dv[2][U], sv[2][U];
    auto load = [&](int r, int to) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ru = r + u * cv.rpi;
        const size_t at = base + (size_t)(ru < hi ? ru : lo) * cv.c;      // (a row that does not exist: read, not added)
        xv[to][u].load(x + at);
        if (BWD) dv[to][u].load(dy + at);
        if (BWD && ACT != ACT_NONE && side) sv[to][u].load(side + at);
      }
    };
    auto sum = [&](int r, int from) {
#pragma unroll
      for (int j = 0; j < V; ++j) t0[j] = t1[j] = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * cv.rpi < hi) add(xv[from][u], dv[from][u], sv[from][u]);
#pragma unroll
      for (int j = 0; j < V; ++j) { s0[j] += (double)t0[j]; s1[j] += (double)t1[j]; }
    };
    const int trip = U * cv.rpi;
    int r = lo + lane_r;
    load(r, 0);
    for (; r < hi; r += 2 * trip) {
      load(r + trip, 1);
      sum(r, 0);
      load(r + 2 * trip, 0);
      sum(r + trip, 1);
    }
  }
  // the rows of threads, in order: values j of neighbouring threads side by side (no bank twice), a thread per channel
  const int wide = cv.tpr * V;
  if (lane_r < cv.rpi) {
#pragma unroll
    for (int j = 0; j < V; ++j) { red[0][lane_r * wide + j * cv.tpr + lane_c] = s0[j]; red[1][lane_r * wide + j * cv.tpr + lane_c] = s1[j]; }
  }
  __syncthreads();
  const double rows = (double)(hi - lo);
  double c0[V], c1[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int at = tid + i * THREADS, j = at / cv.tpr, chn = ch0 + (at - j * cv.tpr) * V + j;
    c0[i] = c1[i] = 0.0;
    if (at >= wide || chn >= ch1) continue;
    for (int rr = 0; rr < cv.rpi; ++rr) { c0[i] += red[0][rr * wide + at]; c1[i] += red[1][rr * wide + at]; }
    if (BWD) {
      const size_t to = ((size_t)img * cv.slabs + slab) * 2 * cv.c + chn;
      chan[to] = (float)c0[i];
      chan[to + cv.c] = (float)c1[i];
      const double f = (double)gamma[chn];
      c0[i] *= f;
      c1[i] *= f;
    } else {
      const double q = (double)Elem<T>::load(x + ((size_t)img * cv.hw + lo) * cv.c + chn);
      c1[i] += q * (2.0 * c0[i] + rows * q);
      c0[i] += rows * q;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int at = tid + i * THREADS, j = at / cv.tpr;
    if (at < wide) { red[0][(at - j * cv.tpr) * V + j] = c0[i]; red[1][(at - j * cv.tpr) * V + j] = c1[i]; }
  }
  __syncthreads();
  // the channels of a group: a thread each where they are few, else a wave
  const int per = cv.s > 1 ? ch1 - ch0 : cv.per, count = cv.s > 1 ? 1 : (ch1 - ch0) / cv.per, slot0 = cv.s > 1 ? slice : slice * cv.k;
  double* const out = pairs + (((size_t)img * cv.slabs + slab) * cv.slots() + slot0) * 2;
  if (per <= 8) {
    for (int i = tid; i < 2 * count; i += THREADS) {
      double t = 0.0;
      for (int j = 0; j < per; ++j) t += red[i & 1][(i >> 1) * per + j];
      out[i] = t;
    }
  } else {
    for (int i = tid >> 6; i < 2 * count; i += THREADS / 64) {
      double t = 0.0;
      for (int j = tid & 63; j < per; j += 64) t += red[i & 1][(i >> 1) * per + j];
      t = wave_sum(t);
      if ((tid & 63) == 0) out[i] = t;
    }
  }
}

// The slabs of a workgroup's groups joined: out[group of the slice][2] in LDS.  Groups side by side along the threads, 2^q threads each.
constexpr int kMaxCoverGroups = 256;
__device__ __forceinline__ void join_pairs(const double* __restrict__ pairs, int img, int slice, const Cover& cv, double (*out)[2]) {
  const int tid = threadIdx.x, count = cv.s > 1 ? 1 : (cv.end(slice) - cv.first(slice)) / cv.per;
  const int entries = cv.slabs * cv.s;                 // of a group
  int q = 1;
  while (q < 64 && q < entries && 2 * q * count <= THREADS) q *= 2;
  const int slot0 = cv.s > 1 ? slice / cv.s * cv.s : slice * cv.k;
  const double* const base = pairs + (size_t)img * cv.slabs * cv.slots() * 2;
  for (int g = tid / q; g < (count + THREADS / q - 1) / (THREADS / q) * (THREADS / q); g += THREADS / q) {
    double a = 0.0, b = 0.0;
    if (g < count) {
#pragma unroll 4
      for (int i = tid % q; i < entries; i += q) {
        const int slab = i / cv.s, sub = i - slab * cv.s;
        const double2 v = *reinterpret_cast<const double2*>(base + ((size_t)slab * cv.slots() + slot0 + (cv.s > 1 ? sub : g)) * 2);
        a += v.x;
        b += v.y;
      }
    }
    for (int o = 1; o < q; o <<= 1) { a += __shfl_xor(a, o); b += __shfl_xor(b, o); }
    if (g < count && tid % q == 0) { out[g][0] = a; out[g][1] = b; }
  }
  __syncthreads();
}

// dbeta and dgamma: `rows` rows of 2 c sums added up in order, 32 columns of a workgroup
__device__ __forceinline__ void sum_params(const float* __restrict__ chan, float* __restrict__ dgamma, float* __restrict__ dbeta, long rows, int c, int block,
                                           double* red) {
  const int col = block * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;      // 8 parts of the rows
  double s = 0.0;
  if (col < 2 * c) {
#pragma unroll 4
    for (long i = part; i < rows; i += THREADS / 32) s += (double)chan[(size_t)i * 2 * c + col];
  }
  red[threadIdx.x] = s;
  __syncthreads();
  if (part || col >= 2 * c) return;
#pragma unroll
  for (int k = 1; k < THREADS / 32; ++k) s += red[threadIdx.x + 32 * k];
  if (col < c) dbeta[col] = (float)s; else dgamma[col - c] = (float)s;
}
__global__ __launch_bounds__(THREADS) void gn_params_kernel(const float* __restrict__ chan, float* __restrict__ dgamma, float* __restrict__ dbeta, int n, int c) {
  __shared__ double red[THREADS];
  sum_params(chan, dgamma, dbeta, n, c, blockIdx.x, red);
}

// The second launch.  Rows of a workgroup so that there are some workgroups per compute unit; 13 images of 51x51, 120 channels, bf16, residual 8.6 us (24 MB, of
// which x comes from the caches), backward below, fp32, 19 images of 55x55, 128 channels 23 us (88 MB, 3.8 TB/s).
template <int ACT, class T, int V>
__global__ __launch_bounds__(THREADS) void gn_apply_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, const T* res,
                                                           const double* __restrict__ pairs, float* __restrict__ mean, float* __restrict__ istd, T* y, float eps,
                                                           Cover cv) {
  __shared__ double sums[kMaxCoverGroups][2];
  const int tid = threadIdx.x, lane_r = tid / cv.tpr, lane_c = tid - lane_r * cv.tpr;
  const int slice = blockIdx.x % cv.slices, rest = blockIdx.x / cv.slices, cut = rest % cv.cuts, img = rest / cv.cuts;
  const int ch0 = cv.first(slice), ch1 = cv.end(slice), ch = ch0 + lane_c * V;
  const bool active = lane_r < cv.rpi && ch < ch1;
  const int lo = cut * cv.rows_per_cut, hi = min(lo + cv.rows_per_cut, cv.hw);
  const size_t base = (size_t)img * cv.hw * cv.c + ch;
  int r = lo + lane_r;
  Vec<T, V> xv[2], rv[2];
  auto load = [&](int row) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int ru = row + u * cv.rpi;
      const size_t at = base + (size_t)(ru < hi ? ru : row) * cv.c;
      xv[u].load(x + at);
      if (res) rv[u].load(res + at);
    }
  };
  if (active && r < hi) load(r);                       // on their way beside the sums
  join_pairs(pairs, img, slice, cv, sums);
  const double m = (double)cv.per * cv.hw;
  const int count = cv.s > 1 ? 1 : (ch1 - ch0) / cv.per, g0 = ch0 / cv.per;
  for (int g = tid; g < count; g += THREADS) {
    const double mu = sums[g][0] / m;
    double var = sums[g][1] / m - mu * mu;
    if (var < 0.0) var = 0.0;
    const double is = 1.0 / sqrt(var + (double)eps);
    float* const put = reinterpret_cast<float*>(&sums[g][0]);
    put[0] = (float)mu;
    put[1] = (float)is;
    if (cut == 0 && (cv.s == 1 || slice % cv.s == 0)) {
      mean[(size_t)img * cv.groups + g0 + g] = (float)mu;
      istd[(size_t)img * cv.groups + g0 + g] = (float)is;
    }
  }
  __syncthreads();
  if (!active) return;
  float mu[V], is[V], ga[V], be[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float* const got = reinterpret_cast<const float*>(&sums[(ch + j) / cv.per - g0][0]);
    mu[j] = got[0]; is[j] = got[1];
  }
  load_params<V>(gamma + ch, ga);
  load_params<V>(beta + ch, be);
  auto all_rows = [&](auto past) {
    for (; r < hi; r += 2 * cv.rpi) {
      if (r != lo + lane_r) load(r);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (r + u * cv.rpi >= hi) continue;
        float o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float z = fmaf((xv[u].get(j) - mu[j]) * is[j], ga[j], be[j]);
          if (res) z += rv[u].get(j);
          o[j] = act<ACT>(z);
        }
        Vec<T, V> out;
        out.set(o);
        T* const to = y + base + (size_t)(r + u * cv.rpi) * cv.c;
        if constexpr (decltype(past)::value) out.store_past(to); else out.store(to);
      }
    }
  };
  if (cv.past) all_rows(Yes()); else all_rows(No());      // (two loops: one with a choice of stores would lose their kind)
}

// The workgroups from `blocks` on add up dgamma and dbeta.
template <int ACT, class T, int V>
__global__ __launch_bounds__(THREADS) void gn_bwd_apply_kernel(const T* x, const T* dy, const T* side, const float* __restrict__ gamma,
                                                               const float* __restrict__ beta, const float* __restrict__ mean, const float* __restrict__ istd,
                                                               const double* __restrict__ pairs, const float* __restrict__ chan, T* dx, T* dres,
                                                               float* __restrict__ dgamma, float* __restrict__ dbeta, long chan_rows, int blocks, Cover cv) {
  __shared__ double sums[kMaxCoverGroups][2];
  if ((int)blockIdx.x >= blocks) {
    sum_params(chan, dgamma, dbeta, chan_rows, cv.c, (int)blockIdx.x - blocks, &sums[0][0]);
    return;
  }
  const int tid = threadIdx.x, lane_r = tid / cv.tpr, lane_c = tid - lane_r * cv.tpr;
  const int slice = blockIdx.x % cv.slices, rest = blockIdx.x / cv.slices, cut = rest % cv.cuts, img = rest / cv.cuts;
  const int ch0 = cv.first(slice), ch1 = cv.end(slice), ch = ch0 + lane_c * V;
  const bool active = lane_r < cv.rpi && ch < ch1;
  const int lo = cut * cv.rows_per_cut, hi = min(lo + cv.rows_per_cut, cv.hw);
  const size_t base = (size_t)img * cv.hw * cv.c + ch;
  int r = lo + lane_r;
  Vec<T, V> xv, dv, sv;
  auto load = [&](int row) {
    const size_t at = base + (size_t)row * cv.c;
    xv.load(x + at);
    dv.load(dy + at);
    if (ACT != ACT_NONE && side) sv.load(side + at);
  };
  if (active && r < hi) load(r);
  join_pairs(pairs, img, slice, cv, sums);
  if (!active) return;
  const int g0 = ch0 / cv.per;
  const double m = (double)cv.per * cv.hw;
  float mu[V], is[V], ga[V], be[V], ca[V], cb[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int g = (ch + j) / cv.per;
    mu[j] = mean[(size_t)img * cv.groups + g]; is[j] = istd[(size_t)img * cv.groups + g];
    ca[j] = (float)(sums[g - g0][0] / m); cb[j] = (float)(sums[g - g0][1] / m);
  }
  load_params<V>(gamma + ch, ga);
  load_params<V>(beta + ch, be);
  auto all_rows = [&](auto past) {
    for (; r < hi; r += cv.rpi) {
      if (r != lo + lane_r) load(r);
      const size_t at = base + (size_t)r * cv.c;
      float o[V], gv[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float xs = xv.get(j), xh = (xs - mu[j]) * is[j];
        gv[j] = slope_times<ACT, T, V>(dv.get(j), ACT == ACT_RELU ? sv.get(j) : 0.f, xs, mu[j], is[j], ga[j], be[j],
                                       ACT == ACT_SILU && side ? sv.get(j) : 0.f);
        o[j] = is[j] * (gv[j] * ga[j] - ca[j] - xh * cb[j]);
      }
      Vec<T, V> out;
      out.set(o);
      if constexpr (decltype(past)::value) out.store_past(dx + at); else out.store(dx + at);
      if (dres) {
        out.set(gv);
        if constexpr (decltype(past)::value) out.store_past(dres + at); else out.store(dres + at);
      }
    }
  };
  if (cv.past) all_rows(Yes()); else all_rows(No());
}

// ---------------------------------------------------------------------------------- small images: one read, the values stay in registers
//
// A workgroup takes all rows of a few neighbouring groups of one image, 64 bytes of channels or more, and keeps them: thread t has V channels of the rows
// t / tpr, t / tpr + rpi, ...  Forward: mean, then the squares of the deviations from it, both in fp32 (a thread adds at most R values one behind
// the other, the rest in a tree).  The XCD-wise order of workgroups lets neighbouring slices of a row meet in one L2.
// The sum over a wave, in every lane, in a fixed order: neighbouring lanes first, by moves that stay in registers (a butterfly through LDS is six
// trips one after the other).
__device__ __forceinline__ float wave_sum_f(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
#define ACC_DPP(ctrl, rows) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, true))
  v += ACC_DPP(0x111, 0xf);                            // lanes 1, 2, 4, 8 to the left within a row of sixteen
  v += ACC_DPP(0x112, 0xf);
  v += ACC_DPP(0x114, 0xf);
  v += ACC_DPP(0x118, 0xf);
  v += ACC_DPP(0x142, 0xa);                            // the row's last lane to the next row
  v += ACC_DPP(0x143, 0xc);                            // lane 31 to the upper half
#undef ACC_DPP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
#else
  return v;
#endif
}
// Values of the threads, added up per group: val[NV] of a thread belong to NV parts of its channels; `to`: where they go in red, whose
// entries of a group lie side by side (count of them).  out: one per group, finish() of the sum.
template <int NT, int NV, class F>
__device__ __forceinline__ void group_sums(const float (&val)[NV], const int (&to)[NV], float* red, float* out, int groups, int count, F finish) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (to[j] >= 0) red[to[j]] = val[j];
  __syncthreads();
  for (int g = wave; g < groups; g += NT / 64) {
    float t = 0.f;
    int i = lane;
    for (; i + 192 < count; i += 256) t += (red[g * count + i] + red[g * count + i + 64]) + (red[g * count + i + 128] + red[g * count + i + 192]);
    for (; i < count; i += 64) t += red[g * count + i];
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

// One pass over the data: a slice's rows stay in registers between the sums and the results.  Bound by memory: 64 images of 56x56, 256 channels, bf16 42 us for
// 206 MB (4.9 TB/s; every value is fetched once and written once), where the two launches take 56.
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
  const int rows = active ? sl.trips + (row0 < sl.rest ? 1 : 0) : 0;      // of this thread
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
  load_params<V>(gamma + (active ? ch : 0), ga);
  load_params<V>(beta + (active ? ch : 0), be);
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
  // a row of threads has tpr * NV parts, a group `parts` neighbouring ones
  const int parts = sl.tpr * NV / sl.k, count = parts * sl.rpi;
  int g[NV], to_red[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    g[j] = active ? (col * NV + j) / parts : 0;
    to_red[j] = active ? g[j] * count + row0 * parts + (col * NV + j - g[j] * parts) : -1;
  }
  group_sums<NT, NV>(val, to_red, red, mu_sh, sl.k, count, [&](float t) { return t / m; });
  float mu[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
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
  group_sums<NT, NV>(val, to_red, red, is_sh, sl.k, count, [&](float t) { return (float)(1.0 / sqrt((double)(t / m) + (double)eps)); });
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
// gn_params_kernel and added up to A and B here.  64 images of 28x28, 512 channels, bf16, ReLU, residual: 46 us for 257 MB where the memory-side cache still
// holds some of it, 65 where not; x, dy and y are fetched once.
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
  const int rows = active ? sl.trips + (row0 < sl.rest ? 1 : 0) : 0;
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
  load_params<V>(gamma + (active ? ch : 0), ga);
  load_params<V>(beta + (active ? ch : 0), be);
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

// How the two launches cover a tensor, V channels per thread; false: a row has no slices of whole threads (then one value at a time does).
constexpr long kSumGroups = 1024, kApplyGroups = 2048;   // workgroups, about
bool cover(int n, int hw, int c, int groups, int v, Cover* out) {
  Cover cv{};
  cv.hw = hw; cv.c = c; cv.groups = groups; cv.per = c / groups;
  if (c % v) return false;
  const int most = THREADS * v;
  if (cv.per > most) {                                 // a group is several slices
    if (cv.per % v) return false;
    cv.k = 1;
    cv.s = (cv.per + most - 1) / most;
    cv.width = ((cv.per + cv.s - 1) / cv.s + v - 1) / v * v;
    cv.slices = groups * cv.s;
  } else {
    int step = 1;                                      // groups that are whole threads
    while (step * cv.per % v) ++step;
    if (step * cv.per > most) return false;
    int fit = most / (step * cv.per) * step;
    if (fit > kMaxCoverGroups) fit = kMaxCoverGroups;  // (a multiple of step, which divides v)
    cv.s = 1;
    cv.slices = (groups + fit - 1) / fit;
    cv.k = ((groups + cv.slices - 1) / cv.slices + step - 1) / step * step;
    cv.slices = (groups + cv.k - 1) / cv.k;
    cv.width = cv.k * cv.per;
  }
  cv.tpr = cv.width / v;
  cv.rpi = THREADS / cv.tpr;
  auto parts = [&](long target, int trips, long limit, int* count, int* rows) {
    long p = (target + (long)n * cv.slices - 1) / ((long)n * cv.slices);
    const long enough = ((long)hw + (long)cv.rpi * trips - 1) / ((long)cv.rpi * trips);
    if (p > enough) p = enough;
    if (p > limit) p = limit;
    if (p < 1) p = 1;
    *rows = (int)((hw + p - 1) / p);
    *count = (hw + *rows - 1) / *rows;
  };
  // (every workgroup of the second launch joins an image's slabs: more than 64 only where they are large)
  const long mib = ((long)hw * c) >> 18;
  parts(kSumGroups, 4, mib < 64 ? 64 : mib < kGnMaxSlabs ? mib : kGnMaxSlabs, &cv.slabs, &cv.rows_per_slab);
  parts(kApplyGroups, 4, 1L << 30, &cv.cuts, &cv.rows_per_cut);
  // what the second launch writes would drive out of the caches what it reads for the second time (64 channels, 32 images of 112x112 fp32, 103 MB:
  // forward 65 -> 53 us, backward 151 -> 127; bf16 32.6 -> 31.4 and 77 -> 72)
  cv.past = (long)n * hw * c >= 16L << 20;
  *out = cv;
  return true;
}
// four or eight values per thread where rows allow it
int cover_for(int n, int hw, int c, int groups, int dtype, Cover* cv) {
  const int v = dtype == DT_F32 ? 4 : 8;
  if (cover(n, hw, c, groups, v, cv)) return v;
  cover(n, hw, c, groups, 1, cv);
  return 1;
}
// sums of the slabs, per group (fp64) and, backward, per channel (fp32)
size_t pair_bytes(int n, const Cover& cv) { return (size_t)n * cv.slabs * cv.slots() * 2 * sizeof(double); }
size_t chan_bytes(int n, const Cover& cv) { return (size_t)n * cv.slabs * 2 * cv.c * sizeof(float); }

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
void forward_any(const GnArgs& a, const Cover& cv) {
  double* pairs = static_cast<double*>(a.workspace);
  hipLaunchKernelGGL((gn_sums_kernel<0, ACT_NONE, T, V>), dim3((unsigned)((long)a.n * cv.slabs * cv.slices)), dim3(THREADS), 0, a.st, (const T*)a.x,
                     (const T*)nullptr, (const T*)nullptr, nullptr, nullptr, nullptr, nullptr, pairs, nullptr, cv);
  hipLaunchKernelGGL((gn_apply_kernel<ACT, T, V>), dim3((unsigned)((long)a.n * cv.cuts * cv.slices)), dim3(THREADS), 0, a.st, (const T*)a.x, a.gamma, a.beta,
                     (const T*)a.side, pairs, a.mean, a.istd, (T*)a.out, a.eps, cv);
}

template <int ACT, class T, int V>
void backward_any(const GnArgs& a, const Cover& cv) {
  double* pairs = static_cast<double*>(a.workspace);
  float* chan = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + pair_bytes(a.n, cv));
  hipLaunchKernelGGL((gn_sums_kernel<1, ACT, T, V>), dim3((unsigned)((long)a.n * cv.slabs * cv.slices)), dim3(THREADS), 0, a.st, (const T*)a.x,
                     (const T*)a.dy, (const T*)a.side, a.gamma, a.beta, a.mean_in, a.istd_in, pairs, chan, cv);
  const int blocks = (int)((long)a.n * cv.cuts * cv.slices), params = (2 * a.c + 31) / 32;
  hipLaunchKernelGGL((gn_bwd_apply_kernel<ACT, T, V>), dim3((unsigned)(blocks + params)), dim3(THREADS), 0, a.st, (const T*)a.x, (const T*)a.dy,
                     (const T*)a.side, a.gamma, a.beta, a.mean_in, a.istd_in, pairs, chan, (T*)a.out, (T*)a.dres, a.dgamma, a.dbeta, (long)a.n * cv.slabs, blocks,
                     cv);
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

#define ACC_GN_ACT(F, T, V)                            \
  switch (act) {                                       \
    case ACT_NONE: F<ACT_NONE, T, V>(a, cv); break;    \
    case ACT_RELU: F<ACT_RELU, T, V>(a, cv); break;    \
    default: F<ACT_SILU, T, V>(a, cv); break;          \
  }
#define ACC_GN(F)                                                                                  \
  do {                                                                                             \
    Cover cv;                                                                                      \
    const int v = cover_for(a.n, a.hw, a.c, a.groups, dtype, &cv);                                 \
    if (dtype == DT_F32) { if (v == 4) ACC_GN_ACT(F, float, 4) else ACC_GN_ACT(F, float, 1) }      \
    else { if (v == 8) ACC_GN_ACT(F, bf16_t, 8) else ACC_GN_ACT(F, bf16_t, 1) }                    \
  } while (0)

bool shape_ok(int n, int hw, int c, int groups, int act, int dtype) {
  if (n <= 0 || hw <= 0 || c <= 0 || groups <= 0 || c % groups != 0 || act < ACT_NONE || act > ACT_SILU) return false;
  if (dtype != DT_F32 && dtype != DT_BF16) return false;
  if (hw >= (1 << 30) || c >= (1 << 24) || (long)n * groups >= 1L << 31) return false;      // (a thread counts its rows in 31 bits)
  Cover cv;
  cover_for(n, hw, c, groups, dtype, &cv);
  const long most = (long)n * cv.slices * (cv.slabs > cv.cuts ? cv.slabs : cv.cuts) + (2L * c + 31) / 32;
  return most < 1L << 24;                              // (a launch has fewer than 2^32 threads)
}

}  // namespace

// (0: refused, for either storage type, as the calls are: one size serves both)
size_t gn_workspace_bytes(int n, int hw, int c, int groups) {
  if (!shape_ok(n, hw, c, groups, ACT_NONE, DT_F32) || !shape_ok(n, hw, c, groups, ACT_NONE, DT_BF16)) return 0;
  // the sums of a backward pass in slabs, or one pair of sums per image and channel; whichever storage type needs more
  size_t most = (size_t)n * 2 * c * sizeof(float);
  for (int dtype : {(int)DT_F32, (int)DT_BF16}) {
    Cover cv;
    cover_for(n, hw, c, groups, dtype, &cv);
    const size_t b = pair_bytes(n, cv) + chan_bytes(n, cv);
    if (b > most) most = b;
  }
  return most;
}
// whether the sizes are taken and the workspace holds what a call writes into it
static bool room_ok(int n, int hw, int c, int groups, int act, int dtype, size_t workspace_bytes) {
  const size_t need = gn_workspace_bytes(n, hw, c, groups);
  return need && workspace_bytes >= need && shape_ok(n, hw, c, groups, act, dtype);
}

hipError_t gn_forward(const void* x, const float* gamma, const float* beta, const void* res, void* y, float* mean, float* istd, int n, int hw, int c,
                      int groups, int act, float eps, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!x || !gamma || !beta || !y || !mean || !istd || !workspace || !(eps >= 0.f)) return hipErrorInvalidValue;
  if (!room_ok(n, hw, c, groups, act, dtype, workspace_bytes)) return hipErrorInvalidValue;
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
  if (!room_ok(n, hw, c, groups, act, dtype, workspace_bytes)) return hipErrorInvalidValue;
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
