// The products of the linear cross-entropy (linear_ce.hip) for bf16 operands, on the bf16 matrix cores, with what surrounds them in their
// epilogues: logits leave a tile as the largest one of its columns and the sum of exponentials, or as dz.
//
// dz is left without the factor 1 / rows (a label's value is then -1 where its probability is small, exact in bf16) as the sum of two bf16
// values, hi + lo, which hold 16 bits of it.  dw, an fp32 result, is multiplied from both (relative error of a value 2^-17 at most, where hi alone
// would leave 2^-9); dx, which is rounded to bf16 itself, from hi.  The factor is applied to the fp32 accumulators.
#include "kernels.h"
#include "dtype.h"
#include "gemm_bf16.h"
#include "linear_ce.h"

#include <climits>

namespace acc {
namespace {

constexpr float LOG2E = 1.44269504088896341f;
// e^t to 2 roundings for t <= 0 (the result's error relative to it is that of t * log2 e, which is small where the result matters)
__device__ __forceinline__ float exp_fast(float t) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_exp2f(t * LOG2E);
#else
  return t;
#endif
}

// Tile `at` of a launch: every XCD takes a contiguous range (neighbours share operand rows in its L2), rows innermost.
__device__ __forceinline__ int xcd_tile(int blocks) { return ((int)blockIdx.x & 7) * (blocks >> 3) + ((int)blockIdx.x >> 3); }

template <class C>
__device__ __forceinline__ void add_bias(GemmAcc<C>& acc, const float* __restrict__ bias, int col0, int cols) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < C::NB; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = col0 + 32 * j + 8 * q + 4 * (lane >> 5);
      float b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = bias && n + e < cols ? bias[n + e] : 0.f;
#pragma unroll
      for (int i = 0; i < C::MB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += b[e];
    }
}

struct LogitArgs {
  GemmOperand x, w;
  const float* bias;                 // of the piece, or null
  const int32_t* labels;
  int n, d, cols, v0;                // rows, width, classes of the piece, its first class
  int tiles_m, tiles;
  // sums
  float *part, *z_label;
  int split0, splits;
  // dz
  const float *row_max, *row_rest;
  bf16_t *hi, *lo;
  int pitch, ignore;
  float* db_part;                    // null: not wanted
};

template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_sums_kernel(LogitArgs a, int blocks) {
  constexpr int RED = C::WN * C::BM * 3 * 4;
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS > RED ? C::LDS : RED];
  const int at = xcd_tile(blocks);
  if (at >= a.tiles) return;
  const int tile_n = at / a.tiles_m, tile_m = at - tile_n * a.tiles_m, m0 = tile_m * C::BM, n0 = tile_n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(a.x, a.x, a.w, m0, n0, 0, a.d, lds, acc);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn = wave % C::WN, wn0 = wn * 32 * C::NB;
  if (a.bias) add_bias<C>(acc, a.bias, n0 + wn0, a.cols);
  float(*red)[C::BM][3] = reinterpret_cast<float(*)[C::BM][3]>(lds);
  const bool edge = n0 + C::BN > a.cols;
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    if (edge) {
#pragma unroll
      for (int j = 0; j < C::NB; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (n0 + wn0 + 32 * j + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3) >= a.cols) acc[i][j][v] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, acc[i][j][v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    float s = 0.f, equal = 0.f;
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float t = acc[i][j][v] - mx;
        const bool top = acc[i][j][v] == mx;
        s += top ? 0.f : exp_fast(t);
        equal += top ? 1.f : 0.f;
      }
    s += __shfl_xor(s, 32);
    equal += __shfl_xor(equal, 32);
    const int row = wm0 + 32 * i + (lane & 31), m = m0 + row;
    if (lane < 32) {
      red[wn][row][0] = mx;
      red[wn][row][1] = s;
      red[wn][row][2] = equal;
    }
    // the label's logit, if it is one of the wave's
    const int lab = m < a.n ? a.labels[m] - a.v0 - (n0 + wn0) - 4 * (lane >> 5) : -1;
    const bool mine = m < a.n && (unsigned)a.labels[m] >= (unsigned)a.v0 && lab >= 0 && lab < 32 * C::NB && !(lab & 4) && lab + n0 + wn0 + 4 * (lane >> 5) < a.cols;
    if (__any(mine)) {
#pragma unroll
      for (int j = 0; j < C::NB; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (mine && lab == 32 * j + 8 * (v >> 2) + (v & 3)) a.z_label[m] = acc[i][j][v];
    }
  }
  __syncthreads();
  for (int row = tid; row < C::BM; row += C::THREADS) {
    if (m0 + row >= a.n) continue;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < C::WN; ++w) mx = fmaxf(mx, red[w][row][0]);
    float s = 0.f, equal = 0.f;
#pragma unroll
    for (int w = 0; w < C::WN; ++w) {
      const float mw = red[w][row][0], sw = red[w][row][1], ew = red[w][row][2];
      const bool top = mw == mx;
      s += top ? sw : (mw == -INFINITY ? sw : (sw + ew) * exp_fast(mw - mx));      // (no column there: ew counts what equals minus infinity)
      equal += top ? ew : 0.f;
    }
    float* p = a.part + (size_t)(m0 + row) * 2 * a.splits + a.split0 + tile_n;
    p[0] = mx;
    p[a.splits] = mx == -INFINITY && !(s != s) ? -1.f : s + (equal - 1.f);
  }
}

// sum over the 32 lanes of each half of the wave, in lanes 31 and 63
__device__ __forceinline__ float half_sum(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
#define ACC_DPP(ctrl, rows) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, true))
  v += ACC_DPP(0x111, 0xf);
  v += ACC_DPP(0x112, 0xf);
  v += ACC_DPP(0x114, 0xf);
  v += ACC_DPP(0x118, 0xf);
  v += ACC_DPP(0x142, 0xa);
#undef ACC_DPP
#endif
  return v;
}

template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_dz_kernel(LogitArgs a, int blocks) {
  constexpr int EP = C::NB * 64 + 16, OUT = C::WM * C::WN * 32 * EP * 2;      // per wave 32 staged rows of hi and lo
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS > OUT ? C::LDS : OUT];
  const int at = xcd_tile(blocks);
  if (at >= a.tiles) return;
  const int tile_n = at / a.tiles_m, tile_m = at - tile_n * a.tiles_m, m0 = tile_m * C::BM, n0 = tile_n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(a.x, a.x, a.w, m0, n0, 0, a.d, lds, acc);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
  if (a.bias) add_bias<C>(acc, a.bias, n0 + wn0, a.cols);
  const bool edge = n0 + C::BN > a.cols;
  char* const stg = lds + wave * (32 * EP * 2);
  float sum[C::NB][16];
#pragma unroll
  for (int j = 0; j < C::NB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[j][v] = 0.f;
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    const int m = m0 + wm0 + 32 * i + (lane & 31);
    const bool row_ok = m < a.n;
    const int label = row_ok ? a.labels[m] : -1;
    const float mx = row_ok ? a.row_max[m] : 0.f, rest = row_ok ? a.row_rest[m] : 0.f, inv = 1.f / (1.f + rest);
    const bool skip = !row_ok || (a.ignore != INT_MIN && label == a.ignore);
    const int lab = label - a.v0 - (n0 + wn0) - 4 * (lane >> 5);
    const bool mine = row_ok && (unsigned)label >= (unsigned)a.v0 && lab >= 0 && lab < 32 * C::NB && !(lab & 4);
    const bool any = __any(mine);
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float p[4], l[4];
        uint2 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = acc[i][j][4 * q + e] - mx;
          p[e] = exp_fast(t) * inv;
          if (any && mine && lab == 32 * j + 8 * q + e) p[e] = (expm1f(t) - rest) * inv;
          if (skip) p[e] = 0.f;
          if (edge && n0 + wn0 + 32 * j + 8 * q + 4 * (lane >> 5) + e >= a.cols) p[e] = 0.f;
          sum[j][4 * q + e] += p[e];
        }
        hi.x = pack_bf16(p[0], p[1]);
        hi.y = pack_bf16(p[2], p[3]);
        l[0] = p[0] - __uint_as_float(hi.x << 16);
        l[1] = p[1] - __uint_as_float(hi.x & 0xffff0000u);
        l[2] = p[2] - __uint_as_float(hi.y << 16);
        l[3] = p[3] - __uint_as_float(hi.y & 0xffff0000u);
        lo.x = pack_bf16(l[0], l[1]);
        lo.y = pack_bf16(l[2], l[3]);
        char* const to = stg + (lane & 31) * EP + (32 * j + 8 * q + 4 * (lane >> 5)) * 2;
        *reinterpret_cast<uint2*>(to) = hi;
        *reinterpret_cast<uint2*>(to + 32 * EP) = lo;
      }
    // whole rows: eight values per lane
    constexpr int PPR = C::NB * 4, RPI = 64 / PPR;
    const int c8 = lane % PPR, prow = lane / PPR, col = n0 + wn0 + 8 * c8;
#pragma unroll
    for (int it = 0; it < 32 / RPI; ++it) {
      const int r = prow + RPI * it, mm = m0 + wm0 + 32 * i + r;
      if (mm >= a.n || col >= a.pitch) continue;       // (the pitch is a multiple of 8)
      *reinterpret_cast<v4u*>(a.hi + (size_t)mm * a.pitch + col) = *reinterpret_cast<const v4u*>(stg + r * EP + c8 * 16);
      *reinterpret_cast<v4u*>(a.lo + (size_t)mm * a.pitch + col) = *reinterpret_cast<const v4u*>(stg + 32 * EP + r * EP + c8 * 16);
    }
  }
  if (!a.db_part) return;
  float* const to = a.db_part + (size_t)(tile_m * C::WM + wave / C::WN) * a.pitch;
#pragma unroll
  for (int j = 0; j < C::NB; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float t = half_sum(sum[j][v]);
      const int n = n0 + wn0 + 32 * j + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
      if ((lane & 31) == 31 && n < a.pitch) to[n] = t;
    }
}

// dx: sums[split][n][d] (+)= dz w over the split's classes of the piece
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_dx_kernel(GemmOperand dz, GemmOperand w, float* __restrict__ sums, int n, int d, int k, int k_per_split,
                                                               int tiles_m, int tiles, int splits, int add, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work >= tiles * splits) return;
  const int split = work / tiles, at = work - split * tiles, tile_n = at / tiles_m, tile_m = at - tile_n * tiles_m, m0 = tile_m * C::BM, n0 = tile_n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(dz, dz, w, m0, n0, split * k_per_split, min(k, (split + 1) * k_per_split), lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
  float* const out = sums + (size_t)split * n * d;
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j) {
      const int col = n0 + wn0 + 32 * j + (lane & 31);
      if (col >= d) continue;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int m = m0 + wm0 + 32 * i + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
        if (m >= n) continue;
        float* const o = out + (size_t)m * d + col;
        *o = add ? *o + acc[i][j][v] : acc[i][j][v];
      }
    }
}

// dx = scale * the splits' sums in order, rounded to bf16
__global__ __launch_bounds__(256) void lce_dx_finish_kernel(const float* __restrict__ sums, const float* __restrict__ scale, bf16_t* __restrict__ dx, size_t count,
                                                            int splits) {
  const float sc = scale[0];
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= count) return;
  if (i + 4 <= count && (count & 3) == 0) {
    float4 s = *reinterpret_cast<const float4*>(sums + i);
    for (int k = 1; k < splits; ++k) {
      const float4 q = *reinterpret_cast<const float4*>(sums + k * count + i);
      s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
    }
    const float v[4] = {s.x * sc, s.y * sc, s.z * sc, s.w * sc};
    Elem<bf16_t>::store4(dx + i, v);
    return;
  }
  for (size_t e = i; e < count && e < i + 4; ++e) {
    float s = sums[e];
    for (int k = 1; k < splits; ++k) s += sums[k * count + e];
    Elem<bf16_t>::store(dx + e, s * sc);
  }
}

// dw[class][d] = scale * sum over the rows of (hi + lo)[row][class] * x[row][d]
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_dw_kernel(GemmOperand hi, GemmOperand lo, GemmOperand x, const float* __restrict__ scale,
                                                               float* __restrict__ dw, int n, int d, int cols, int tiles_m, int tiles, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int at = xcd_tile(blocks);
  if (at >= tiles) return;
  const int tile_n = at / tiles_m, tile_m = at - tile_n * tiles_m, m0 = tile_m * C::BM, n0 = tile_n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(hi, lo, x, m0, n0, 0, n, lds, acc);
  const float sc = scale[0];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j) {
      const int col = n0 + wn0 + 32 * j + (lane & 31);
      if (col >= d) continue;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int m = m0 + wm0 + 32 * i + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
        if (m < cols) dw[(size_t)m * d + col] = acc[i][j][v] * sc;
      }
    }
}

__global__ __launch_bounds__(256) void lce_db_kernel(const float* __restrict__ part, const float* __restrict__ scale, float* __restrict__ db, int parts, int pitch,
                                                     int cols) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= cols) return;
  double s = 0.0;
  for (int k = 0; k < parts; ++k) s += (double)part[(size_t)k * pitch + j];
  db[j] = (float)(s * (double)scale[0]);
}

// out[r][0 .. pitch) = in[r][0 .. d), then zeros
__global__ __launch_bounds__(256) void lce_pad_kernel(const bf16_t* __restrict__ in, bf16_t* __restrict__ out, size_t total, int d, int pitch) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (size_t)gridDim.x * 256) {
    const size_t r = i / pitch, c = i - r * pitch;
    out[i] = c < (size_t)d ? in[r * d + c] : (bf16_t)0;
  }
}

//                WM WN MB NB BK NS   AT     BT  PARTS SWAP
typedef GemmCfg<2, 4, 4, 2, 64, 2, false, false, 1, true> Z256;
typedef GemmCfg<2, 2, 2, 2, 64, 2, false, false, 1, true> Z128;
typedef GemmCfg<2, 4, 4, 2, 64, 2, false, true, 1, false> X256;
typedef GemmCfg<2, 2, 2, 2, 64, 2, false, true, 1, false> X128;
typedef GemmCfg<2, 4, 4, 2, 32, 3, true, true, 2, false> W256;
typedef GemmCfg<2, 2, 2, 2, 32, 2, true, true, 2, false> W128;

inline size_t al256(size_t b) { return (b + 255) & ~(size_t)255; }
inline long up(long v, long m) { return (v + m - 1) / m * m; }
inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

// 256 x 256 tiles where there are enough of them for the compute units
inline bool large_tiles(long m, long n) { return ceil_div(m, 256) * ceil_div(n, 256) >= 192; }

struct Plan16 {
  int dp;                        // width as it is multiplied, a multiple of 8
  long piece, pieces, splits;    // classes of a piece (a multiple of 256), pieces, columns of `part`
  int pitch;                     // of dz
  bool z256, x256, w256;
  int dx_splits, dx_k;           // parts of a piece's classes, classes of a part
  size_t stats, part, x, w, hi, lo, dx, db, total;
};

Plan16 plan16(int n, int d, int classes, bool grads) {
  Plan16 p{};
  p.dp = (int)up(d, 8);
  // 256 MiB of dz, 1 GiB of filter
  long most = (1L << 26) / n / 256 * 256;
  if (most > (1L << 29) / p.dp / 256 * 256) most = (1L << 29) / p.dp / 256 * 256;
  if (!grads) {                  // (nothing of a piece is kept; a launch has fewer than 2^32 threads)
    most = (1L << 29) / p.dp / 256 * 256;
    const long by_grid = (1L << 20) / ceil_div(n, 128) * 256;
    if (most > by_grid) most = by_grid;
  }
  if (most < 256) most = 256;
  p.piece = up(classes, 256) <= most ? up(classes, 256) : most;
  p.pieces = ceil_div(classes, p.piece);
  p.z256 = large_tiles(n, p.piece);
  p.x256 = d >= 192 && n >= 192;
  p.w256 = large_tiles(p.piece, d);
  const int bn = p.z256 ? 256 : 128;
  p.splits = p.pieces * (p.piece / bn);
  p.pitch = (int)(p.pieces > 1 ? p.piece : up(classes, 64));
  const int bm = p.x256 ? 256 : 128;
  const long tiles = ceil_div(n, bm) * ceil_div(d, bm), slots = p.x256 ? 256 : 512;
  long s = slots / tiles;
  if (s > p.pitch / 256) s = p.pitch / 256;
  if (s < 1) s = 1;
  while (s > 1 && s * n * d > (1L << 26)) --s;
  p.dx_k = (int)up(ceil_div(p.pitch, s), 64);
  p.dx_splits = (int)ceil_div(p.pitch, p.dx_k);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.stats = take((size_t)(4 * (size_t)n + 64) * 4);
  p.part = take((size_t)n * 2 * p.splits * 4);
  p.x = take(p.dp != d ? (size_t)n * p.dp * 2 : 0);
  p.w = take(p.dp != d ? (size_t)p.piece * p.dp * 2 : 0);
  if (grads) {
    p.hi = take((size_t)n * p.pitch * 2);
    p.lo = take((size_t)n * p.pitch * 2);
    p.dx = take((size_t)p.dx_splits * n * d * 4);
    p.db = take((size_t)2 * ceil_div(n, 128) * p.pitch * 4);
  }
  p.total = at;
  return p;
}

template <class C> inline dim3 grid_of(long work, int* blocks) {
  *blocks = (int)((work + 7) / 8 * 8);
  return dim3((unsigned)*blocks);
}

}  // namespace

// the operands' rows fit 32-bit byte ranges
bool linear_ce_bf16_takes(int n, int d, int classes) { return (long)n * up(d, 8) * 2 <= 0xFFFFFF00L && d >= 16; }

size_t linear_ce_bf16_workspace_bytes(int n, int d, int classes, bool grads) { return plan16(n, d, classes, grads).total; }

hipError_t linear_ce_bf16(const LceArgs& a) {
  const bool grads = a.dx || a.dw || a.db;
  const Plan16 p = plan16(a.n, a.d, a.classes, grads);
  const LceStats s = lce_stats(a, p.stats);
  hipStream_t st = a.st;
  const bf16_t* x = (const bf16_t*)a.x;
  auto pad = [&](const void* in, size_t at, long rows) {
    const size_t total = (size_t)rows * p.dp;
    const unsigned blocks = (unsigned)(total / 256 + 1 < 4096 ? total / 256 + 1 : 4096);
    hipLaunchKernelGGL(lce_pad_kernel, dim3(blocks), dim3(256), 0, st, (const bf16_t*)in, (bf16_t*)(a.ws + at), total, a.d, p.dp);
    return (const bf16_t*)(a.ws + at);
  };
  if (p.dp != a.d) x = pad(a.x, p.x, a.n);
  LogitArgs g{};
  g.x = GemmOperand{x, a.n, p.dp, p.dp};
  g.labels = a.labels;
  g.n = a.n; g.d = p.dp;
  g.part = (float*)(a.ws + p.part); g.z_label = s.z_label; g.splits = (int)p.splits;
  g.row_max = s.row_max; g.row_rest = s.row_rest;
  g.hi = (bf16_t*)(a.ws + p.hi); g.lo = (bf16_t*)(a.ws + p.lo); g.pitch = p.pitch; g.ignore = a.ignore;
  g.db_part = a.db ? (float*)(a.ws + p.db) : nullptr;
  const int bm = p.z256 ? 256 : 128;
  g.tiles_m = (int)ceil_div(a.n, bm);
  auto piece = [&](long k) {
    g.v0 = (int)(k * p.piece);
    g.cols = (int)(a.classes - g.v0 < p.piece ? a.classes - g.v0 : p.piece);
    const bf16_t* w = (const bf16_t*)a.w + (size_t)g.v0 * a.d;
    if (p.dp != a.d) w = pad(w, p.w, g.cols);
    g.w = GemmOperand{w, g.cols, p.dp, p.dp};
    g.bias = a.bias ? a.bias + g.v0 : nullptr;
    g.split0 = (int)(k * (p.piece / bm));
  };
  int blocks;
  for (long k = 0; k < p.pieces; ++k) {
    piece(k);
    // every column of `part`: those of a last piece that has fewer classes, too
    g.tiles = (int)(g.tiles_m * (p.piece / bm));
    if (p.z256) hipLaunchKernelGGL(lce_sums_kernel<Z256>, grid_of<Z256>(g.tiles, &blocks), dim3(Z256::THREADS), 0, st, g, blocks);
    else hipLaunchKernelGGL(lce_sums_kernel<Z128>, grid_of<Z128>(g.tiles, &blocks), dim3(Z128::THREADS), 0, st, g, blocks);
  }
  if (const hipError_t e = lce_join(a, s, g.part, (int)p.splits); e != hipSuccess || !grads) return e;
  for (long k = 0; k < p.pieces; ++k) {
    if (k > 0 || p.pieces > 1) piece(k);
    const int pitch_here = p.pieces > 1 ? (int)up(g.cols, 64) : p.pitch;        // classes of the piece that are multiplied
    g.tiles = (int)(g.tiles_m * ceil_div(pitch_here, bm));
    if (p.z256) hipLaunchKernelGGL(lce_dz_kernel<Z256>, grid_of<Z256>(g.tiles, &blocks), dim3(Z256::THREADS), 0, st, g, blocks);
    else hipLaunchKernelGGL(lce_dz_kernel<Z128>, grid_of<Z128>(g.tiles, &blocks), dim3(Z128::THREADS), 0, st, g, blocks);
    if (a.db)
      hipLaunchKernelGGL(lce_db_kernel, dim3((unsigned)((g.cols + 255) / 256)), dim3(256), 0, st, g.db_part, s.scale, a.db + g.v0, 2 * g.tiles_m, p.pitch, g.cols);
    const GemmOperand hi{g.hi, a.n, p.pitch, p.pitch}, lo{g.lo, a.n, p.pitch, p.pitch};
    if (a.dx) {
      float* const sums = (float*)(a.ws + p.dx);
      const int tm = (int)ceil_div(a.n, p.x256 ? 256 : 128), tiles = tm * (int)ceil_div(a.d, p.x256 ? 256 : 128);
      const long work = (long)tiles * p.dx_splits;
      if (p.x256)
        hipLaunchKernelGGL(lce_dx_kernel<X256>, grid_of<X256>(work, &blocks), dim3(X256::THREADS), 0, st, hi, g.w, sums, a.n, a.d, pitch_here, p.dx_k, tm, tiles,
                           p.dx_splits, k > 0, blocks);
      else
        hipLaunchKernelGGL(lce_dx_kernel<X128>, grid_of<X128>(work, &blocks), dim3(X128::THREADS), 0, st, hi, g.w, sums, a.n, a.d, pitch_here, p.dx_k, tm, tiles,
                           p.dx_splits, k > 0, blocks);
    }
    if (a.dw) {
      const int tm = (int)ceil_div(g.cols, p.w256 ? 256 : 128), tiles = tm * (int)ceil_div(a.d, p.w256 ? 256 : 128);
      float* const dw = a.dw + (size_t)g.v0 * a.d;
      if (p.w256)
        hipLaunchKernelGGL(lce_dw_kernel<W256>, grid_of<W256>(tiles, &blocks), dim3(W256::THREADS), 0, st, hi, lo, g.x, s.scale, dw, a.n, a.d, g.cols, tm, tiles, blocks);
      else
        hipLaunchKernelGGL(lce_dw_kernel<W128>, grid_of<W128>(tiles, &blocks), dim3(W128::THREADS), 0, st, hi, lo, g.x, s.scale, dw, a.n, a.d, g.cols, tm, tiles, blocks);
    }
  }
  if (a.dx) {
    const size_t count = (size_t)a.n * a.d;
    hipLaunchKernelGGL(lce_dx_finish_kernel, dim3((unsigned)((count + 1023) / 1024)), dim3(256), 0, st, (const float*)(a.ws + p.dx), s.scale, (bf16_t*)a.dx, count,
                       p.dx_splits);
  }
  return hipGetLastError();
}

}  // namespace acc
