// The products of the linear cross-entropy (linear_ce.hip) for bf16 operands, on the bf16 matrix cores, with what surrounds them in their
// epilogues: logits leave a tile as the largest one of its columns and the sum of exponentials, or as dz.
//
// dz is left without the factor 1 / rows (a label's value is then -1 where its probability is small, exact in bf16) as the sum of two or three
// bf16 values, the first the nearest one, the next the nearest to what is left: one leaves a relative error of up to 2^-8, two of 2^-16, three of 2^-24.
// dw, an fp32 result, is multiplied from all of them.  Two leave 1.2e-6 to 1.7e-6 of it, however many rows there are, where the roundings of a sum in
// fp32 grow with the root of the rows (relative errors of dw, 1e-6, 64 / 512 / 1024 / 2048 / 4096 / 8192 / 16384 rows: fp32 throughout 0.2 / 0.4 / 0.6 /
// 0.8 / 1.15 / 1.6 / 2.3; three values 0.1 / 0.25 / 0.3 / 0.4 / 0.6 / 0.3 / 0.4; 256 to 512 wide, 1000 to 4000 classes).  So from 4096 rows on, where two
// values are off by at most half as much again as fp32 sums, there are two, and three below, where they would be off by two to eight times as much
// (4096 x 2048 x 65536, all results, two / three: 5.5 / 6.7 ms).  dx is multiplied from the first two: one would do if its errors stayed beside the result's
// own rounding, but a row of dz sums to zero, so that what the classes' weights have in common cancels in dx and its errors do not (relative error of dx,
// 300 x 128 x 10, weights with a common part of 10 and 30 times their spread: one value 0.012 and 0.038, two 0.0017, which is the rounding of the result;
// 4096 x 2048 x 65536, all results, 4720 and 5525 us).  The factor is applied to the fp32 accumulators.
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

template <class C>
__device__ __forceinline__ void add_bias(GemmAcc<C>& acc, const float* __restrict__ bias, int col0, int cols) {
  const int lane = threadIdx.x & 63;
  const bool whole = col0 + 32 * C::NB <= cols;        // the wave's columns exist
#pragma unroll
  for (int j = 0; j < C::NB; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = col0 + 32 * j + 8 * q + 4 * (lane >> 5);
      float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
      if (whole) {
        b = *reinterpret_cast<const float4*>(bias + n);        // (a piece starts at a multiple of 256 classes)
      } else {
        if (n < cols) b.x = bias[n];
        if (n + 1 < cols) b.y = bias[n + 1];
        if (n + 2 < cols) b.z = bias[n + 2];
        if (n + 3 < cols) b.w = bias[n + 3];
      }
#pragma unroll
      for (int i = 0; i < C::MB; ++i) {
        acc[i][j][4 * q] += b.x;
        acc[i][j][4 * q + 1] += b.y;
        acc[i][j][4 * q + 2] += b.z;
        acc[i][j][4 * q + 3] += b.w;
      }
#if defined(__HIP_DEVICE_COMPILE__)
      __builtin_amdgcn_sched_barrier(0);               // (all of them at once would not fit the registers beside the accumulators)
#endif
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
  float* z;                          // sums: the logits are kept here, too (null: not)
  bf16_t* dz[3];
  int pitch, ignore;
  float* db_part;                    // null: not wanted
  // dz that joins the rows' sums itself
  int join, classes;
  float *loss_rows, *scale;
};

// Logits of a tile, of which the largest one of a row and the sum of exponentials leave it.  4096 x 2048 x 16384: 250 us, 1097 TFLOP/s (a large library product
// reaches 1378); matrix cores busy 60 % of the time.
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_sums_kernel(LogitArgs a, int blocks) {
  constexpr int RED = C::WN * C::BM * 3 * 4;
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS > RED ? C::LDS : RED];
  const int at = xcd_tile(blocks);
  if (at >= a.tiles) return;
  const TileAt where = tile_at(at, a.tiles_m, a.tiles);
  const int tile_m = where.m, tile_n = where.n, m0 = tile_m * C::BM, n0 = tile_n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(a.x, a.w, m0, n0, 0, a.d, lds, acc);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn = wave % C::WN, wn0 = wn * 32 * C::NB;
  if (a.bias) add_bias<C>(acc, a.bias, n0 + wn0, a.cols);
  float(*red)[C::BM][3] = reinterpret_cast<float(*)[C::BM][3]>(lds);
  const bool edge = n0 + C::BN > a.cols;
  if (a.z) {                                           // four columns of a row per lane
#pragma unroll
    for (int i = 0; i < C::MB; ++i) {
      const int m = m0 + wm0 + 32 * i + (lane & 31);
      float* const to = a.z + (size_t)m * a.pitch;
#pragma unroll
      for (int j = 0; j < C::NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = n0 + wn0 + 32 * j + 8 * q + 4 * (lane >> 5);
          if (m < a.n && n < a.pitch)
            *reinterpret_cast<float4*>(to + n) = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        }
    }
  }
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

// The logits again, which leave as dz, and the columns' sums of a tile.  4096 x 2048 x 16384, two parts: 291 us, 945 TFLOP/s beside writing 268 MB.
template <class C, int PARTS>
__global__ __launch_bounds__(C::THREADS, 2) void lce_dz_kernel(LogitArgs a, int blocks) {
  constexpr int EP = C::NB * 64 + 16, OUT = C::WM * C::WN * 32 * EP * PARTS;      // per wave 32 staged rows of every part
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS > OUT ? C::LDS : OUT];
  constexpr bool JOINS = C::BM == 64;                  // (the larger tiles' registers are full)
  __shared__ float row_max[JOINS ? C::BM : 1], row_rest[JOINS ? C::BM : 1];
  if (JOINS && (int)blockIdx.x >= blocks) {                     // (with `join`)
    mean_of_rows<C::THREADS>(nullptr, a.labels, a.ignore, a.n, a.scale, nullptr);
    return;
  }
  const int at = xcd_tile(blocks);
  if (at >= a.tiles) return;
  const TileAt where = tile_at(at, a.tiles_m, a.tiles);
  const int tile_m = where.m, tile_n = where.n, m0 = tile_m * C::BM, n0 = tile_n * C::BN;
  constexpr int LANES = C::THREADS / C::BM;            // of a row
  if (const int r = threadIdx.x / LANES, m = m0 + r; JOINS && m < a.n) {
    RowStats st{0.f, 0.f, 0.f};
    if (a.join) st = join_row(a.part, a.z_label, a.labels, a.ignore, m, a.splits, a.classes, LANES);
    else { st.max = a.row_max[m]; st.rest = a.row_rest[m]; }
    if (threadIdx.x % LANES == 0) {
      row_max[r] = st.max; row_rest[r] = st.rest;
      if (a.join && tile_n == 0) a.loss_rows[m] = st.loss;
    }
  }
  GemmAcc<C> acc;
  gemm_tile<C>(a.x, a.w, m0, n0, 0, a.d, lds, acc);
  if (JOINS) __syncthreads();                          // the rows' sums are there
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
  if (a.bias) add_bias<C>(acc, a.bias, n0 + wn0, a.cols);
  const bool edge = n0 + C::BN > a.cols;
  char* const stg = lds + wave * (32 * EP * PARTS);
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
    const float mx = !row_ok ? 0.f : JOINS ? row_max[m - m0] : a.row_max[m], rest = !row_ok ? 0.f : JOINS ? row_rest[m - m0] : a.row_rest[m], inv = 1.f / (1.f + rest);
    const bool skip = !row_ok || (a.ignore != INT_MIN && label == a.ignore);
    const int lab = label - a.v0 - (n0 + wn0) - 4 * (lane >> 5);
    const bool mine = row_ok && (unsigned)label >= (unsigned)a.v0 && lab >= 0 && lab < 32 * C::NB && !(lab & 4);
    const bool any = __any(mine);
    const float p_label = mine ? (expm1f(a.z_label[m] - mx) - rest) * inv : 0.f;
    const int at_label = mine ? lab : -1;
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = exp_fast(acc[i][j][4 * q + e] - mx) * inv;
          if (any) p[e] = at_label == 32 * j + 8 * q + e ? p_label : p[e];
          p[e] = skip ? 0.f : p[e];
          if (edge && n0 + wn0 + 32 * j + 8 * q + 4 * (lane >> 5) + e >= a.cols) p[e] = 0.f;
          sum[j][4 * q + e] += p[e];
        }
        char* const to = stg + (lane & 31) * EP + (32 * j + 8 * q + 4 * (lane >> 5)) * 2;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const uint2 w = make_uint2(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]));
          *reinterpret_cast<uint2*>(to + part * 32 * EP) = w;
          if (part + 1 < PARTS) {                      // what is left
            p[0] -= __uint_as_float(w.x << 16);
            p[1] -= __uint_as_float(w.x & 0xffff0000u);
            p[2] -= __uint_as_float(w.y << 16);
            p[3] -= __uint_as_float(w.y & 0xffff0000u);
          }
        }
#if defined(__HIP_DEVICE_COMPILE__)
        __builtin_amdgcn_sched_barrier(0);             // four values at a time: more do not fit the registers beside the accumulators
#endif
      }
    // whole rows: eight values per lane
    constexpr int PPR = C::NB * 4, RPI = 64 / PPR;
    const int c8 = lane % PPR, prow = lane / PPR, col = n0 + wn0 + 8 * c8;
#pragma unroll
    for (int it = 0; it < 32 / RPI; ++it) {
      const int r = prow + RPI * it, mm = m0 + wm0 + 32 * i + r;
      if (mm >= a.n || col >= a.pitch) continue;       // (the pitch is a multiple of 8)
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        *reinterpret_cast<v4u*>(a.dz[part] + (size_t)mm * a.pitch + col) = *reinterpret_cast<const v4u*>(stg + part * 32 * EP + r * EP + c8 * 16);
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

// dz from kept logits: eight columns per thread, a workgroup's rows one after the other (DZ_ROWS of them), and their columns' sums.  4096 x 16384, two parts:
// 109 us for 537 MB, 4.9 TB/s.
constexpr int DZ_ROWS = 16;
template <int PARTS>
__global__ __launch_bounds__(256) void lce_dz_kept_kernel(LogitArgs a, int blocks_across) {
  const int across = (int)blockIdx.x % blocks_across, slab = (int)blockIdx.x / blocks_across;
  const int col = (across * 256 + (int)threadIdx.x) * 8;
  if (col >= a.pitch) return;                          // (a multiple of 64)
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  const int r0 = slab * DZ_ROWS, r1 = min(r0 + DZ_ROWS, a.n);
  for (int r = r0; r < r1; r += 2) {                   // two rows on their way at once
    float4 lo[2], hi[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float* from = a.z + (size_t)min(r + u, r1 - 1) * a.pitch + col;
      lo[u] = *reinterpret_cast<const float4*>(from);
      hi[u] = *reinterpret_cast<const float4*>(from + 4);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (r + u >= r1) break;
      const int label = a.labels[r + u], lab = label - a.v0 - col;
      const bool skip = a.ignore != INT_MIN && label == a.ignore, mine = (unsigned)label >= (unsigned)a.v0 && lab >= 0 && lab < 8;
      const float mx = a.row_max[r + u], rest = a.row_rest[r + u], inv = 1.f / (1.f + rest);
      float p[8] = {lo[u].x, lo[u].y, lo[u].z, lo[u].w, hi[u].x, hi[u].y, hi[u].z, hi[u].w};
      const float p_label = mine ? (expm1f(a.z_label[r + u] - mx) - rest) * inv : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = exp_fast(p[e] - mx) * inv;
        if (mine && lab == e) p[e] = p_label;
        if (skip || col + e >= a.cols) p[e] = 0.f;
        sum[e] += p[e];
      }
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        v4u w;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          w[q] = pack_bf16(p[2 * q], p[2 * q + 1]);
          p[2 * q] -= __uint_as_float(w[q] << 16);
          p[2 * q + 1] -= __uint_as_float(w[q] & 0xffff0000u);
        }
        *reinterpret_cast<v4u*>(a.dz[part] + (size_t)(r + u) * a.pitch + col) = w;
      }
    }
  }
  if (!a.db_part) return;
  float* const to = a.db_part + (size_t)slab * a.pitch + col;
  *reinterpret_cast<float4*>(to) = make_float4(sum[0], sum[1], sum[2], sum[3]);
  *reinterpret_cast<float4*>(to + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
}

// dx: sums[split][n][d] (+)= dz w over the split's classes of the piece, dz as the sum of its first two parts, or dx itself where there is one split of one piece.
// 4096 x 2048 x 16384: 449 us, 1225 TFLOP/s of the matrix cores (72 % busy).
struct DxArgs {
  GemmOperand dz, w;
  float* sums;
  bf16_t* dx;                    // not null: scaled and rounded here
  const float* scale;
  int n, d, k, k_per_split, tiles_m, tiles, work, add;
};
template <class C>
__device__ __forceinline__ void dx_tile(const DxArgs& a, int work, char* lds) {
  const int split = work / a.tiles, at = work - split * a.tiles, n = a.n, d = a.d;
  const TileAt where = tile_at(at, a.tiles_m, a.tiles);
  const int m0 = where.m * C::BM, n0 = where.n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(a.dz, a.w, m0, n0, split * a.k_per_split, min(a.k, (split + 1) * a.k_per_split), lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
  float* const out = a.sums + (size_t)split * n * d;
  const bool direct = C::BM == 64 && a.dx;             // (of launches with few tiles only)
  const float sc = direct ? a.scale[0] : 1.f;
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j) {
      const int col = n0 + wn0 + 32 * j + (lane & 31), mb = m0 + wm0 + 32 * i + 4 * (lane >> 5);
      if (col >= d) continue;
      if (direct) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 8 * (v >> 2) + (v & 3);
          if (mb + r < n) Elem<bf16_t>::store(a.dx + (size_t)(mb + r) * d + col, acc[i][j][v] * sc);
        }
        continue;
      }
      float* const o = out + (size_t)mb * d + col;
      float old[16];                                   // asked for together (one after the other, each behind the store before it: 80 us of 337)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = 8 * (v >> 2) + (v & 3);
        old[v] = a.add && mb + r < n ? o[(size_t)r * d] : 0.f;
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = 8 * (v >> 2) + (v & 3);
        if (mb + r < n) o[(size_t)r * d] = old[v] + acc[i][j][v];
      }
    }
}
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_dx_kernel(DxArgs a, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work < a.work) dx_tile<C>(a, work, lds);
}

// dx = scale * the splits' sums in order, rounded to bf16
__device__ __forceinline__ void finish_dx(const float* __restrict__ sums, float sc, bf16_t* __restrict__ dx, size_t count, int splits, size_t block) {
  const size_t i = (block * 256 + threadIdx.x) * 4;
  if (i >= count) return;
  if ((count & 3) == 0) {
    float4 s = *reinterpret_cast<const float4*>(sums + i);
#pragma unroll 4
    for (int k = 1; k < splits; ++k) {
      const float4 q = *reinterpret_cast<const float4*>(sums + k * count + i);
      s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
    }
    *reinterpret_cast<uint2*>(dx + i) = make_uint2(pack_bf16(s.x * sc, s.y * sc), pack_bf16(s.z * sc, s.w * sc));
    return;
  }
  for (size_t e = i; e < count && e < i + 4; ++e) {
    float s = sums[e];
    for (int k = 1; k < splits; ++k) s += sums[k * count + e];
    Elem<bf16_t>::store(dx + e, s * sc);
  }
}
// db = scale * the row tiles' sums of a piece
__device__ __forceinline__ void finish_db(const float* __restrict__ part, float sc, float* __restrict__ db, int parts, int pitch, int cols, int block) {
  const int j = block * 256 + threadIdx.x;
  if (j >= cols) return;
  double s = 0.0;
#pragma unroll 8
  for (int k = 0; k < parts; ++k) s += (double)part[(size_t)k * pitch + j];
  db[j] = (float)(s * (double)sc);
}
// dw = scale * the splits' sums in order
__device__ __forceinline__ void finish_dw(const float* __restrict__ sums, float sc, float* __restrict__ dw, size_t count, int splits, size_t block) {
  for (size_t i = block * 1024 + threadIdx.x; i < count && i < (block + 1) * 1024; i += 256) {
    float s = sums[i];
#pragma unroll 4
    for (int k = 1; k < splits; ++k) s += sums[k * count + i];
    dw[i] = s * sc;
  }
}
struct Finish {
  const float *sums, *part, *scale, *dw_sums;
  bf16_t* dx;
  float *db, *dw;
  size_t count, dw_count;
  int splits, dw_splits, dx_blocks, dw_blocks, parts, pitch, cols;
};
__global__ __launch_bounds__(256) void lce_finish_kernel(Finish f) {
  const float sc = f.scale[0];
  if ((int)blockIdx.x < f.dx_blocks) finish_dx(f.sums, sc, f.dx, f.count, f.splits, blockIdx.x);
  else if ((int)blockIdx.x < f.dx_blocks + f.dw_blocks) finish_dw(f.dw_sums, sc, f.dw, f.dw_count, f.dw_splits, blockIdx.x - f.dx_blocks);
  else finish_db(f.part, sc, f.db, f.parts, f.pitch, f.cols, (int)blockIdx.x - f.dx_blocks - f.dw_blocks);
}

// dw[class][d] = scale * sum over the rows of dz[row][class] * x[row][d], dz as the sum of its parts; with several splits of the rows their sums
// (without the factor) lie one behind the other.  4096 x 2048 x 16384, two parts: 418 us, 1315 TFLOP/s of the matrix cores (75 % busy).
struct DwArgs {
  GemmOperand dz, x;
  const float* scale;
  float* out;
  int n, d, cols, n_per_split, tiles_m, tiles, splits;
};
template <class C>
__device__ __forceinline__ void dw_tile(const GemmOperand& dz, const GemmOperand& x, const float* __restrict__ scale, float* __restrict__ out, int n, int d, int cols,
                                        int n_per_split, int tiles_m, int tiles, int splits, int work, char* lds) {
  const int split = work / tiles, at = work - split * tiles;
  const TileAt where = tile_at(at, tiles_m, tiles);
  const int m0 = where.m * C::BM, n0 = where.n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(dz, x, m0, n0, split * n_per_split, min(n, (split + 1) * n_per_split), lds, acc);
  const float sc = splits > 1 ? 1.f : scale[0];
  float* const dw = out + (size_t)split * cols * d;
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
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void lce_dw_kernel(GemmOperand dz, GemmOperand x, const float* __restrict__ scale, float* __restrict__ out, int n, int d,
                                                               int cols, int n_per_split, int tiles_m, int tiles, int splits, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work >= tiles * splits) return;
  dw_tile<C>(dz, x, scale, out, n, d, cols, n_per_split, tiles_m, tiles, splits, work, lds);
}

struct MeanArgs {
  const float* loss_rows;
  const int32_t* labels;
  float* loss;
  int n, ignore;
};
// dx, dw, db (and the mean loss) in one launch: they all wait for dz only, so where there are few tiles two launches less (us, all results, before / with it:
// 64 x 64 x 64 22.3 / 18.9, 1000 x 1024 x 1000 59.6 / 49.6; and with the rows' sums joined by dz, 64 x 64 x 64 14.9)
template <class CX, class CW>
__global__ __launch_bounds__(256, 2) void lce_grads_kernel(DxArgs x, DwArgs w, Finish rest, MeanArgs mean, int x_blocks, int w_blocks, int db_blocks) {
  static_assert(CX::THREADS == 256 && CW::THREADS == 256, "one shape of workgroups");
  __shared__ __attribute__((aligned(1024))) char lds[CX::LDS > CW::LDS ? CX::LDS : CW::LDS];
  const int block = blockIdx.x;                        // (each part begins at a multiple of eight)
  if (block < x_blocks) {
    const int work = (block & 7) * (x_blocks >> 3) + (block >> 3);
    if (work < x.work) dx_tile<CX>(x, work, lds);
  } else if (block < x_blocks + w_blocks) {
    const int work = (block & 7) * (w_blocks >> 3) + ((block - x_blocks) >> 3);
    if (work < w.tiles * w.splits) dw_tile<CW>(w.dz, w.x, w.scale, w.out, w.n, w.d, w.cols, w.n_per_split, w.tiles_m, w.tiles, w.splits, work, lds);
  } else if (block < x_blocks + w_blocks + db_blocks) {
    finish_db(rest.part, rest.scale[0], rest.db, rest.parts, rest.pitch, rest.cols, block - x_blocks - w_blocks);
  } else {
    mean_of_rows<256>(mean.loss_rows, mean.labels, mean.ignore, mean.n, nullptr, mean.loss);
  }
}

// out[r][0 .. pitch) = in[r][0 .. d), then zeros; eight values per thread, read at any address (11261 rows of 3015: 62 us one by one, 28 so)
__global__ __launch_bounds__(256) void lce_pad_kernel(const bf16_t* __restrict__ in, bf16_t* __restrict__ out, size_t eights, int d, int pitch) {
  typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
  const size_t across = pitch / 8;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < eights; i += (size_t)gridDim.x * 256) {
    const size_t r = i / across;
    const int c = (int)(i - r * across) * 8;
    const bf16_t* from = in + r * d + c;
    v4u v;
    if (c + 8 <= d) {
      const any q = *reinterpret_cast<const any*>(from);
      v = v4u{q.x, q.y, q.z, q.w};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = (c + 2 * e < d ? (uint32_t)from[2 * e] : 0u) | (c + 2 * e + 1 < d ? (uint32_t)from[2 * e + 1] << 16 : 0u);
    }
    *reinterpret_cast<v4u*>(out + i * 8) = v;
  }
}

//                WM WN MB NB BK NS   AT     BT  PARTS SWAP
typedef GemmCfg<2, 4, 4, 2, 64, 2, false, false, 1, true> Z256;
typedef GemmCfg<2, 2, 2, 2, 64, 2, false, false, 1, true> Z128;
typedef GemmCfg<2, 2, 1, 1, 64, 4, false, false, 1, true> Z64;
typedef GemmCfg<2, 4, 4, 2, 32, 3, false, true, 2, false> X256;        // dx
typedef GemmCfg<2, 2, 2, 2, 32, 3, false, true, 2, false> X128;
typedef GemmCfg<2, 2, 1, 1, 32, 4, false, true, 2, false> X64;
typedef GemmCfg<2, 4, 4, 2, 32, 3, true, true, 2, false> W256;
typedef GemmCfg<2, 2, 2, 2, 32, 2, true, true, 2, false> W128;
typedef GemmCfg<2, 2, 1, 1, 32, 4, true, true, 2, false> W64;
typedef GemmCfg<2, 4, 4, 2, 32, 2, true, true, 3, false> V256;        // dw with three parts of dz
typedef GemmCfg<2, 2, 2, 2, 32, 2, true, true, 3, false> V128;
typedef GemmCfg<2, 2, 1, 1, 32, 3, true, true, 3, false> V64;

struct Plan16 {
  int dp;                        // width as it is multiplied, a multiple of 8
  int parts;                     // bf16 values that dz is the sum of
  long piece, pieces, splits;    // classes of a piece (a multiple of 256), pieces, columns of `part`
  int pitch;                     // of dz
  bool keep;                     // the last piece's logits are kept from the first sweep for the second, which begins with it
  int zt;                        // tiles of the logits
  bool together;                 // dx, dw and db in one launch of 64 x 64 tiles
  bool join;                     // the rows' sums are joined by the workgroups of dz, not by a launch of their own
  Choice dx, dw;
  size_t stats, part, x, w, z, dz[3], dx_sums, dw_sums, db, total;
};

Plan16 plan16(int n, int d, int classes, bool grads) {
  Plan16 p{};
  p.dp = (int)up(d, 8);
  p.parts = n < 4096 ? 3 : 2;
  // 2^26 values of dz (128 MiB for each part, 256 MiB of kept logits), 1 GiB of filter, 256 classes at least (more than 2^18 rows then have more)
  long most = (1L << 26) / n / 256 * 256;
  if (most > (1L << 29) / p.dp / 256 * 256) most = (1L << 29) / p.dp / 256 * 256;
  if (!grads) {                  // (nothing of a piece is kept; a launch has fewer than 2^32 threads)
    most = (1L << 29) / p.dp / 256 * 256;
    const long by_grid = (1L << 20) / ceil_div(n, 64) * 256;
    if (most > by_grid) most = by_grid;
  }
  if (most < 256) most = 256;
  p.piece = up(classes, 256) <= most ? up(classes, 256) : most;
  p.pieces = ceil_div(classes, p.piece);
  const long whole = p.pieces > 1 ? p.piece : classes;
  p.zt = choose(RowsByRows, n, whole, p.dp, 1, 0, 1L << 30).tile;
  p.splits = (p.pieces - 1) * (p.piece / p.zt) + ceil_div(classes - (p.pieces - 1) * p.piece, p.zt);
  p.pitch = (int)(p.pieces > 1 ? p.piece : up(classes, 64));
  p.dx = choose(ByColumns, n, d, p.pitch, 2, 1L << 25, 256);
  p.dw = choose(ByColumns, whole, d, n, p.parts, 1L << 24, 128);
  const Choice dx = choose(ByColumns, n, d, p.pitch, 2, 1L << 25, 256, 2), dw = choose(ByColumns, whole, d, n, p.parts, 1L << 24, 128, 2);
  p.together = p.pieces == 1 && ceil_div(d, 64) * (ceil_div(n, 64) * dx.splits + ceil_div(whole, 64) * dw.splits) <= 1024;
  if (p.together) { p.dx = dx; p.dw = dw; }
  // (a row's sums are then read by every tile across)
  p.join = grads && p.together && p.zt == 64 && p.splits <= 16;
  // The last piece's logits are kept where working them out again takes longer than writing and reading them, by predicted times: a launch, of up to sixteen rows
  // one behind the other, the columns' sums of sixteen rows each, which a thread adds up (66 ns each), and another launch for the rows' sums where dz would
  // join them.  us, all results, worked out again / kept: 43 x 1064 x 10 21 / 28, 1000 x 1024 x 1000 42 / 51, 200 x 1024 x 3000 46 / 50, 4096 x 512 x 16384
  // 565 / 619, 65536 x 1024 x 1000 971 / 1186, 131072 x 512 x 100 506 / 889; 1 x 1024 x 1000 26 / 23, 6 x 216 x 49305 73 / 57, 777 x 512 x 50001 489 / 448,
  // 4096 x 2048 x 16384 1394 / 1314.  Of 140 sizes (up to 2^20 rows, widths 16 to 4096, 2 to 100000 classes) four take the slower way by more than 5 %, 10 at most.
  const double again = tile_us(RowsByRows, p.zt == 256 ? 0 : p.zt == 128 ? 1 : 2, ceil_div(n, p.zt) * ceil_div(whole, p.zt), p.dp / 64.0);
  const double kept = 3.5 + 0.5 * (n < DZ_ROWS ? n : DZ_ROWS) + (double)n * p.pitch * 8 / 5e6 + 0.066 * (ceil_div(n, DZ_ROWS) - ceil_div(n, p.zt)) + (p.join ? 5.0 : 0.0);
  p.keep = grads && again > kept;
  if (p.keep) p.join = false;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.stats = take((size_t)(4 * (size_t)n + 64) * 4);
  p.part = take((size_t)n * 2 * p.splits * 4);
  p.x = take(p.dp != d ? (size_t)n * p.dp * 2 : 0);
  p.w = take(p.dp != d ? (size_t)p.piece * p.dp * 2 : 0);
  if (grads) {
    for (int i = 0; i < p.parts; ++i) p.dz[i] = take((size_t)n * p.pitch * 2);
    p.z = take(p.keep ? (size_t)n * p.pitch * 4 : 0);
    p.dx_sums = take((size_t)p.dx.splits * n * d * 4);
    p.dw_sums = take(p.dw.splits > 1 ? (size_t)p.dw.splits * whole * d * 4 : 0);
    const long slabs = ceil_div(n, DZ_ROWS), tiles = 2 * ceil_div(n, p.zt);
    p.db = take((size_t)(p.keep && slabs > tiles ? slabs : tiles) * p.pitch * 4);
  }
  p.total = at;
  return p;
}

template <class C> inline dim3 grid_of(long work, int* blocks) {
  *blocks = (int)((work + 7) / 8 * 8);
  return dim3((unsigned)*blocks);
}
template <class C> void launch_sums(const LogitArgs& g, hipStream_t st) {
  int blocks;
  const dim3 grid = grid_of<C>(g.tiles, &blocks);
  hipLaunchKernelGGL(lce_sums_kernel<C>, grid, dim3(C::THREADS), 0, st, g, blocks);
}
template <class C> void launch_dz(const LogitArgs& g, int parts, hipStream_t st) {
  int blocks;
  dim3 grid = grid_of<C>(g.tiles, &blocks);
  if (g.join) ++grid.x;
  if (parts == 3) hipLaunchKernelGGL((lce_dz_kernel<C, 3>), grid, dim3(C::THREADS), 0, st, g, blocks);
  else hipLaunchKernelGGL((lce_dz_kernel<C, 2>), grid, dim3(C::THREADS), 0, st, g, blocks);
}
template <class C> void launch_dx(const DxArgs& g, hipStream_t st) {
  int blocks;
  const dim3 grid = grid_of<C>(g.work, &blocks);
  hipLaunchKernelGGL(lce_dx_kernel<C>, grid, dim3(C::THREADS), 0, st, g, blocks);
}
template <class C> void launch_dw(const DwArgs& g, hipStream_t st) {
  int blocks;
  const dim3 grid = grid_of<C>((long)g.tiles * g.splits, &blocks);
  hipLaunchKernelGGL(lce_dw_kernel<C>, grid, dim3(C::THREADS), 0, st, g.dz, g.x, g.scale, g.out, g.n, g.d, g.cols, g.n_per_split, g.tiles_m, g.tiles, g.splits, blocks);
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
    const size_t eights = (size_t)rows * p.dp / 8;
    const unsigned blocks = (unsigned)(eights / 256 + 1 < 4096 ? eights / 256 + 1 : 4096);
    hipLaunchKernelGGL(lce_pad_kernel, dim3(blocks), dim3(256), 0, st, (const bf16_t*)in, (bf16_t*)(a.ws + at), eights, a.d, p.dp);
    return (const bf16_t*)(a.ws + at);
  };
  if (p.dp != a.d) x = pad(a.x, p.x, a.n);
  LogitArgs g{};
  g.x = GemmOperand{x, {}, a.n, p.dp, p.dp};
  g.labels = a.labels;
  g.n = a.n; g.d = p.dp;
  g.part = (float*)(a.ws + p.part); g.z_label = s.z_label; g.splits = (int)p.splits;
  g.row_max = s.row_max; g.row_rest = s.row_rest;
  for (int i = 0; i < p.parts; ++i) g.dz[i] = (bf16_t*)(a.ws + p.dz[i]);
  g.pitch = p.pitch; g.ignore = a.ignore;
  g.db_part = a.db ? (float*)(a.ws + p.db) : nullptr;
  g.tiles_m = (int)ceil_div(a.n, p.zt);
  g.join = p.join; g.classes = a.classes; g.loss_rows = s.loss_rows; g.scale = s.scale;
  auto piece = [&](long k) {
    g.v0 = (int)(k * p.piece);
    g.cols = (int)(a.classes - g.v0 < p.piece ? a.classes - g.v0 : p.piece);
    const bf16_t* w = (const bf16_t*)a.w + (size_t)g.v0 * a.d;
    if (p.dp != a.d) w = pad(w, p.w, g.cols);
    g.w = GemmOperand{w, {}, g.cols, p.dp, p.dp};
    g.bias = a.bias ? a.bias + g.v0 : nullptr;
    g.split0 = (int)(k * (p.piece / p.zt));
  };
  for (long k = 0; k < p.pieces; ++k) {
    piece(k);
    g.tiles = (int)(g.tiles_m * ceil_div(g.cols, p.zt));
    g.z = p.keep && k + 1 == p.pieces ? (float*)(a.ws + p.z) : nullptr;
    if (p.zt == 256) launch_sums<Z256>(g, st);
    else if (p.zt == 128) launch_sums<Z128>(g, st);
    else launch_sums<Z64>(g, st);
  }
  if (!p.join) {
    if (const hipError_t e = lce_join(a, s, g.part, (int)p.splits); e != hipSuccess || !grads) return e;
  }
  float* const sums = (float*)(a.ws + p.dx_sums);
  for (long k = p.pieces - 1; k >= 0; --k) {           // (the last piece is still there)
    const bool first = k + 1 == p.pieces, last = k == 0;
    if (!first) piece(k);
    const int wide = p.pieces > 1 ? (int)up(g.cols, 64) : p.pitch;        // classes of the piece that are multiplied
    int db_parts = 2 * g.tiles_m;
    if (first && p.keep) {
      const int across = (p.pitch / 8 + 255) / 256;
      db_parts = (int)ceil_div(a.n, DZ_ROWS);
      if (p.parts == 3) hipLaunchKernelGGL(lce_dz_kept_kernel<3>, dim3((unsigned)(across * db_parts)), dim3(256), 0, st, g, across);
      else hipLaunchKernelGGL(lce_dz_kept_kernel<2>, dim3((unsigned)(across * db_parts)), dim3(256), 0, st, g, across);
    } else {
      g.tiles = (int)(g.tiles_m * ceil_div(wide, p.zt));
      if (p.zt == 256) launch_dz<Z256>(g, p.parts, st);
      else if (p.zt == 128) launch_dz<Z128>(g, p.parts, st);
      else launch_dz<Z64>(g, p.parts, st);
    }
    const GemmOperand dz{g.dz[0], {g.dz[1], g.dz[2]}, a.n, p.pitch, p.pitch};
    DxArgs gx{};
    DwArgs gw{};
    const bool direct = p.together && p.dx.splits == 1;
    if (a.dx) {
      gx.dz = dz; gx.w = g.w; gx.sums = sums; gx.dx = direct ? (bf16_t*)a.dx : nullptr; gx.scale = s.scale;
      gx.n = a.n; gx.d = a.d; gx.k = wide; gx.k_per_split = p.dx.k; gx.add = first ? 0 : 1;
      gx.tiles_m = (int)ceil_div(a.n, p.dx.tile); gx.tiles = gx.tiles_m * (int)ceil_div(a.d, p.dx.tile); gx.work = gx.tiles * p.dx.splits;
    }
    float* const dw = a.dw ? a.dw + (size_t)g.v0 * a.d : nullptr;
    float* const dw_sums = (float*)(a.ws + p.dw_sums);
    if (a.dw) {
      gw.dz = dz; gw.x = g.x; gw.scale = s.scale; gw.out = p.dw.splits > 1 ? dw_sums : dw;
      gw.n = a.n; gw.d = a.d; gw.cols = g.cols; gw.n_per_split = p.dw.k;
      gw.tiles_m = (int)ceil_div(g.cols, p.dw.tile); gw.tiles = gw.tiles_m * (int)ceil_div(a.d, p.dw.tile); gw.splits = p.dw.splits;
    }
    if (!p.together && a.dx) {
      if (p.dx.tile == 256) launch_dx<X256>(gx, st);
      else if (p.dx.tile == 128) launch_dx<X128>(gx, st);
      else launch_dx<X64>(gx, st);
    }
    if (!p.together && a.dw) {
#define ACC_DW(C) launch_dw<C>(gw, st)
      if (p.parts == 3) { if (p.dw.tile == 256) ACC_DW(V256); else if (p.dw.tile == 128) ACC_DW(V128); else ACC_DW(V64); }
      else { if (p.dw.tile == 256) ACC_DW(W256); else if (p.dw.tile == 128) ACC_DW(W128); else ACC_DW(W64); }
#undef ACC_DW
    }
    Finish f{};
    f.scale = s.scale;
    if (a.dx && last && !direct) {
      f.sums = sums; f.dx = (bf16_t*)a.dx; f.count = (size_t)a.n * a.d; f.splits = p.dx.splits;
      f.dx_blocks = (int)((f.count + 1023) / 1024);
    }
    if (a.dw && p.dw.splits > 1) {
      f.dw_sums = dw_sums; f.dw = dw; f.dw_count = (size_t)g.cols * a.d; f.dw_splits = p.dw.splits;
      f.dw_blocks = (int)((f.dw_count + 1023) / 1024);
    }
    if (a.db) { f.part = g.db_part; f.db = a.db + g.v0; f.parts = db_parts; f.pitch = p.pitch; f.cols = g.cols; }
    const int db_blocks = a.db ? (g.cols + 255) / 256 : 0;
    if (p.together) {
      const int bx = (gx.work + 7) / 8 * 8, bw = (gw.tiles * gw.splits + 7) / 8 * 8;
      const MeanArgs mean{s.loss_rows, a.labels, a.loss, a.n, a.ignore};
      const dim3 grid((unsigned)(bx + bw + db_blocks + (p.join && a.loss ? 1 : 0)));
      if (p.parts == 3) hipLaunchKernelGGL((lce_grads_kernel<X64, V64>), grid, dim3(256), 0, st, gx, gw, f, mean, bx, bw, db_blocks);
      else hipLaunchKernelGGL((lce_grads_kernel<X64, W64>), grid, dim3(256), 0, st, gx, gw, f, mean, bx, bw, db_blocks);
    }
    const int blocks = f.dx_blocks + f.dw_blocks + (p.together ? 0 : db_blocks);
    if (blocks) hipLaunchKernelGGL(lce_finish_kernel, dim3((unsigned)blocks), dim3(256), 0, st, f);
  }
  return hipGetLastError();
}

}  // namespace acc
