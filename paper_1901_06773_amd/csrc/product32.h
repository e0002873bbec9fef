// Whole products of fp32 operands by the tiles of gemm_f32.h, the sum over k in parts where there are few tiles, and what adds the parts.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>

#include "dtype.h"
#include "gemm_f32.h"
#include "gemm_tiles.h"

namespace acc {

// out[split][m][n] (+)= A B over the split's values of k
struct Product32 {
  Gemm32Operand a, b;
  float* out;
  int k, k_per_split, add, tiles_m, tiles, work;
};
template <class C>
__device__ __forceinline__ void product32(const Product32& a, int work, float* lds) {
  const int split = work / a.tiles;
  const TileAt where = tile_at(work - split * a.tiles, a.tiles_m, a.tiles);
  const int rows = a.a.extent, cols = a.b.extent, m0 = where.m * C::BM, n0 = where.n * C::BN;
  Gemm32Acc<C> acc;
  gemm32_tile<C>(a.a, a.b, m0, n0, split * a.k_per_split, min(a.k, (split + 1) * a.k_per_split), lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row0 = m0 + (wave / C::WN) * 16 * C::MB + (lane & 15), col0 = n0 + (wave % C::WN) * 16 * C::NB + 4 * (lane >> 4);
  float* const out = a.out + (size_t)split * rows * cols;
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j) {
      const int m = row0 + 16 * i, c = col0 + 16 * j;
      if (m >= rows || c >= cols) continue;
      float* const to = out + (size_t)m * cols + c;
      if (c + 4 <= cols) {
        f32x4 v = acc[i][j];
        if (a.add) v += *reinterpret_cast<const f32x4_any*>(to);
        *reinterpret_cast<f32x4_any*>(to) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (c + e < cols) to[e] = a.add ? to[e] + acc[i][j][e] : acc[i][j][e];
      }
    }
}
template <class C>
__global__ __launch_bounds__(C::THREADS) void product32_kernel(Product32 a, int blocks) {
  __shared__ __attribute__((aligned(16))) float lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work < a.work) product32<C>(a, work, lds);
}

// 1024 values of a workgroup at a time; 2^20 workgroups at most, as a launch has fewer than 2^32 threads
inline unsigned join_blocks(size_t count) { const size_t b = (count + 1023) / 1024; return (unsigned)(b < 1u << 20 ? b : 1u << 20); }
template <class T>
__device__ __forceinline__ void join_sums(const float* __restrict__ sums, T* __restrict__ out, size_t count, int splits, size_t block, size_t blocks) {
  for (; block * 1024 < count; block += blocks)
    for (size_t i = block * 1024 + threadIdx.x; i < count && i < (block + 1) * 1024; i += 256) {
      float s = sums[i];
      int k = 1;
      for (; k + 8 <= splits; k += 8) {
        float q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) q[u] = sums[(k + u) * count + i];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += q[u];
      }
      for (; k < splits; ++k) s += sums[k * count + i];
      Elem<T>::store(out + i, s);
    }
}
// Tiles and, for a product whose sum over k may be cut, parts of 128 values of k or more.  Predicted time, us: the chunks of a tile one after the other,
// or all chunks of the busiest compute unit at the rate that its workgroups reach together; the sums of the parts cost writing and reading.  Constants from
// every tile on ten shapes (16 to 3835 rows); measured, 32 x 128 / 64 x 64 / 128 x 128 (split): logits 16 x 816 x 16719 27 / 39 / 60, 1024 x 1024 x 8192
// 180 / 171 / 104; dx 666 x 57 x 55313 177 / 85 / 82, 2520 x 304 x 14775 588 / 287 / 166; dw 344 x 816 x 63060 434 / 389 / 251.
struct Cut {
  int tile, splits, k;           // tile: 0 32 x 128, 1 64 x 64, 2 128 x 128; k: values of it in one part
  double us;                     // predicted
};
inline constexpr int kTile32[3][2] = {{32, 128}, {64, 64}, {128, 128}};
inline constexpr double kChunk32[3][2] = {{0.93, 0.68}, {0.88, 0.66}, {2.1, 1.4}};
inline Cut cut32(long m, long n, long k, long most_sums, int only = -1) {
  Cut best{1, 1, (int)up(k, 32), 0.0};
  double us = 0;
  for (int t = only < 0 ? 0 : only; t < (only < 0 ? 3 : only + 1); ++t) {
    const long tiles = ceil_div(m, kTile32[t][0]) * ceil_div(n, kTile32[t][1]);
    for (int i = 0; i < 10; ++i) {
      const long s = i < 7 ? 1L << i : (256L << (i - 7)) / tiles;
      if (s < 1) continue;
      const long each = up(ceil_div(k, s), 32), splits = ceil_div(k, each);
      if (s > 1 && (each < 128 || splits * m * n > most_sums)) continue;
      const double one = each / 32.0 * kChunk32[t][0], all = ceil_div(tiles * splits, 256) * (each / 32.0) * kChunk32[t][1];
      const double v = (one > all ? one : all) + (splits > 1 ? (only < 0 ? 2.0 : 5.0) + 0.15 * splits + (double)splits * m * n * 8 / 5e6 : 0.0);
      if (us == 0 || v < us) {
        us = v;
        best = Cut{t, (int)splits, (int)each, v};
      }
    }
  }
  return best;
}

inline unsigned whole_eights(long work) { return (unsigned)((work + 7) / 8 * 8); }

inline void cut_into(Product32& g, const Cut& c) {
  g.tiles_m = (int)ceil_div(g.a.extent, kTile32[c.tile][0]);
  g.tiles = g.tiles_m * (int)ceil_div(g.b.extent, kTile32[c.tile][1]);
  g.k_per_split = c.k;
  g.work = g.tiles * c.splits;
}
template <bool AT, bool BT> hipError_t launch_product32(const Product32& g, const Cut& c, hipStream_t st) {
  const unsigned blocks = whole_eights(g.work);
  if (c.tile == 0) hipLaunchKernelGGL((product32_kernel<Gemm32Cfg<1, 4, 2, 2, AT, BT, false>>), dim3(blocks), dim3(256), 0, st, g, (int)blocks);
  else if (c.tile == 1) hipLaunchKernelGGL((product32_kernel<Gemm32Cfg<2, 2, 2, 2, AT, BT, false>>), dim3(blocks), dim3(256), 0, st, g, (int)blocks);
  else hipLaunchKernelGGL((product32_kernel<Gemm32Cfg<2, 2, 4, 4, AT, BT, true>>), dim3(blocks), dim3(256), 0, st, g, (int)blocks);
  return hipGetLastError();
}

}  // namespace acc
