// The products of the gated layer (glu.hip) for bf16 operands, on the bf16 matrix cores.
//
// Gate and value of the same columns are products of one tile (GemmCfg's PAIR): they meet in the same registers, where h = act(a) b, or in the backward pass,
// which works them out again, their gradients da and db, leaves them.  Those are [rows][2 f] = dz, and the rest is that of a linear layer: dx = dz w, dw = dz^T
// x.
//
// dz is kept as the sum of bf16 values, the first the nearest one, the next the nearest to what is left (relative errors of 2^-8, 2^-16, 2^-24).  dx, rounded
// to bf16 itself, is multiplied from two: one would do if its errors stayed beside the result's own rounding, but where a row of dh sums to zero, as in front
// of a normalisation, and the values are alike, what the gates' weights have in common cancels in dx and its errors do not (relative error of dx, 300 x 128 x
// 64, a common part of 10 and 30 times the weights' spread: one value 0.014 and 0.021, two 0.0017, which is the rounding of the result; nothing in common:
// 0.0023 and 0.0017; 12544 rows, 1024 to 2 x 4096, all gradients of kept projections 672 and 810 us).  dw, an fp32 result, is multiplied from three, from 10240
// rows on from two, whose errors are there at most 1.4 times those of a sum of so many terms in fp32.  Relative error of dw, 1e-7, two / three / all in fp32:
// 64 rows 24 / 1.1 / 1.5, 1500 24 / 1.7 / 7.0, 4096 25 / 5.4 / 11.8, 8192 25 / 7.3 / 16.5, 10000 25 / 8.0 / 18.1, 12544 26 / - / 20, 16384 26 / - / 23, 32768
// 25 / - / 32; all gradients of kept projections of 4096 rows, 512 wide, 2 x 1024, 65 / 76 us, of 8192, 2 x 2048, 235 / 269.
//
// All bound by the matrix cores but for the smallest, which are launches behind each other.  12544 rows, 1024 to 2 x 4096 (210 GFLOP a product), us: forward
// 204 (1030 TFLOP/s; 218 where the projections are kept), dz from the projections worked out again 320 (660: behind each tile's sums the gradients of its 65536
// values, which no other workgroup covers), dx from two values 350 (1200 TFLOP/s of both), dw from two values 300-315 (1370).  A library's product of these
// sizes alone takes 141 to 175.
#include "glu.h"

#include "gemm_bf16.h"
#include "gemm_tiles.h"

namespace acc {
namespace {

struct PairArgs {
  GemmOperand x, w;            // w.p the gate's rows, w.more[0] the value's
  const float* bias;           // [2 f], or null
  int rows, d, f, act, tiles_m, tiles;
  bf16_t *h, *ab;              // forward
  const bf16_t* dh;            // backward
  bf16_t* dz[3];
  int pitch, half;             // of dz: columns, and where the value's begin
  float* db_part;              // sums of a wave's rows
  int whole;                   // forward: tiles in one piece; those behind them (a last, short round of the compute units) in four
};

// 32 rows of COLS values of a wave by way of LDS, so that memory sees whole pieces of rows: EP bytes a staged row, PER lanes to a row.
template <int COLS_> struct Stage {
  static constexpr int COLS = COLS_, EP = COLS * 2 + 16, PER = COLS / 8, ROWS = 64 / PER, ONE = 32 * EP, PARTS = 32 / ROWS;
  v4u v[PARTS];                                        // what a lane moves of them

  __device__ __forceinline__ void from_lds(const char* stg) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int it = 0; it < PARTS; ++it) v[it] = *reinterpret_cast<const v4u*>(stg + (lane / PER + ROWS * it) * EP + 16 * (lane % PER));
  }
  __device__ __forceinline__ void to_lds(char* stg) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int it = 0; it < PARTS; ++it) *reinterpret_cast<v4u*>(stg + (lane / PER + ROWS * it) * EP + 16 * (lane % PER)) = v[it];
  }
  // To and from rows of `pitch` values (2^17 at most) at any address that bf16 values may have; columns [0, left) and rows [0, rows) exist.  Eights that are
  // whole go out here, what is left of a row's last one by ends_out() from LDS.
  typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
  __device__ __forceinline__ void out(bf16_t* to, size_t pitch, int rows, int left) const {
    const int lane = threadIdx.x & 63, c = 8 * (lane % PER);
#pragma unroll
    for (int it = 0; it < PARTS; ++it) {
      const int r = lane / PER + ROWS * it;
      if (r < rows && c + 8 <= left) *reinterpret_cast<any*>(to + ((uint32_t)r * (uint32_t)pitch + (uint32_t)c)) = any{v[it].x, v[it].y, v[it].z, v[it].w};
    }
  }
  // Rows of eight values or more: the last eight end with the row and are shifted, zeros behind them.  What lies outside is read from the last row and column
  // that exist and dropped: a branch around a load, with all accumulators alive, made the compiler spill some of them.
  __device__ __forceinline__ void in(const bf16_t* from, int pitch, int rows, int left) {
    const int lane = threadIdx.x & 63, c = 8 * (lane % PER), over = c + 8 > left ? c + 8 - left : 0;
#pragma unroll
    for (int it = 0; it < PARTS; ++it) {
      const int r = lane / PER + ROWS * it;
      const any q = *reinterpret_cast<const any*>(from + (min(r, rows - 1) * pitch + c - over));
      const bool there = r < rows && over < 8;
      v[it] = v4u{there ? q.x : 0u, there ? q.y : 0u, there ? q.z : 0u, there ? q.w : 0u};
    }
    const bool shifted = ends(left);
#pragma unroll
    for (int it = 0; it < PARTS; ++it) {
      v4u q = v[it];
      if (shifted && (over & 4)) q = v4u{q.z, q.w, 0, 0};
      if (shifted && (over & 2)) q = v4u{q.y, q.z, q.w, 0};
      if (shifted && (over & 1)) q = v4u{q.x >> 16 | q.y << 16, q.y >> 16 | q.z << 16, q.z >> 16 | q.w << 16, q.w >> 16};
      v[it] = q;
    }
  }
  static __device__ __forceinline__ bool ends(int left) { return left > 0 && left < COLS && (left & 7) != 0; }
  static __device__ __forceinline__ void ends_out(const char* stg, bf16_t* to, size_t pitch, int rows, int left) {
    const int first = left & ~7, count = left & 7;
#pragma unroll 1
    for (int i = threadIdx.x & 63; i < 32 * count; i += 64) {
      const int r = i / count, c = first + i % count;
      if (r < rows) to[r * pitch + c] = *reinterpret_cast<const bf16_t*>(stg + r * EP + 2 * c);
    }
  }
};
__device__ __forceinline__ void wave_lds_done() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#endif
}

// The accumulators one by one: as sixteen registers that must lie side by side, some of them were spilled between their uses.
template <class C> using Values = float[C::MB][C::NB][16];
template <class C> __device__ __forceinline__ void values_of(const GemmAcc<C>& acc, Values<C>& v) {
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) v[i][j][e] = acc[i][j][e];
}
// f >= 4.  Read without a branch of their own: the last four end with the row and are shifted, zeros behind them.
template <class C>
__device__ __forceinline__ void add_pair_bias(Values<C>& acc, const float* __restrict__ bias, int col0, int f) {
  typedef float any __attribute__((ext_vector_type(4), aligned(4)));
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < C::NB; ++j) {
    any b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = col0 + 32 * (j >> 1) + 8 * q + 4 * (lane >> 5);
      b[q] = *reinterpret_cast<const any*>(bias + min(n, f - 4) + (j & 1 ? f : 0));
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int n = col0 + 32 * (j >> 1) + 8 * q + 4 * (lane >> 5), over = n - min(n, f - 4);
      any v = b[q];
      if (over & 2) v = any{v.z, v.w, 0.f, 0.f};
      if (over & 1) v = any{v.y, v.z, v.w, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < C::MB; ++i) acc[i][j][4 * q + e] += over < 4 ? v[e] : 0.f;
    }
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
#endif
  }
}

// LDS of a tile: its operands, then its results, three at once of every wave
template <class C> struct TileLds {
  static constexpr int WAVE = 3 * Stage<16 * C::NB>::ONE, OUT = C::WM * C::WN * WAVE, value = C::LDS > OUT ? C::LDS : OUT;
};
// h, and the projections where they are kept, of the tile that begins at row m0 and column n0
template <class C>
__device__ __forceinline__ void glu_fwd_tile(const PairArgs& a, int m0, int n0, char* lds) {
  typedef Stage<16 * C::NB> S;
  Values<C> acc;
  m0 = __builtin_amdgcn_readfirstlane(m0);
  n0 = __builtin_amdgcn_readfirstlane(n0);
  {
    GemmAcc<C> sums;
    gemm_tile<C>(a.x, a.w, m0, n0, 0, a.d, lds, sums);
    values_of<C>(sums, acc);
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm0 = (wave / C::WN) * 32 * C::MB, col0 = n0 + (wave % C::WN) * S::COLS;
  if (a.bias) add_pair_bias<C>(acc, a.bias, col0, a.f);
  char *const stg = lds + wave * TileLds<C>::WAVE, *const mine = stg + (lane & 31) * S::EP + 8 * (lane >> 5);
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    const int m = m0 + wm0 + 32 * i, rows = a.rows - m, left = a.f - col0;
    auto put = [&](int which, auto value) {
#pragma unroll
      for (int j = 0; j < C::NB / 2; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = value(acc[i][2 * j][4 * q + e], acc[i][2 * j + 1][4 * q + e]);
          *reinterpret_cast<uint2*>(mine + which * S::ONE + 64 * j + 16 * q) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        }
    };
    put(0, [&](float g, float v) { return glu_act(a.act, g) * v; });
    if (a.ab) {
      put(1, [](float g, float) { return g; });
      put(2, [](float, float v) { return v; });
    }
    wave_lds_done();
    bf16_t *const h = a.h + (size_t)m * a.f + col0, *const ab = a.ab + (size_t)m * 2 * a.f + col0;
    S p, g, v;
    p.from_lds(stg);
    if (a.ab) {
      g.from_lds(stg + S::ONE);
      v.from_lds(stg + 2 * S::ONE);
      g.out(ab, 2 * (size_t)a.f, rows, left);
      v.out(ab + a.f, 2 * (size_t)a.f, rows, left);
    }
    p.out(h, a.f, rows, left);
    if (S::ends(left)) {
      S::ends_out(stg, h, a.f, rows, left);
      if (a.ab) {
        S::ends_out(stg + S::ONE, ab, 2 * (size_t)a.f, rows, left);
        S::ends_out(stg + 2 * S::ONE, ab + a.f, 2 * (size_t)a.f, rows, left);
      }
    }
    wave_lds_done();
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

// The projections again, which leave as dz, and the columns' sums of each 32 C::MB rows of a tile
template <class C, int PARTS>
__device__ __forceinline__ void glu_dz_tile(const PairArgs& a, int m0, int n0, char* lds) {
  typedef Stage<16 * C::NB> S;
  Values<C> acc;
  m0 = __builtin_amdgcn_readfirstlane(m0);
  n0 = __builtin_amdgcn_readfirstlane(n0);
  {
    GemmAcc<C> sums;
    gemm_tile<C>(a.x, a.w, m0, n0, 0, a.d, lds, sums);
    values_of<C>(sums, acc);
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm0 = (wave / C::WN) * 32 * C::MB, col0 = n0 + (wave % C::WN) * S::COLS;
  if (a.bias) add_pair_bias<C>(acc, a.bias, col0, a.f);
  char *const stg = lds + wave * TileLds<C>::WAVE, *const mine = stg + (lane & 31) * S::EP + 8 * (lane >> 5);
  auto ask = [&](int i) {
    const int m = m0 + wm0 + 32 * i;
    S rows;
    rows.in(a.dh + (size_t)m * a.f + col0, a.f, a.rows - m, a.f - col0);
    return rows;
  };
  S next = ask(0);                                     // (one block of rows ahead)
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    const int m = m0 + wm0 + 32 * i;
    next.to_lds(stg);
    if (i + 1 < C::MB) next = ask(i + 1);
    wave_lds_done();
    const bool there = m + (lane & 31) < a.rows;     // (a row that isn't has the bias for its projections, and a dh of zero)
#pragma unroll
    for (int j = 0; j < C::NB / 2; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint2 w = *reinterpret_cast<const uint2*>(mine + 64 * j + 16 * q);
        const float dh[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float da, db;
          glu_slopes(a.act, acc[i][2 * j][4 * q + e], acc[i][2 * j + 1][4 * q + e], dh[e], da, db);
          acc[i][2 * j][4 * q + e] = there ? da : 0.f;
          acc[i][2 * j + 1][4 * q + e] = there ? db : 0.f;
        }
#if defined(__HIP_DEVICE_COMPILE__)
        __builtin_amdgcn_sched_barrier(0);             // (four values at a time: the registers are full beside the accumulators)
#endif
      }
    wave_lds_done();
  }
  if (a.db_part) {
    float* const to = a.db_part + (size_t)((m0 + wm0) / (32 * C::MB)) * a.pitch;
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < C::MB; ++i) t += acc[i][j][v];
        t = half_sum(t);
        const int n = col0 + 32 * (j >> 1) + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
        if ((lane & 31) == 31 && n < a.half) to[n + (j & 1 ? a.half : 0)] = t;
      }
  }
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    const int m = m0 + wm0 + 32 * i;
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int j = 0; j < C::NB / 2; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float* const p = acc[i][2 * j + side];
            const uint2 w = make_uint2(pack_bf16(p[4 * q], p[4 * q + 1]), pack_bf16(p[4 * q + 2], p[4 * q + 3]));
            *reinterpret_cast<uint2*>(mine + side * S::ONE + 64 * j + 16 * q) = w;
            if (part + 1 < PARTS) {                    // what is left
              p[4 * q] -= __uint_as_float(w.x << 16);
              p[4 * q + 1] -= __uint_as_float(w.x & 0xffff0000u);
              p[4 * q + 2] -= __uint_as_float(w.y << 16);
              p[4 * q + 3] -= __uint_as_float(w.y & 0xffff0000u);
            }
          }
      wave_lds_done();
      S g, v;
      g.from_lds(stg);
      v.from_lds(stg + S::ONE);
      bf16_t* const to = a.dz[part] + (size_t)m * a.pitch + col0;
      g.out(to, a.pitch, a.rows - m, a.half - col0);                   // (whole eights)
      v.out(to + a.half, a.pitch, a.rows - m, a.half - col0);
      wave_lds_done();
    }
  }
}

// C: the tiles; Q: a quarter of one, in as many threads
template <class C, class Q, class F> __device__ __forceinline__ void each_pair_tile(const PairArgs& a, int blocks, F f) {
  const int block = blockIdx.x;
  if (block < blocks) {
    const int at = (block & 7) * (blocks >> 3) + (block >> 3);
    if (at >= a.whole) return;
    const TileAt where = tile_at(at, a.tiles_m, a.tiles);
    f(C(), where.m * C::BM, where.n * (C::BN / 2));
  } else {
    const int rest = (int)gridDim.x - blocks, in = block - blocks, sub = (in & 7) * (rest >> 3) + (in >> 3), at = a.whole + (sub >> 2);
    if (at >= a.tiles) return;
    const TileAt where = tile_at(at, a.tiles_m, a.tiles);
    const int m0 = where.m * C::BM + (sub & 1) * Q::BM, n0 = where.n * (C::BN / 2) + ((sub >> 1) & 1) * (Q::BN / 2);
    if (m0 < a.rows && n0 < a.half) f(Q(), m0, n0);
  }
}
template <class C, class Q>
__global__ __launch_bounds__(C::THREADS, 2) void glu_fwd_kernel(PairArgs a, int blocks) {
  static_assert(C::THREADS == Q::THREADS, "one shape of workgroups");
  __shared__ __attribute__((aligned(1024))) char lds[TileLds<C>::value > TileLds<Q>::value ? TileLds<C>::value : TileLds<Q>::value];
  each_pair_tile<C, Q>(a, blocks, [&](auto c, int m0, int n0) { glu_fwd_tile<decltype(c)>(a, m0, n0, lds); });
}
template <class C, int PARTS>
__global__ __launch_bounds__(C::THREADS, 2) void glu_dz_kernel(PairArgs a, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[TileLds<C>::value];
  const int at = xcd_tile(blocks);
  if (at >= a.tiles) return;
  const TileAt where = tile_at(at, a.tiles_m, a.tiles);
  glu_dz_tile<C, PARTS>(a, where.m * C::BM, where.n * (C::BN / 2), lds);
}

// out[split][rows][cols] = A B over the split's k, fp32, or rounded to bf16 where there is one split
struct ProductArgs {
  GemmOperand a, b;
  float* sums;
  bf16_t* out;                 // not null: here
  int rows, cols, k, k_per_split, tiles_m, tiles, work;
};
template <class C>
__device__ __forceinline__ void glu_product(const ProductArgs& a, int work, char* lds) {
  static_assert(C::SWAP, "four columns of a row to a lane");
  const int split = work / a.tiles;
  const TileAt where = tile_at(work - split * a.tiles, a.tiles_m, a.tiles);
  const int m0 = where.m * C::BM, n0 = where.n * C::BN;
  GemmAcc<C> acc;
  gemm_tile<C>(a.a, a.b, m0, n0, split * a.k_per_split, min(a.k, (split + 1) * a.k_per_split), lds, acc);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
  if (a.out) {                                         // (whole pieces of rows: 15 us less than four values of a lane as they are, of 41379 x 1056 x 136)
    typedef Stage<32 * C::NB> S;
    static_assert(C::WM * C::WN * S::ONE <= C::LDS, "the results' rows fit the operands' place");
    char* const stg = lds + wave * S::ONE;
    const int n = n0 + wn0, left = a.cols - n;
#pragma unroll
    for (int i = 0; i < C::MB; ++i) {
      const int m = m0 + wm0 + 32 * i;
#pragma unroll
      for (int j = 0; j < C::NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint2*>(stg + (lane & 31) * S::EP + 8 * (lane >> 5) + 64 * j + 16 * q) =
              make_uint2(pack_bf16(acc[i][j][4 * q], acc[i][j][4 * q + 1]), pack_bf16(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
      wave_lds_done();
      S rows;
      rows.from_lds(stg);
      bf16_t* const to = a.out + (size_t)m * a.cols + n;
      rows.out(to, a.cols, a.rows - m, left);
      if (S::ends(left)) S::ends_out(stg, to, a.cols, a.rows - m, left);
      wave_lds_done();
    }
    return;
  }
  const bool whole = (a.cols & 7) == 0;
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    const int m = m0 + wm0 + 32 * i + (lane & 31);
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn0 + 32 * j + 8 * q + 4 * (lane >> 5);
        if (m >= a.rows || n >= a.cols) continue;
        const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        float* const o = a.sums + (size_t)split * a.rows * a.cols + (size_t)m * a.cols + n;
        if (whole) { *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]); continue; }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < a.cols) o[e] = v[e];
      }
  }
}
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void glu_product_kernel(ProductArgs a, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work < a.work) glu_product<C>(a, work, lds);
}

// dw[column of dz][d] = sum over the split's rows of dz x, dz as the sum of its parts
struct GluDwArgs {
  GemmOperand dz, x;
  float* out;                  // [split][2 f][d]
  int rows, d, f, half, per_split, tiles_m, tiles, work;
};
template <class C>
__device__ __forceinline__ void glu_dw(const GluDwArgs& a, int work, char* lds) {
  const int split = work / a.tiles;
  const TileAt where = tile_at(work - split * a.tiles, a.tiles_m, a.tiles);
  const int m0 = where.m * C::BM, n0 = where.n * C::BN, first = split * a.per_split, count = min(a.per_split, a.rows - first);
  // (from the split's first row on: its rows take fewer than 4 GiB)
  GemmOperand dz = a.dz, x = a.x;
  dz.p = static_cast<const bf16_t*>(dz.p) + (size_t)first * dz.pitch;
#pragma unroll
  for (int p = 0; p + 1 < C::PARTS; ++p) dz.more[p] = static_cast<const bf16_t*>(dz.more[p]) + (size_t)first * dz.pitch;
  x.p = static_cast<const bf16_t*>(x.p) + (size_t)first * x.pitch;
  dz.rows = x.rows = count;
  GemmAcc<C> acc;
  gemm_tile<C>(dz, x, m0, n0, 0, count, lds, acc);
  float* const out = a.out + (size_t)split * 2 * a.f * a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm0 = (wave / C::WN) * 32 * C::MB, wn0 = (wave % C::WN) * 32 * C::NB;
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j) {
      const int col = n0 + wn0 + 32 * j + (lane & 31);
      if (col >= a.d) continue;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int m = m0 + wm0 + 32 * i + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), side = m >= a.half ? 1 : 0, r = m - side * a.half;
        if (r < a.f) out[(size_t)(r + side * a.f) * a.d + col] = acc[i][j][v];
      }
    }
}
template <class C>
__global__ __launch_bounds__(C::THREADS, 2) void glu_dw_kernel(GluDwArgs a, int blocks) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work < a.work) glu_dw<C>(a, work, lds);
}
// dx, dw and db in one launch where there are few tiles: they all wait for dz only
template <class CX, class CW>
__global__ __launch_bounds__(256, 2) void glu_grads_kernel(ProductArgs x, GluDwArgs w, GluFinish f, int x_blocks, int w_blocks) {
  static_assert(CX::THREADS == 256 && CW::THREADS == 256, "one shape of workgroups");
  __shared__ __attribute__((aligned(1024))) char lds[CX::LDS > CW::LDS ? CX::LDS : CW::LDS];
  const int block = blockIdx.x;                        // (each part begins at a multiple of eight)
  if (block < x_blocks) {
    const int work = (block & 7) * (x_blocks >> 3) + (block >> 3);
    if (work < x.work) glu_product<CX>(x, work, lds);
  } else if (block < x_blocks + w_blocks) {
    const int work = (block & 7) * (w_blocks >> 3) + ((block - x_blocks) >> 3);
    if (work < w.work) glu_dw<CW>(w, work, lds);
  } else {
    glu_db(f, block - x_blocks - w_blocks);
  }
}

// out[r][0 .. pitch) = in[r][0 .. cols), then zeros; of 2 * split_row rows the second half goes to row r + gap, the `gap` rows before it and behind it are
// zero.  Eight values per thread, read at any address.
__global__ __launch_bounds__(256) void glu_pad_kernel(const bf16_t* __restrict__ in, bf16_t* __restrict__ out, size_t eights, int cols, int pitch, int split_row, int gap) {
  typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
  const size_t across = pitch / 8;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < eights; i += (size_t)gridDim.x * 256) {
    const size_t to = i / across;
    const int c = (int)(i - to * across) * 8;
    const bool between = to >= (size_t)split_row && to < (size_t)split_row + gap;
    const size_t r = to < (size_t)split_row ? to : to - gap;
    const bf16_t* from = in + r * cols + c;
    v4u v = {0, 0, 0, 0};
    if (between || r >= 2 * (size_t)split_row) {       // (between the two and behind them)
    } else if (c + 8 <= cols) {
      const any q = *reinterpret_cast<const any*>(from);
      v = v4u{q.x, q.y, q.z, q.w};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = (c + 2 * e < cols ? (uint32_t)from[2 * e] : 0u) | (c + 2 * e + 1 < cols ? (uint32_t)from[2 * e + 1] << 16 : 0u);
    }
    *reinterpret_cast<v4u*>(out + i * 8) = v;
  }
}

//                WM WN MB NB BK NS   AT     BT  PARTS SWAP  PAIR
typedef GemmCfg<4, 2, 2, 4, 64, 2, false, false, 1, true, true> G256;      // gate and value
typedef GemmCfg<4, 2, 1, 2, 64, 3, false, false, 1, true, true> G256Q;     // a quarter of that
typedef GemmCfg<2, 2, 4, 2, 32, 3, false, false, 1, true, true> G256N;     // 256 x 128: two workgroups a compute unit
typedef GemmCfg<2, 2, 2, 2, 64, 2, false, false, 1, true, true> G128;
typedef GemmCfg<2, 1, 1, 2, 64, 3, false, false, 1, true, true> G64;
typedef GemmCfg<2, 2, 2, 2, 64, 2, false, false, 1, true> S128;            // projections in parts
typedef GemmCfg<2, 2, 1, 1, 64, 4, false, false, 1, true> S64;
typedef GemmCfg<2, 4, 4, 2, 32, 3, false, true, 2, true> X256;             // dx
typedef GemmCfg<2, 2, 2, 2, 32, 3, false, true, 2, true> X128;
typedef GemmCfg<2, 2, 1, 1, 32, 4, false, true, 2, true> X64;
typedef GemmCfg<2, 4, 4, 2, 32, 3, true, true, 2, false> W256;             // dw
typedef GemmCfg<2, 2, 2, 2, 32, 2, true, true, 2, false> W128;
typedef GemmCfg<2, 2, 1, 1, 32, 4, true, true, 2, false> W64;
typedef GemmCfg<2, 4, 4, 2, 32, 2, true, true, 3, false> V256;             // dw with three parts of dz
typedef GemmCfg<2, 2, 2, 2, 32, 2, true, true, 3, false> V128;
typedef GemmCfg<2, 2, 1, 1, 32, 3, true, true, 3, false> V64;

// Which tile of gate and value, by predicted time as in gemm_tiles.h.  Constants from sixty sizes (rows 32 to 30000, widths 32 to 4096 and 6000), every tile on
// each.
struct PairTile {
  int m, n, db_rows;           // n: columns of both together; rows of a wave
  bool alone;                  // one workgroup a compute unit
  TileCost cost[2];            // forward, backward
};
constexpr PairTile kPair[4] = {{256, 256, 64, true, {{6.0, 1.2, 7.7, 1.86}, {22.7, 1.27, 30.3, 1.7}}},
                               {256, 128, 128, false, {{4.0, 1.2, 4.0, 1.0}, {14.5, 1.2, 10.9, 0.92}}},
                               {128, 128, 64, false, {{0.1, 0.79, 2.2, 0.5}, {9.9, 0.84, 7.4, 0.5}}},
                               {64, 64, 32, false, {{1.3, 0.24, 0.85, 0.225}, {5.6, 0.42, 1.8, 0.12}}}};
// Tiles in one piece, forward: those of whole rounds of the compute units, where what is left is half a round at most.  us, without quarters / with: 12544
// rows, 1024 to 2 x 4096 (6.1 rounds) 219 / 206, 8449, 1024 to 2 x 1040 (1.2) 52 / 43, 4161, 1536 to 2 x 2200 (1.2) 73 / 60.
long pair_whole(const PairTile& t, long tiles) {
  const long rest = tiles % 256;
  return t.alone && tiles > 256 && rest <= 128 ? tiles - rest : tiles;
}
double pair_us(const PairTile& t, bool backward, long tiles, double steps) {
  const TileCost& c = t.cost[backward];
  const double first = c.first + c.first_step * steps, next = c.next + c.next_step * steps;
  if (t.alone) {
    const long whole = backward ? tiles : pair_whole(t, tiles);
    return 3.0 + first + (ceil_div(whole, 256) - 1) * next + ceil_div(4 * (tiles - whole), 256) * 0.35 * next;
  }
  const long most = ceil_div(tiles, 256);
  auto round = [&](long r) { return r == 0 ? 0.0 : first > r * next ? first : r * next; };
  return 3.0 + (most / 2) * round(2) + round(most % 2);
}

constexpr double kSaved = 3.0;         // us: a launch that adds parts

struct GluPlan16 {
  int dp, fp;                  // widths as they are multiplied, multiples of 8
  bool pad_x, pad_w;
  int parts;                   // bf16 values that dz is the sum of
  PairTile tile;               // of gate and value together
  bool cut;                    // the projections' sums in parts, and what follows value by value
  Choice proj, dx, dw;
  bool together;               // dx and dw in one launch of 64 x 64 tiles
  int db_parts;
  size_t x, w, sums, dz[3], dx_sums, dw_sums, db, slabs, total;
};

GluPlan16 glu_plan16(int rows, int d, int f, bool backward, bool kept) {
  GluPlan16 p{};
  p.dp = (int)up(d, 8);
  p.fp = (int)up(f, 8);
  p.pad_x = p.dp != d;
  p.parts = rows < 10240 ? 3 : 2;
  const long wide = 2L * p.fp;
  double us = 0;
  for (const PairTile& t : kPair) {
    const double v = pair_us(t, backward, ceil_div(rows, t.m) * ceil_div(p.fp, t.n / 2), p.dp / 64.0);
    if (us == 0 || v < us) { us = v; p.tile = t; }
  }
  // few tiles of a long sum: parts of it, whose sums a second launch adds up (us, so / whole: forward 64 x 4096 x 1024 13.3 / 18.7, 1000 x 4096 x 64 12.6 /
  // 18.9; backward 43 / 49, 32 / 40)
  p.proj = choose(RowsByRows, rows, wide, p.dp, 1, 1L << 24, p.dp > 2048 ? up(ceil_div(p.dp, 16), 64) : 128, 1);       // (sixteen parts at most)
  // (and rows of fewer than eight values, which the pair's tiles do not read)
  p.cut = !kept && ((p.proj.splits > 1 && p.proj.us + (backward ? 7.0 : 2.0) < us) || f < 8);
  // (the pair's tiles take gate and value from where they lie; a product over both, or over their rows, wants each half a multiple of eight)
  p.pad_w = p.pad_x || (p.fp != f && (backward || p.cut));
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.x = take(p.pad_x ? (size_t)rows * p.dp * 2 : 0);
  p.w = take(p.pad_w ? (size_t)wide * p.dp * 2 : 0);
  p.sums = take(p.cut ? (size_t)p.proj.splits * rows * wide * 4 : 0);
  if (backward) {
    p.dx = choose(ByColumns, rows, d, wide, 2, 1L << 25, 256);
    p.dw = choose(ByColumns, wide, d, rows, p.parts, 1L << 25, 128);
    const Choice dx = choose(ByColumns, rows, d, wide, 2, 1L << 25, 256, 2), dw = choose(ByColumns, wide, d, rows, p.parts, 1L << 25, 128, 2);      // 64 x 64
    const long tx = ceil_div(d, 64) * ceil_div(rows, 64), tw = ceil_div(d, 64) * ceil_div(wide, 64);
    // (whole sums save the launch that adds parts)
    const Choice x1 = choose(ByColumns, rows, d, wide, 2, 0, 256, 2), w1 = choose(ByColumns, wide, d, rows, p.parts, 0, 128, 2);
    const bool sums = !(x1.us < dx.us + kSaved && w1.us < dw.us + kSaved);
    const Choice &cx = sums ? dx : x1, &cw = sums ? dw : w1;
    // Up to 1024 workgroups, or 2048 of few steps: 64 x 64 tiles take twice the LDS reads of larger ones.  (us, all gradients of kept projections, so / each
    // for itself: 196 x 512 x 1024 18.0 / 22.6, 4096 x 512 x 1024 76 / 79, 3867 x 304 x 1936 121 / 130, 5000 x 768 x 1024 125 / 107, 10000 x 512 x 1024 185 /
    // 192, 8192 x 512 x 2048 334 / 269)
    const long workgroups = tx * cx.splits + tw * cw.splits, steps = tx * ceil_div(wide, 64) * 2 + tw * ceil_div(rows, 64) * p.parts;
    p.together = workgroups <= 1024 || (workgroups <= 2048 && steps <= 420 * 256);
    if (p.together) { p.dx = cx; p.dw = cw; }
    // rows of a part of dw: fewer than 4 GiB of dz and of x
    const long most = (0xF0000000L / (2 * (wide > p.dp ? wide : p.dp))) / 64 * 64;
    if (p.dw.k > most) {
      p.dw.k = (int)most;
      p.dw.splits = (int)ceil_div(rows, most);
    }
    for (int i = 0; i < p.parts; ++i) p.dz[i] = take((size_t)rows * wide * 2);
    p.dx_sums = take(p.dx.splits > 1 ? (size_t)p.dx.splits * rows * d * 4 : 0);
    p.dw_sums = take(p.dw.splits > 1 ? (size_t)p.dw.splits * 2 * f * d * 4 : 0);
    PointArgs q{};
    q.rows = rows; q.f = f;
    p.db_parts = kept || p.cut ? glu_point_shape(q, DT_BF16) : (int)ceil_div(rows, p.tile.db_rows);
    p.db = take((size_t)(kept || p.cut ? p.db_parts : up(rows, p.tile.m) / p.tile.db_rows) * wide * 4);
    p.slabs = take(p.db_parts > kDbMany ? (size_t)kDbSlabs * wide * 4 : 0);
  }
  p.total = at;
  return p;
}

unsigned whole_eights16(long work) { return (unsigned)((work + 7) / 8 * 8); }

template <class C, class Q> void launch_pair(const PairArgs& g, bool backward, int parts, hipStream_t st) {
  const unsigned blocks = whole_eights16(backward ? g.tiles : g.whole), grid = blocks + whole_eights16(4L * (g.tiles - g.whole));
  if (!backward) hipLaunchKernelGGL((glu_fwd_kernel<C, Q>), dim3(grid), dim3(C::THREADS), 0, st, g, (int)blocks);
  else if (parts == 3) hipLaunchKernelGGL((glu_dz_kernel<C, 3>), dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
  else if (parts == 0) hipLaunchKernelGGL((glu_dz_kernel<C, 0>), dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
  else hipLaunchKernelGGL((glu_dz_kernel<C, 2>), dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
}
template <class C> void launch_product(const ProductArgs& g, hipStream_t st) {
  const unsigned blocks = whole_eights16(g.work);
  hipLaunchKernelGGL(glu_product_kernel<C>, dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
}
template <class C> void launch_dw(const GluDwArgs& g, hipStream_t st) {
  const unsigned blocks = whole_eights16(g.work);
  hipLaunchKernelGGL(glu_dw_kernel<C>, dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
}

}  // namespace

size_t glu_bf16_workspace_bytes(int rows, int d, int f, bool backward) {
  const size_t again = glu_plan16(rows, d, f, backward, false).total, kept = backward ? glu_plan16(rows, d, f, true, true).total : 0;
  return again > kept ? again : kept;
}

hipError_t glu_bf16(const GluArgs& a, bool backward) {
  const bool kept = backward && a.ab_in;
  const GluPlan16 p = glu_plan16(a.rows, a.d, a.f, backward, kept);
  hipStream_t st = a.st;
  const bf16_t *x = (const bf16_t*)a.x, *w = (const bf16_t*)a.w;
  auto pad = [&](const bf16_t* in, size_t at, long rows_out, int split_row, int gap) {
    const size_t eights = (size_t)rows_out * p.dp / 8;
    const unsigned blocks = (unsigned)(eights / 256 + 1 < 4096 ? eights / 256 + 1 : 4096);
    hipLaunchKernelGGL(glu_pad_kernel, dim3(blocks), dim3(256), 0, st, in, (bf16_t*)(a.ws + at), eights, a.d, p.dp, split_row, gap);
    return (const bf16_t*)(a.ws + at);
  };
  if (p.pad_x && (!kept || a.dw)) x = pad(x, p.x, a.rows, a.rows, 0);
  if (p.pad_w && (!kept || a.dx)) w = pad(w, p.w, 2L * p.fp, a.f, p.fp - a.f);
  const int wide = 2 * p.fp;
  bf16_t* dz[3] = {(bf16_t*)(a.ws + p.dz[0]), (bf16_t*)(a.ws + p.dz[1]), (bf16_t*)(a.ws + p.dz[2])};
  float* const db_part = backward && a.db ? (float*)(a.ws + p.db) : nullptr;
  const int parts = a.dw ? p.parts : a.dx ? 2 : 0;     // values of dz that something is multiplied from
  if (kept || p.cut) {
    PointArgs q{};
    q.ab_in = a.ab_in; q.dh = a.dh; q.h = a.h; q.ab = a.ab;
    q.rows = a.rows; q.f = a.f; q.act = a.act; q.half = p.fp; q.pitch = wide;
    for (int i = 0; i < 3; ++i) q.dz[i] = dz[i];
    q.db_part = db_part;
    if (!kept) {
      ProductArgs g{};
      g.a = GemmOperand{x, {}, a.rows, p.dp, p.dp};
      g.b = GemmOperand{w, {}, wide, p.dp, p.dp};
      g.sums = (float*)(a.ws + p.sums);
      g.rows = a.rows; g.cols = wide; g.k = p.dp; g.k_per_split = p.proj.k;
      g.tiles_m = (int)ceil_div(a.rows, p.proj.tile); g.tiles = g.tiles_m * (int)ceil_div(wide, p.proj.tile); g.work = g.tiles * p.proj.splits;
      if (p.proj.tile == 128) launch_product<S128>(g, st);
      else launch_product<S64>(g, st);
      q.sums = g.sums; q.splits = p.proj.splits; q.bias = a.bias;
    }
    glu_point_shape(q, DT_BF16);
    if (const hipError_t e = glu_point(q, backward, parts, DT_BF16, st); e != hipSuccess || !backward) return e;
  } else {
    PairArgs g{};
    g.x = GemmOperand{x, {}, a.rows, p.dp, p.dp};
    g.w = GemmOperand{w, {w + (size_t)(p.pad_w ? p.fp : a.f) * p.dp}, a.f, p.dp, p.dp};
    g.bias = a.bias;
    g.rows = a.rows; g.d = p.dp; g.f = a.f; g.act = a.act;
    g.tiles_m = (int)ceil_div(a.rows, p.tile.m); g.tiles = g.tiles_m * (int)ceil_div(p.fp, p.tile.n / 2);
    g.whole = (int)pair_whole(p.tile, g.tiles);
    g.h = (bf16_t*)a.h; g.ab = (bf16_t*)a.ab; g.dh = (const bf16_t*)a.dh;
    for (int i = 0; i < 3; ++i) g.dz[i] = dz[i];
    g.pitch = wide; g.half = p.fp; g.db_part = db_part;
    if (p.tile.m == 256 && p.tile.n == 256) launch_pair<G256, G256Q>(g, backward, parts, st);
    else if (p.tile.m == 256) launch_pair<G256N, G256N>(g, backward, parts, st);
    else if (p.tile.m == 128) launch_pair<G128, G128>(g, backward, parts, st);
    else launch_pair<G64, G64>(g, backward, parts, st);
    if (!backward) return hipGetLastError();
  }
  const GemmOperand z{dz[0], {dz[1], dz[2]}, a.rows, wide, wide};
  ProductArgs gx{};
  GluDwArgs gw{};
  GluFinish f{};
  if (a.dx) {
    gx.a = z;
    gx.b = GemmOperand{w, {}, wide, p.dp, p.dp};
    gx.sums = (float*)(a.ws + p.dx_sums); gx.out = p.dx.splits > 1 ? nullptr : (bf16_t*)a.dx;
    gx.rows = a.rows; gx.cols = a.d; gx.k = wide; gx.k_per_split = p.dx.k;
    gx.tiles_m = (int)ceil_div(a.rows, p.dx.tile); gx.tiles = gx.tiles_m * (int)ceil_div(a.d, p.dx.tile); gx.work = gx.tiles * p.dx.splits;
    if (p.dx.splits > 1) { f.dx_sums = gx.sums; f.dx = a.dx; f.dx_count = (size_t)a.rows * a.d; f.dx_splits = p.dx.splits; }
  }
  if (a.dw) {
    gw.dz = z;
    gw.x = GemmOperand{x, {}, a.rows, p.dp, p.dp};
    gw.out = p.dw.splits > 1 ? (float*)(a.ws + p.dw_sums) : a.dw;
    gw.rows = a.rows; gw.d = a.d; gw.f = a.f; gw.half = p.fp; gw.per_split = p.dw.k;
    gw.tiles_m = (int)ceil_div(wide, p.dw.tile); gw.tiles = gw.tiles_m * (int)ceil_div(a.d, p.dw.tile); gw.work = gw.tiles * p.dw.splits;
    if (p.dw.splits > 1) { f.dw_sums = gw.out; f.dw = a.dw; f.dw_count = 2 * (size_t)a.f * a.d; f.dw_splits = p.dw.splits; }
  }
  if (a.db) { f.db_part = db_part; f.db = a.db; f.db_parts = p.db_parts; f.pitch = wide; f.half = p.fp; f.f = a.f; }
  if (const hipError_t e = glu_db_slabs(f, (float*)(a.ws + p.slabs), st); e != hipSuccess) return e;
  if (p.together) {
    const unsigned bx = whole_eights16(gx.work), bw = whole_eights16(gw.work);
    const dim3 grid(bx + bw + glu_db_blocks(f));
    if (p.parts == 3) hipLaunchKernelGGL((glu_grads_kernel<X64, V64>), grid, dim3(256), 0, st, gx, gw, f, (int)bx, (int)bw);
    else hipLaunchKernelGGL((glu_grads_kernel<X64, W64>), grid, dim3(256), 0, st, gx, gw, f, (int)bx, (int)bw);
  } else {
    if (a.dx) {
      if (p.dx.tile == 256) launch_product<X256>(gx, st);
      else if (p.dx.tile == 128) launch_product<X128>(gx, st);
      else launch_product<X64>(gx, st);
    }
    if (a.dw) {
      if (p.parts == 3) { if (p.dw.tile == 256) launch_dw<V256>(gw, st); else if (p.dw.tile == 128) launch_dw<V128>(gw, st); else launch_dw<V64>(gw, st); }
      else { if (p.dw.tile == 256) launch_dw<W256>(gw, st); else if (p.dw.tile == 128) launch_dw<W128>(gw, st); else launch_dw<W64>(gw, st); }
    }
  }
  return glu_finish(f, !p.together, DT_BF16, st);
}

}  // namespace acc
