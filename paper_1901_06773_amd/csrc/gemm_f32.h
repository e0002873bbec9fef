// One tile of a plain matrix product of fp32 operands, for kernels that do something of their own with it:
//
//   acc[m][n] = sum_k A[m][k] * B[k][n],   m in [m0, m0 + BM), n in [n0, n0 + BN), k in [k_lo, k_hi)
//
// Each operand lies in memory with its values of k side by side (rows of m resp. n) or with its values of m resp. n side by side (rows of k), at any
// width: 16 bytes at a time from addresses that need be aligned to 4 only, so odd widths cost no copy.  Loads that would pass the end of a row begin
// earlier and are shifted; rows that don't exist repeat the last one, whose results nobody stores, and values of k beyond k_hi are zero in both operands.
// A chunk of 32 values of k waits in registers while the one before it is multiplied out of LDS; one stage of LDS leaves room for two workgroups and more
// on a compute unit, which cover each other's barriers.
//
// Small tiles multiply on the fp32 matrix cores (256 operations per cycle and compute unit; LDS traffic a tenth of that).  Large ones (SPLIT) write each
// value to LDS as the sum of three bf16 values, which hold its 24 bits, and add the six products that matter on the bf16 matrix cores: a chunk of 128 x 128
// takes them 1536 cycles in place of 4096, beside some 800 of splitting.  1024 x 2048 x 32768, us, all in fp32 / split: 1134 / 686 (200 TFLOP/s).
// The three products left out are at most 2^-21 of the whole one together, 2.3e-8 of a sum of 2048 (whose fp32 roundings are 3.5e-7).  An infinity has no such
// sum (what is left of it is NaN, and so are its products), and of values below 2^-110 the last parts fall under the smallest bf16 value: they are held to
// 2^-134, not to 24 bits.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "dtype.h"

namespace acc {

// WM x WN waves, each MB x NB blocks of 16 x 16.  AT / BT: the operand lies in rows of k.  SPLIT: products on the bf16 matrix cores.  PAIR: B is two matrices
// of the same sizes (`second` floats apart); blocks of 16 of their rows take turns, so that block 2 j + 1 of a wave holds the second matrix's products of the
// columns that its block 2 j holds the first one's of: n0 and BN / 2 columns of each.
template <int WM_, int WN_, int MB_, int NB_, bool AT_, bool BT_, bool SPLIT_, bool PAIR_ = false> struct Gemm32Cfg {
  static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, BK = 32;
  static constexpr bool AT = AT_, BT = BT_, SPLIT = SPLIT_, PAIR = PAIR_;
  static_assert(!PAIR_ || (!BT_ && NB_ % 2 == 0), "rows of k side by side, whole pairs");
  static constexpr int THREADS = 64 * WM * WN, BM = 16 * MB * WM, BN = 16 * NB * WN;
  static constexpr int SPLIT_PITCH = 20;               // a row's 32 bf16 values, and 16 bytes that set the next row off
  // floats between staged rows: the sixteen rows (resp. four groups of sixteen columns) that a read takes at once fall on different banks
  static constexpr int A_PITCH = AT ? BM + 4 : BK + 4, B_PITCH = BT ? BN + 4 : BK + 4;
  static constexpr int A_FLOATS = SPLIT ? 3 * BM * SPLIT_PITCH : (AT ? BK : BM) * A_PITCH, B_FLOATS = SPLIT ? 3 * BN * SPLIT_PITCH : (BT ? BK : BN) * B_PITCH;
  static constexpr int LDS = A_FLOATS + B_FLOATS;      // floats
  static constexpr int AI = BM * BK / 4 / THREADS, BI = BN * BK / 4 / THREADS;     // loads of a thread per chunk
  static_assert(AI * THREADS * 4 == BM * BK && BI * THREADS * 4 == BN * BK, "whole loads");
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct Gemm32Operand {
  const float* p;
  int extent;            // of m resp. n
  int pitch;             // floats between rows
  uint32_t second = 0;   // floats to the second matrix of a pair
};

template <class C> using Gemm32Acc = f32x4[C::MB][C::NB];

// Values [at, at + 4) of a row of `limit` values, zero beyond it: fewer than four, or read (from where four exist) and shifted
__device__ __forceinline__ f32x4 load_few(const float* row, int at, int limit) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (at + e < limit) v[e] = row[at + e];
  return v;
}
__device__ __forceinline__ f32x4 load_end(const float* row, int at, int limit) { return *reinterpret_cast<const f32x4_any*>(row + min(at, limit - 4)); }
__device__ __forceinline__ f32x4 shift_end(f32x4 v, int at, int limit) {
  const int by = at - min(at, limit - 4);
  if (by & 1) v = f32x4{v.y, v.z, v.w, 0.f};
  if (by & 2) v = f32x4{v.z, v.w, 0.f, 0.f};
  return by < 4 ? v : f32x4{0.f, 0.f, 0.f, 0.f};
}

// One operand: EXTENT values of m resp. n from x0, T: in rows of k
template <int EXTENT, bool T, int LOADS, int PITCH, int THREADS> struct Gemm32Loader {
  f32x4 q[LOADS];
  const float* base;     // of the next chunk
  uint32_t off[LOADS];   // floats
  int end;               // rows of k: where the columns end, seen from x0; else unused
  bool edge;
  __device__ __forceinline__ void start(const Gemm32Operand& o, int x0, int k_lo, bool pair = false) {
    const int left = o.extent - x0;
    base = T ? o.p + (size_t)k_lo * o.pitch + x0 : o.p + (size_t)x0 * o.pitch + k_lo;
    end = left;
    edge = T && left < EXTENT;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int u = threadIdx.x + i * THREADS;
      if (T) off[i] = (uint32_t)(u / (EXTENT / 4)) * (uint32_t)o.pitch + (uint32_t)(u % (EXTENT / 4)) * 4u;
      else if (pair) off[i] = (uint32_t)min(((u / 8) >> 5) * 16 + ((u / 8) & 15), left - 1) * (uint32_t)o.pitch + (uint32_t)(u % 8) * 4u + (((u / 8) & 16) ? o.second : 0u);
      else off[i] = (uint32_t)min(u / 8, left - 1) * (uint32_t)o.pitch + (uint32_t)(u % 8) * 4u;
    }
  }
  // the chunk of which `left` values of k exist
  __device__ __forceinline__ void load(const Gemm32Operand& o, int left) {
    if (left >= 32 && !edge) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) q[i] = *reinterpret_cast<const f32x4_any*>(base + off[i]);
    } else {
      const int limit = T ? end : left < 32 ? left : 32;
      auto row = [&](int u, int i) { return T ? base + (size_t)min(u / (EXTENT / 4), left - 1) * o.pitch : base + off[i] - (u % 8) * 4; };
      auto at = [](int u) { return (T ? u % (EXTENT / 4) : u % 8) * 4; };
      if (limit >= 4) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) q[i] = load_end(row(threadIdx.x + i * THREADS, i), at(threadIdx.x + i * THREADS), limit);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) q[i] = shift_end(q[i], at(threadIdx.x + i * THREADS), limit);      // (once all are on their way)
      } else {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) q[i] = load_few(row(threadIdx.x + i * THREADS, i), at(threadIdx.x + i * THREADS), limit);
      }
      if (T && left < 32) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          if ((threadIdx.x + i * THREADS) / (EXTENT / 4) >= left) q[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    base += T ? (size_t)32 * o.pitch : 32;
  }
  __device__ __forceinline__ void stage(float* lds) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int u = threadIdx.x + i * THREADS;
      const int at = T ? (u / (EXTENT / 4)) * PITCH + (u % (EXTENT / 4)) * 4 : (u / 8) * PITCH + (u % 8) * 4;
      *reinterpret_cast<f32x4*>(lds + at) = q[i];
    }
  }
};

// v = h + m + l, each a bf16 value (8 significant bits), of four values that lie side by side
struct Split4 {
  uint2 h, m, l;
};
__device__ __forceinline__ Split4 split4(f32x4 v) {
  auto rest = [](f32x4 a, uint2 p) {
    return f32x4{a.x - __uint_as_float(p.x << 16), a.y - __uint_as_float(p.x & 0xffff0000u), a.z - __uint_as_float(p.y << 16),
                 a.w - __uint_as_float(p.y & 0xffff0000u)};
  };
  auto pack = [](f32x4 a) { return make_uint2(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w)); };
  // (the upper half as it is: rounded, the largest values would become infinite)
  auto upper = [](float a, float b) { return (__float_as_uint(a) >> 16) | (__float_as_uint(b) & 0xffff0000u); };
  Split4 s;
  s.h = make_uint2(upper(v.x, v.y), upper(v.z, v.w));
  v = rest(v, s.h);
  s.m = pack(v);
  s.l = pack(rest(v, s.m));
  return s;
}

// The same for products on the bf16 matrix cores: three planes of EXTENT rows of 32 values of k.  Rows of k: a thread takes four of them in four columns
// 32 apart, so that its values of k lie side by side in LDS and those of neighbouring threads in neighbouring rows.
template <int EXTENT, bool T, int LOADS, int PITCH, int THREADS> struct Gemm32SplitLoader : Gemm32Loader<EXTENT, T, LOADS, PITCH, THREADS> {
  typedef Gemm32Loader<EXTENT, T, LOADS, PITCH, THREADS> Base;
  static_assert(!T || (EXTENT == 128 && THREADS == 256 && LOADS == 4), "eight groups of four values of k");
  using Base::q;
  __device__ __forceinline__ void load(const Gemm32Operand& o, int left) {
    if constexpr (T) {
      const int k = (threadIdx.x >> 5) * 4, c = threadIdx.x & 31;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool there = k + e < left;
        const float* row = this->base + (size_t)min(k + e, left - 1) * o.pitch;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = row[min(c + 32 * i, this->end - 1)];
          q[i][e] = there ? v : 0.f;
        }
      }
      this->base += (size_t)32 * o.pitch;
    } else {
      Base::load(o, left);
    }
  }
  __device__ __forceinline__ void stage(float* lds) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int u = threadIdx.x + i * THREADS;
      const int at = T ? ((threadIdx.x & 31) + 32 * i) * PITCH + (threadIdx.x >> 5) * 2 : (u / 8) * PITCH + (u % 8) * 2;
      const Split4 s = split4(q[i]);
      *reinterpret_cast<uint2*>(lds + at) = s.h;
      *reinterpret_cast<uint2*>(lds + EXTENT * PITCH + at) = s.m;
      *reinterpret_cast<uint2*>(lds + 2 * EXTENT * PITCH + at) = s.l;
    }
  }
};

template <bool SPLIT, int EXTENT, bool T, int LOADS, int PITCH, int SPLIT_PITCH, int THREADS> struct Gemm32LoaderOf {
  typedef Gemm32Loader<EXTENT, T, LOADS, PITCH, THREADS> type;
};
template <int EXTENT, bool T, int LOADS, int PITCH, int SPLIT_PITCH, int THREADS> struct Gemm32LoaderOf<true, EXTENT, T, LOADS, PITCH, SPLIT_PITCH, THREADS> {
  typedef Gemm32SplitLoader<EXTENT, T, LOADS, SPLIT_PITCH, THREADS> type;
};

// The accumulators are those of the transposed block: a lane holds columns 4 * (lane / 16) .. + 3 of row lane % 16.
template <class C>
__device__ __forceinline__ void gemm32_tile(const Gemm32Operand& A, const Gemm32Operand& B, int m0, int n0, int k_lo, int k_hi, float* lds,
                                            Gemm32Acc<C>& acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm0 = (wave / C::WN) * 16 * C::MB, wn0 = (wave % C::WN) * 16 * C::NB;
  const int row = lane & 15, group = lane >> 4;
  float *const la = lds, *const lb = lds + C::A_FLOATS;
#pragma unroll
  for (int i = 0; i < C::MB; ++i)
#pragma unroll
    for (int j = 0; j < C::NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  typename Gemm32LoaderOf<C::SPLIT, C::BM, C::AT, C::AI, C::A_PITCH, C::SPLIT_PITCH, C::THREADS>::type a;
  typename Gemm32LoaderOf<C::SPLIT, C::BN, C::BT, C::BI, C::B_PITCH, C::SPLIT_PITCH, C::THREADS>::type b;
  a.start(A, m0, k_lo);
  b.start(B, n0, k_lo, C::PAIR);
  if (k_lo < k_hi) {
    a.load(A, k_hi - k_lo);
    b.load(B, k_hi - k_lo);
  }
  for (int k = k_lo; k < k_hi; k += C::BK) {
    __syncthreads();
    a.stage(la);
    b.stage(lb);
    __syncthreads();
    if (k + C::BK < k_hi) {
      a.load(A, k_hi - k - C::BK);
      b.load(B, k_hi - k - C::BK);
    }
    if constexpr (C::SPLIT) {
      // lane group g holds values of k 8 g .. 8 g + 7; the six largest products, the smallest of them first
      typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
      bf16x8 fb[3][C::NB];
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int j = 0; j < C::NB; ++j)
          fb[p][j] = *reinterpret_cast<const bf16x8*>(lb + (p * C::BN + wn0 + 16 * j + row) * C::SPLIT_PITCH + 4 * group);
#pragma unroll
      for (int i = 0; i < C::MB; ++i) {
        bf16x8 fa[3];
#pragma unroll
        for (int p = 0; p < 3; ++p) fa[p] = *reinterpret_cast<const bf16x8*>(la + (p * C::BM + wm0 + 16 * i + row) * C::SPLIT_PITCH + 4 * group);
        constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int u = 0; u < 6; ++u)
#pragma unroll
          for (int j = 0; j < C::NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[PB[u]][j], fa[PA[u]], acc[i][j], 0, 0, 0);
      }
      continue;
    }
    // lane group g multiplies values of k 4 g + e of each sixteen in step e
#pragma unroll
    for (int h = 0; h < C::BK; h += 16) {
      f32x4 fa[C::MB], fb[C::NB];
#pragma unroll
      for (int i = 0; i < C::MB; ++i) {
        if constexpr (C::AT) {
#pragma unroll
          for (int e = 0; e < 4; ++e) fa[i][e] = la[(h + 4 * group + e) * C::A_PITCH + wm0 + 16 * i + row];
        } else fa[i] = *reinterpret_cast<const f32x4*>(la + (wm0 + 16 * i + row) * C::A_PITCH + h + 4 * group);
      }
#pragma unroll
      for (int j = 0; j < C::NB; ++j) {
        if constexpr (C::BT) {
#pragma unroll
          for (int e = 0; e < 4; ++e) fb[j][e] = lb[(h + 4 * group + e) * C::B_PITCH + wn0 + 16 * j + row];
        } else fb[j] = *reinterpret_cast<const f32x4*>(lb + (wn0 + 16 * j + row) * C::B_PITCH + h + 4 * group);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < C::MB; ++i)
#pragma unroll
          for (int j = 0; j < C::NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[j][e], fa[i][e], acc[i][j], 0, 0, 0);
    }
  }
#endif
}

}  // namespace acc
