// One tile of a plain matrix product on the fp32 matrix cores, for kernels that do something of their own with it:
//
//   acc[m][n] = sum_k A[m][k] * B[k][n],   m in [m0, m0 + BM), n in [n0, n0 + BN), k in [k_lo, k_hi)
//
// Each operand lies in memory with its values of k side by side (rows of m resp. n) or with its values of m resp. n side by side (rows of k), at any
// width: 16 bytes at a time from addresses that need be aligned to 4 only, so odd widths cost no copy.  Loads that would pass the end of a row begin
// earlier and are shifted; rows that don't exist repeat the last one, whose results nobody stores, and values of k beyond k_hi are zero in both operands.
// A chunk of 32 values of k waits in registers while the one before it is multiplied out of LDS.  The matrix instructions bound it (256 operations per
// cycle and compute unit: a 128 x 128 x 32 chunk takes 4096 cycles, its LDS traffic a tenth of that), so one stage of LDS is enough and leaves room for
// several workgroups on a compute unit.  1024 x 2048 x 32768: 1134 us, 121 TFLOP/s of 157.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace acc {

// WM x WN waves, each MB x NB blocks of 16 x 16.  AT / BT: the operand lies in rows of k.
template <int WM_, int WN_, int MB_, int NB_, bool AT_, bool BT_> struct Gemm32Cfg {
  static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, BK = 32;
  static constexpr bool AT = AT_, BT = BT_;
  static constexpr int THREADS = 64 * WM * WN, BM = 16 * MB * WM, BN = 16 * NB * WN;
  // floats between staged rows: the sixteen rows (resp. four groups of sixteen columns) that a read takes at once fall on different banks
  static constexpr int A_PITCH = AT ? BM + 4 : BK + 4, B_PITCH = BT ? BN + 4 : BK + 4;
  static constexpr int A_FLOATS = (AT ? BK : BM) * A_PITCH, B_FLOATS = (BT ? BK : BN) * B_PITCH, LDS = A_FLOATS + B_FLOATS;
  static constexpr int AI = BM * BK / 4 / THREADS, BI = BN * BK / 4 / THREADS;     // loads of a thread per chunk
  static_assert(AI * THREADS * 4 == BM * BK && BI * THREADS * 4 == BN * BK, "whole loads");
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct Gemm32Operand {
  const float* p;
  int extent;            // of m resp. n
  int pitch;             // floats between rows
};

template <class C> using Gemm32Acc = f32x4[C::MB][C::NB];

// Values [at, at + 4) of a row of `limit` values, zero beyond it
__device__ __forceinline__ f32x4 load_end(const float* row, int at, int limit) {
  if (limit < 4) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (at + e < limit) v[e] = row[at + e];
    return v;
  }
  const int from = at < limit - 4 ? at : limit - 4, by = at - from;
  f32x4 v = *reinterpret_cast<const f32x4_any*>(row + from);
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
  __device__ __forceinline__ void start(const Gemm32Operand& o, int x0, int k_lo) {
    const int left = o.extent - x0;
    base = T ? o.p + (size_t)k_lo * o.pitch + x0 : o.p + (size_t)x0 * o.pitch + k_lo;
    end = left;
    edge = T && left < EXTENT;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int u = threadIdx.x + i * THREADS;
      if (T) off[i] = (uint32_t)(u / (EXTENT / 4)) * (uint32_t)o.pitch + (uint32_t)(u % (EXTENT / 4)) * 4u;
      else off[i] = (uint32_t)min(u / 8, left - 1) * (uint32_t)o.pitch + (uint32_t)(u % 8) * 4u;
    }
  }
  // the chunk of which `left` values of k exist
  __device__ __forceinline__ void load(const Gemm32Operand& o, int left) {
    if (left >= 32 && !edge) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) q[i] = *reinterpret_cast<const f32x4_any*>(base + off[i]);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int u = threadIdx.x + i * THREADS;
        if (T) {
          const int k = u / (EXTENT / 4);
          const f32x4 v = load_end(base + (size_t)min(k, left - 1) * o.pitch, (u % (EXTENT / 4)) * 4, end);
          q[i] = k < left ? v : f32x4{0.f, 0.f, 0.f, 0.f};
        } else {
          const int c = (u % 8) * 4;
          q[i] = load_end(base + off[i] - c, c, left < 32 ? left : 32);
        }
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
  Gemm32Loader<C::BM, C::AT, C::AI, C::A_PITCH, C::THREADS> a;
  Gemm32Loader<C::BN, C::BT, C::BI, C::B_PITCH, C::THREADS> b;
  a.start(A, m0, k_lo);
  b.start(B, n0, k_lo);
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
