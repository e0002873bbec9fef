// A row of values that a workgroup (or a wave) keeps in its registers, sixteen bytes of it at a time.
//
// Rows of an odd number of values begin at any address that their type allows.  A row is cut at multiples of sixteen bytes of memory, not of the row, so
// that every chunk is one aligned load; the first and the last may hold values of the neighbouring rows, which are cut off once all loads are on their way.
// They are written value by value.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "dtype.h"
#include "sizes.h"

namespace acc {

// of the top logits and of the distillation from them: entries of a list, classes, rows
constexpr int kMostTop = 1024, kMostClasses = 1 << 20, kMostRows = 1 << 20;

typedef unsigned chunk16 __attribute__((ext_vector_type(4)));

template <class T> struct RowChunks {
  static constexpr int PER = 16 / (int)sizeof(T);      // values of a chunk
  long first;          // the value of the row that chunk 0 begins with: 0, or up to PER - 1 before it
  long ahead;          // values of the tensor from the row's first on
  int count, chunks;
  __device__ __forceinline__ RowChunks(const T* row, int count_, long ahead_) : ahead(ahead_), count(count_) {
    const int before = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    first = -before;
    chunks = (before + count + PER - 1) / PER;
  }
  __device__ __forceinline__ int at(int c) const { return c * PER + (int)first; }      // value that chunk c begins with
  // chunk c with what lies beside the row in it: what cut() is for
  __device__ __forceinline__ chunk16 load(const T* row, int c) const {
    const int e0 = at(c);
    if (e0 + PER <= ahead) return *reinterpret_cast<const chunk16*>(row + e0);         // (a tensor begins on such an address)
    union { chunk16 v; T e[PER]; } u;                  // the tensor's last values
#pragma unroll
    for (int e = 0; e < PER; ++e) u.e[e] = row[e0 + e < ahead ? e0 + e : ahead - 1];
    return u.v;
  }
  // what lies beyond the row is minus infinity
  __device__ __forceinline__ void cut(chunk16& v, int c) const {
    const int e0 = at(c);
    if (e0 >= 0 && e0 + PER <= count) return;
    union { chunk16 v; T e[PER]; } u;
    u.v = v;
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (e0 + e < 0 || e0 + e >= count) {
        if constexpr (sizeof(T) == 2) u.e[e] = 0xff80;
        else u.e[e] = -INFINITY;
      }
    v = u.v;
  }
  __device__ __forceinline__ void store(T* row, int c, const chunk16& v) const {
    const int e0 = at(c);
    if (e0 >= 0 && e0 + PER <= count) { *reinterpret_cast<chunk16*>(row + e0) = v; return; }
    union { chunk16 v; T e[PER]; } u;
    u.v = v;
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (e0 + e >= 0 && e0 + e < count) row[e0 + e] = u.e[e];
  }
  static __device__ __forceinline__ float value(const chunk16& v, int e) {
    if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
    else return __uint_as_float(v[e]);
  }
  static __device__ __forceinline__ chunk16 pack(const float (&f)[PER]) {
    chunk16 v;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = pack_bf16(f[2 * q], f[2 * q + 1]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = __float_as_uint(f[q]);
    }
    return v;
  }
};

// Reductions over the NT threads that share a row: one wave without a barrier, or a workgroup by way of sh (NT / 64 values of its own for every call
// between two barriers).  Everybody gets the result.
template <int NT> __device__ __forceinline__ void row_sync() {
  if constexpr (NT == 64) {
#if defined(__HIP_DEVICE_COMPILE__)
    __threadfence_block();                             // (a wave's LDS and memory accesses are done)
    __builtin_amdgcn_wave_barrier();
#endif
  } else {
    __syncthreads();
  }
}
// over 2^k = N <= 16 neighbouring lanes, by rotations in a row of sixteen: after each the values repeat with half the period, so that all lanes have the same bits
template <int N, class V, class F> __device__ __forceinline__ V row16_reduce(V v, F op) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two words");
#if defined(__HIP_DEVICE_COMPILE__)
  auto turned = [](V x, auto by) {
    constexpr int ctrl = 0x120 + decltype(by)::value;
    union { V v; int w[sizeof(V) / 4]; } u;
    u.v = x;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(V) / 4); ++i) u.w[i] = __builtin_amdgcn_update_dpp(0, u.w[i], ctrl, 0xf, 0xf, false);
    return u.v;
  };
  if constexpr (N >= 16) v = op(v, turned(v, std::integral_constant<int, 8>()));
  if constexpr (N >= 8) v = op(v, turned(v, std::integral_constant<int, 4>()));
  if constexpr (N >= 4) v = op(v, turned(v, std::integral_constant<int, 2>()));
  if constexpr (N >= 2) v = op(v, turned(v, std::integral_constant<int, 1>()));
#endif
  return v;
}
template <class V, class F> __device__ __forceinline__ V wave_reduce(V v, F op) {
  v = row16_reduce<16>(v, op);
  v = op(v, __shfl_xor(v, 16));
  return op(v, __shfl_xor(v, 32));
}
// the waves' values, which lie in LDS
template <int NT, class V, class F> __device__ __forceinline__ V join_waves(const V* sh, F op) { return row16_reduce<NT / 64>(sh[threadIdx.x & (NT / 64 - 1)], op); }
template <int NT, class V, class F> __device__ __forceinline__ V row_reduce(V v, V* sh, F op) {
  v = wave_reduce(v, op);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = join_waves<NT>(sh, op);
  }
  return v;
}

}  // namespace acc
