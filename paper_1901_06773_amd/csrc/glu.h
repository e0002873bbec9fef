// What the files of the gated layer share: glu.hip (fp32 products, few rows, values one by one, the choice) and glu_bf16.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "act.h"
#include "dtype.h"

namespace acc {

enum { GLU_NONE = 0, GLU_RELU = 1, GLU_SILU = 2 };     // as ACC_ACT_*

__device__ __forceinline__ float glu_act(int act, float a) {
  if (act == GLU_RELU) return a < 0.f ? 0.f : a;       // (a value that is no number stays none)
  if (act == GLU_SILU) return a * sigmoid(a);
  return a;
}
// gradients of h = act(a) b at a and b
__device__ __forceinline__ void glu_slopes(int act, float a, float b, float dh, float& da, float& db) {
  if (act == GLU_RELU) {
    da = a > 0.f ? dh * b : 0.f;
    db = dh * (a < 0.f ? 0.f : a);
  } else if (act == GLU_SILU) {
    const float s = sigmoid(a);
    da = dh * b * (s * (1.f + a * (1.f - s)));
    db = dh * (a * s);
  } else {
    da = dh * b;
    db = dh * a;
  }
}

struct GluArgs {
  const void *x, *w;
  const float* bias;           // [2 f], or null
  const void *ab_in, *dh;      // backward: the kept projections (null: worked out again)
  void *h, *ab;                // forward; ab: null, or the projections are kept there
  void* dx;                    // backward
  float *dw, *db;
  int rows, d, f, act;
  char* ws;
  int dtype;
  hipStream_t st;
};

// Values one by one, in 256 threads: tx threads of V columns across, 256 / tx rows at a time, `slab` rows to a workgroup.
struct PointArgs {
  const float* sums;           // projections in parts: sums[split][rows][2 f]; or null:
  const void* ab_in;           // as they are kept
  const float* bias;           // added to the sums, or null
  const void* dh;
  void *h, *ab;                // forward
  void* dz[3];                 // backward: [rows][pitch], the value's columns from `half` on; bf16: the sum of so many matrices
  float* db_part;              // [slab][pitch], or null
  int rows, f, act, splits, pitch, half, tx, across, slab;
};
hipError_t glu_point(const PointArgs& a, bool backward, int parts, int dtype, hipStream_t st);
// slabs of a launch (rows of db_part); sets tx, across and slab
int glu_point_shape(PointArgs& a, int dtype);

// dx from its splits (dtype), dw from its splits (rows [0, f) and [half, half + f) of m are the gate's and the value's), db from its parts
struct GluFinish {
  const float *dx_sums, *dw_sums, *db_part;
  void* dx;
  float *dw, *db;
  size_t dx_count, dw_count;
  int dx_splits, dw_splits, db_parts, pitch, half, f;
};
// the sums of parts, and db unless another launch has it
hipError_t glu_finish(const GluFinish& f, bool db, int dtype, hipStream_t st);
constexpr int kDbColumns = 16;       // columns of db to a workgroup, sixteen threads down each
inline unsigned glu_db_blocks(const GluFinish& f) { return f.db ? (unsigned)((2L * f.f + kDbColumns - 1) / kDbColumns) : 0; }
__device__ __forceinline__ void glu_db(const GluFinish& f, int block) {
  __shared__ double sh[256];
  const int j = block * kDbColumns + (threadIdx.x & 15);
  double s = 0.0;
  if (j < 2 * f.f) {
    const float* const p = f.db_part + (j < f.f ? j : f.half + j - f.f);
#pragma unroll 8
    for (int k = threadIdx.x >> 4; k < f.db_parts; k += 16) s += (double)p[(size_t)k * f.pitch];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x >= 16 || j >= 2 * f.f) return;
  for (int k = 1; k < 16; ++k) s += sh[threadIdx.x + 16 * k];
  f.db[j] = (float)s;
}

size_t glu_bf16_workspace_bytes(int rows, int d, int f, bool backward);
hipError_t glu_bf16(const GluArgs& a, bool backward);

}  // namespace acc
