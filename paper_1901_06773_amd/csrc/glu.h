// What the files of the gated layer share: glu.hip (fp32 products, few rows, values one by one, the choice) and glu_bf16.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "act.h"
#include "dtype.h"

namespace acc {

enum { GLU_NONE = 0, GLU_RELU = 1, GLU_SILU = 2 };     // as ACC_ACT_*

// act(a) = a s, act'(a) = s (1 + a (1 - s)) with s = 1, s = 1 where a is above 0 and 0 elsewhere (ReLU), or the sigmoid (SiLU): one way for all three.  (A
// branch for each makes the code of a tile, whose registers are named in it value by value, three times as long.)  Where s is 0 act(a) is 0 whatever a is,
// minus infinity too, and where it is 1 the slope is 1, so that an infinite gate times 0 makes no NaN.  What else is not finite stays: a NaN in a, and through
// a closed gate, as 0 times it, b and dh.
__device__ __forceinline__ float glu_share(int act, float a) {
  const float s = sigmoid(a), step = a <= 0.f ? 0.f : 1.f;
  return act == GLU_SILU ? s : act == GLU_RELU ? step : 1.f;
}
__device__ __forceinline__ float glu_act(int act, float a) {
  const float s = glu_share(act, a);
  return s == 0.f ? 0.f : a * s;
}
// gradients of h = act(a) b at a and b
__device__ __forceinline__ void glu_slopes(int act, float a, float b, float dh, float& da, float& db) {
  const float s = glu_share(act, a);
  const bool closed = s == 0.f;
  da = (closed ? dh * 0.f : dh) * b * (closed || s == 1.f ? 1.f : s * (1.f + a * (1.f - s)));      // (dh b alone might overflow)
  db = dh * (closed ? 0.f : a * s);
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
// parts: values that dz is kept as the sum of, 0 where it is not kept
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
// Many parts of db are added up in slabs first, into `slabs` (kDbSlabs rows of `pitch`), which then are its parts (us, dz and db, so / from all parts at once:
// 10^6 rows of 16 to 2 x 16 145 / 230, 3 10^5 of 32 to 2 x 32 56 / 79, 41379 of 1056 to 2 x 136, 650 parts, 52 / 52)
constexpr int kDbSlabs = 64, kDbMany = 512;
hipError_t glu_db_slabs(GluFinish& f, float* slabs, hipStream_t st);
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
