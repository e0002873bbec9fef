// What the files of the linear cross-entropy share: linear_ce.hip (fp32 products, joining of sums, the choice) and linear_ce_bf16.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "gemm_tiles.h"

namespace acc {

// The splits' m and R of a row joined, by `lanes` (a power of two) neighbouring lanes.  part[row][2][splits].
struct RowStats {
  float max, rest, loss;
};
__device__ __forceinline__ RowStats join_row(const float* __restrict__ part, const float* __restrict__ z_label, const int32_t* __restrict__ labels, int ignore,
                                             int row, int splits, int classes, int lanes) {
  const int lane = threadIdx.x & (lanes - 1);
  const float* p = part + (size_t)row * 2 * splits;
  const int lab = labels[row];
  const float at_label = z_label[row];
  float mx = -INFINITY;
  for (int i = lane; i < splits; i += lanes) mx = fmaxf(mx, p[i]);
  for (int o = lanes >> 1; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  float s = 0.f, equal = 0.f;
  for (int i = lane; i < splits; i += lanes) {
    const bool top = p[i] == mx;
    equal += top ? 1.f : 0.f;
    s += top ? p[splits + i] : (1.f + p[splits + i]) * expf(p[i] - mx);
  }
  for (int o = lanes >> 1; o > 0; o >>= 1) { s += __shfl_xor(s, o); equal += __shfl_xor(equal, o); }
  const float rest = mx == -INFINITY ? NAN : s + (equal - 1.f);     // (every class ruled out: no distribution)
  const bool skip = ignore != INT_MIN && lab == ignore, known = (unsigned)lab < (unsigned)classes;
  return RowStats{mx, rest, skip ? 0.f : known ? log1pf(rest) - (at_label - mx) : NAN};
}

// scale[0] = 1 / rows that count (0 if there is none), loss = their mean, of NT threads and in a fixed order.  Any of the three pointers of floats may be null.
template <int NT>
__device__ __forceinline__ void mean_of_rows(const float* loss_rows, const int32_t* __restrict__ labels, int ignore, int n, float* __restrict__ scale,
                                             float* __restrict__ loss) {
  __shared__ double sh[NT / 64];
  __shared__ int counts[NT / 64];
  double s = 0.0;
  int k = 0;
  for (int i = threadIdx.x; i < n; i += NT) {
    if (loss_rows) s += (double)loss_rows[i];
    k += ignore == INT_MIN || labels[i] != ignore ? 1 : 0;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { s += __shfl_xor(s, o); k += __shfl_xor(k, o); }
  if ((threadIdx.x & 63) == 0) { sh[threadIdx.x >> 6] = s; counts[threadIdx.x >> 6] = k; }
  __syncthreads();
  if (threadIdx.x) return;
  double t = 0.0;
  int rows = 0;
  for (int w = 0; w < NT / 64; ++w) { t += sh[w]; rows += counts[w]; }
  if (scale) scale[0] = rows ? 1.f / (float)rows : 0.f;
  if (loss) *loss = rows ? (float)(t / (double)rows) : 0.f;
}

struct LceArgs {
  const void *x, *w;
  const float* bias;
  const int32_t* labels;
  int ignore;
  float *loss_rows, *loss;
  void* dx;
  float *dw, *db;
  int n, d, classes;
  char* ws;
  int dtype;
  hipStream_t st;
};

// Per row the largest logit m, R = the sum of the others' exp(z - m), the label's logit and the loss; scale[0] = 1 / rows that count.
// 4 n + 64 floats of the workspace.
struct LceStats {
  float *row_max, *row_rest, *z_label, *loss_rows, *scale;
};
inline LceStats lce_stats(const LceArgs& a, size_t at) {
  float* const p = reinterpret_cast<float*>(a.ws + at);
  return LceStats{p, p + a.n, p + 2 * (size_t)a.n, a.loss_rows ? a.loss_rows : p + 3 * (size_t)a.n, p + 4 * (size_t)a.n};
}
// part[row][2][splits] (m and R of the splits) joined: row_max, row_rest, loss_rows, scale and the loss, if it is wanted
hipError_t lce_join(const LceArgs& a, const LceStats& s, const float* part, int splits);

bool linear_ce_bf16_takes(int n, int d, int classes);
size_t linear_ce_bf16_workspace_bytes(int n, int d, int classes, bool grads);
hipError_t linear_ce_bf16(const LceArgs& a);

}  // namespace acc
