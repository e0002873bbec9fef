// What the files of the linear cross-entropy share: linear_ce.hip (fp32 products, joining of sums, the choice) and linear_ce_bf16.hip.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace acc {

// Tile `at` of a launch: every XCD takes a contiguous range (neighbours share operand rows in its L2), rows innermost.
__device__ __forceinline__ int xcd_tile(int blocks) { return ((int)blockIdx.x & 7) * (blocks >> 3) + ((int)blockIdx.x >> 3); }

// Which tile: columns in blocks of four, within a block row by row, so that the workgroups of an XCD that run at the same time (thirty-two) stand eight by
// four and share operand rows both ways.
struct TileAt { int m, n; };
__device__ __forceinline__ TileAt tile_at(int at, int tiles_m, int tiles) {
  const int block = at / (4 * tiles_m), in = at - block * 4 * tiles_m, left = tiles / tiles_m - 4 * block, width = left < 4 ? left : 4, m = in / width;
  return TileAt{m, 4 * block + in - m * width};
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
