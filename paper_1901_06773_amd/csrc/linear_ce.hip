// Softmax cross-entropy of a linear layer, in pieces of its classes, so that the logits of all classes are never in memory:
//
//   z = x w^T + b,  lse_i = log sum_v exp z_iv,  loss_i = lse_i - z_i[label_i],  loss = mean over the rows that count
//   dz = (softmax(z) - onehot) / rows that count,  dx = dz w,  dw = dz^T x,  db = sum_i dz_i
//
// Two sweeps over the pieces: the first leaves, per row and piece, the largest logit and the sum of exponentials relative to it (and the
// label's logit), which a short launch joins into lse; the second works the logits out again, turns them into dz and multiplies it with
// both operands.  With one piece the logits of the first sweep are still there.  2 n d classes operations for the loss, 6 more (4 with
// one piece) for the gradients, which is what bounds it.
//
// fp32: logits and dz of a piece in fp32, products by gemm_f32.h, whose epilogue takes the rows' sums along.  Few rows and classes: a launch turns
// whole rows of logits into dz.  Few tiles: dx, dw, db and the mean loss in one launch.
#include "kernels.h"
#include "dtype.h"
#include "gemm_f32.h"
#include "product32.h"
#include "linear_ce.h"

#include <climits>

namespace acc {
namespace {

constexpr int THREADS = 256;

// ---------------------------------------------------------------------------------- the rows' sums
template <class F>
__device__ __forceinline__ float block_reduce(float v, float* sh, F op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = sh[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) r = op(r, sh[w]);
  return r;
}

// A row's exponentials are summed without the largest one, which is 1: with m the largest logit, R = sum of the others' exp(z - m), the sum is
// 1 + R, and where a class is all but certain neither the loss, log1p(R) - (z_label - m), nor the label's gradient, (expm1(z_label - m) - R) /
// (1 + R), loses R to the rounding of 1 + R.  Columns that hold nothing (logits of minus infinity): m = minus infinity, R = -1.

// m and R of the columns [lo, hi) of a row: part[row][2][splits]; z's `parts` matrices (`whole` floats apart) are added up into the first one.
__global__ __launch_bounds__(THREADS) void row_sums_kernel(float* __restrict__ z, const float* __restrict__ bias, const int32_t* __restrict__ labels,
                                                           float* __restrict__ part, float* __restrict__ z_label, int pitch, int cols, int v0,
                                                           int per_split, int splits_here, int split0, int splits, int parts, size_t whole) {
  __shared__ float sh[THREADS / 64];
  const int row = blockIdx.x / splits_here, sp = blockIdx.x - row * splits_here;
  const int lo = sp * per_split, hi = min(lo + per_split, cols);
  float* const zr = z + (size_t)row * pitch;
  float mx = -INFINITY;
  for (int j = lo + threadIdx.x; j < hi; j += THREADS) {
    float v = zr[j];
    if (parts > 1) {
#pragma unroll 4
      for (int k = 1; k < parts; ++k) v += zr[k * whole + j];
      zr[j] = v;
    }
    mx = fmaxf(mx, v + (bias ? bias[v0 + j] : 0.f));
  }
  mx = block_reduce(mx, sh, [](float a, float b) { return fmaxf(a, b); });
  float s = 0.f, equal = 0.f;
  // (a logit that is no number was dropped by the maximum and shows in the sum)
  for (int j = lo + threadIdx.x; j < hi; j += THREADS) {
    const float v = zr[j] + (bias ? bias[v0 + j] : 0.f);
    const bool top = v == mx;
    equal += top ? 1.f : 0.f;
    s += top ? 0.f : expf(v - mx);
  }
  s = block_reduce(s, sh, [](float a, float b) { return a + b; });
  equal = block_reduce(equal, sh, [](float a, float b) { return a + b; });
  if (threadIdx.x == 0) {
    float* p = part + (size_t)row * 2 * splits + split0 + sp;
    p[0] = mx;
    p[splits] = mx == -INFINITY && !(s != s) ? -1.f : s + (equal - 1.f);
    const long at = (long)labels[row] - v0;      // (written by another thread of this workgroup, before the barriers)
    if (at >= lo && at < hi) z_label[row] = zr[at] + (bias ? bias[v0 + at] : 0.f);
  }
}

__global__ __launch_bounds__(THREADS) void join_kernel(const float* __restrict__ part, const float* __restrict__ z_label, const int32_t* __restrict__ labels,
                                                       int ignore, float* __restrict__ row_max, float* __restrict__ row_rest, float* __restrict__ loss_rows,
                                                       int n, int splits, int classes, int lanes) {
  const int row = (blockIdx.x * THREADS + threadIdx.x) / lanes;
  if (row >= n) return;
  const RowStats r = join_row(part, z_label, labels, ignore, row, splits, classes, lanes);
  if ((threadIdx.x & (lanes - 1)) == 0) { row_max[row] = r.max; row_rest[row] = r.rest; loss_rows[row] = r.loss; }
}

__global__ __launch_bounds__(1024) void mean_kernel(const float* __restrict__ loss_rows, const int32_t* __restrict__ labels, int ignore, int n,
                                                    float* __restrict__ scale, float* __restrict__ loss) {
  mean_of_rows<1024>(loss_rows, labels, ignore, n, scale, loss);
}
// both, in one workgroup
__global__ __launch_bounds__(1024) void join_mean_kernel(const float* __restrict__ part, const float* __restrict__ z_label, const int32_t* __restrict__ labels,
                                                         int ignore, float* __restrict__ row_max, float* __restrict__ row_rest, float* loss_rows, int n,
                                                         int splits, int classes, float* __restrict__ scale, float* __restrict__ loss, int lanes) {
  for (int row = threadIdx.x / lanes; row < n; row += 1024 / lanes) {
    const RowStats r = join_row(part, z_label, labels, ignore, row, splits, classes, lanes);
    if ((threadIdx.x & (lanes - 1)) == 0) { row_max[row] = r.max; row_rest[row] = r.rest; loss_rows[row] = r.loss; }
  }
  __threadfence_block();
  __syncthreads();
  mean_of_rows<1024>(loss_rows, labels, ignore, n, scale, loss);
}

// A whole row of logits at once, one workgroup per row, up to V values in a thread's registers: the loss, and with `grads` z -> dz in place, columns beyond
// the classes zero.  The rows that count are counted by every workgroup, while its logits are on their way.
template <int V, int NT>
__global__ __launch_bounds__(NT) void rows_kernel(float* __restrict__ z, const float* __restrict__ bias, const int32_t* __restrict__ labels, int ignore,
                                                  float* __restrict__ loss_rows, int n, int pitch, int cols, int grads, int splits) {
  __shared__ float sh[3][NT / 64];
  __shared__ int counted;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float* const zr = z + (size_t)row * pitch;
  float v[V];
#pragma unroll
  for (int u = 0; u < V; ++u) v[u] = zr[min(tid + u * NT, cols - 1)];
  const size_t whole = (size_t)n * pitch;
  int part = 1;
  constexpr int AHEAD = V >= 8 ? 2 : 4;                 // the product's parts along d, some on their way at once
  for (; part + AHEAD <= splits; part += AHEAD) {
    float q[AHEAD][V];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int u = 0; u < V; ++u) q[a][u] = zr[(part + a) * whole + min(tid + u * NT, cols - 1)];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int u = 0; u < V; ++u) v[u] += q[a][u];
  }
  for (; part < splits; ++part)
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] += zr[part * whole + min(tid + u * NT, cols - 1)];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int j = tid + u * NT;
    if (bias) v[u] += bias[min(j, cols - 1)];
    if (j >= cols) v[u] = -INFINITY;
  }
  const int lab = labels[row];
  const bool skip = ignore != INT_MIN && lab == ignore, known = (unsigned)lab < (unsigned)cols;
  int k = 0;
  if (grads && ignore != INT_MIN)
    for (int i = tid; i < n; i += NT) k += labels[i] != ignore ? 1 : 0;
  if (tid == 0) counted = 0;
  float mx = -INFINITY;
#pragma unroll
  for (int u = 0; u < V; ++u) mx = fmaxf(mx, v[u]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  if (lane == 0) sh[0][wave] = mx;
  __syncthreads();
  if (grads && ignore != INT_MIN) atomicAdd(&counted, k);              // (whole numbers: any order gives the same)
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) mx = fmaxf(mx, sh[0][w]);
  float s = 0.f, equal = 0.f, t_label = 0.f;
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int j = tid + u * NT;
    if (j < cols) {
      const bool top = v[u] == mx;
      const float t = v[u] - mx;
      if (j == lab) t_label = t;
      v[u] = expf(t);
      equal += top ? 1.f : 0.f;
      s += top ? 0.f : v[u];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { s += __shfl_xor(s, o); equal += __shfl_xor(equal, o); }
  if (lane == 0) { sh[1][wave] = s; sh[2][wave] = equal; }
  __syncthreads();
  s = equal = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) { s += sh[1][w]; equal += sh[2][w]; }
  const float rest = mx == -INFINITY ? NAN : s + (equal - 1.f);
  if (known ? tid == lab % NT : tid == 0) loss_rows[row] = skip ? 0.f : known ? log1pf(rest) - t_label : NAN;
  if (!grads) return;
  const int rows = ignore == INT_MIN ? n : counted;
  const float inv = skip || rows == 0 ? 0.f : 1.f / (float)rows / (1.f + rest);
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int j = tid + u * NT;
    if (j >= pitch) continue;
    const float p = j == lab ? expm1f(t_label) - rest : v[u];
    zr[j] = skip || j >= cols ? 0.f : p * inv;
  }
}

// z -> dz in place, columns beyond the classes zero, and the columns' sums over the rows of a workgroup: db_part[workgroup][pitch].  666 x 55313: 48 us for
// 295 MB (6.1 TB/s, the logits being in the memory-side cache).
__global__ __launch_bounds__(THREADS) void dz_kernel(float* __restrict__ z, const float* __restrict__ bias, const int32_t* __restrict__ labels, int ignore,
                                                     const float* __restrict__ row_max, const float* __restrict__ row_rest, const float* __restrict__ scale,
                                                     float* __restrict__ db_part, int n, int pitch, int cols, int v0, int rows) {
  const int j = (blockIdx.x * THREADS + threadIdx.x) * 4;
  if (j >= pitch) return;
  const int r0 = blockIdx.y * rows, r1 = min(r0 + rows, n);
  const float sc = scale[0];
  float b[4], sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = bias && j + e < cols ? bias[v0 + j + e] : 0.f;
  for (int r = r0; r < r1; r += 4) {           // four rows on their way at once
    float4 q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = *reinterpret_cast<const float4*>(z + (size_t)min(r + u, r1 - 1) * pitch + j);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (r + u >= r1) break;
      const int lab = labels[r + u];
      const bool skip = ignore != INT_MIN && lab == ignore;
      const float mx = row_max[r + u], rest = row_rest[r + u], inv = 1.f / (1.f + rest);
      float v[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float t = v[e] + b[e] - mx, p = (lab == v0 + j + e ? expm1f(t) - rest : expf(t)) * inv;
        v[e] = skip || j + e >= cols ? 0.f : p * sc;
        sum[e] += v[e];
      }
      *reinterpret_cast<float4*>(z + (size_t)(r + u) * pitch + j) = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
  if (db_part) *reinterpret_cast<float4*>(db_part + (size_t)blockIdx.y * pitch + j) = make_float4(sum[0], sum[1], sum[2], sum[3]);
}

// ---------------------------------------------------------------------------------- products
struct Logits32 {
  Gemm32Operand x, w;
  const float* bias;             // null: none, or added later
  const int32_t* labels;
  float *z, *part, *z_label;     // z[split][n][pitch], or null; part: m and R of each tile's columns, or null
  int d, k_per_split, pitch, v0, split0, splits, tiles_m, tiles, work;
};
template <class C>
__global__ __launch_bounds__(C::THREADS) void logits32_kernel(Logits32 a, int blocks) {
  __shared__ __attribute__((aligned(16))) float lds[C::LDS];
  const int work = xcd_tile(blocks);
  if (work >= a.work) return;
  const int split = work / a.tiles;
  const TileAt where = tile_at(work - split * a.tiles, a.tiles_m, a.tiles);
  const int n = a.x.extent, cols = a.w.extent, m0 = where.m * C::BM, n0 = where.n * C::BN;
  Gemm32Acc<C> acc;
  gemm32_tile<C>(a.x, a.w, m0, n0, split * a.k_per_split, min(a.d, (split + 1) * a.k_per_split), lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm0 = (wave / C::WN) * 16 * C::MB, wn = wave % C::WN;
  const int col0 = n0 + wn * 16 * C::NB + 4 * (lane >> 4);
#pragma unroll
  for (int j = 0; j < C::NB; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = col0 + 16 * j + e;
      const float b = a.bias && c < cols ? a.bias[c] : 0.f;
#pragma unroll
      for (int i = 0; i < C::MB; ++i) acc[i][j][e] = c < cols ? acc[i][j][e] + b : -INFINITY;
    }
  if (a.z) {
    float* const z = a.z + (size_t)split * n * a.pitch;
#pragma unroll
    for (int i = 0; i < C::MB; ++i) {
      const int m = m0 + wm0 + 16 * i + (lane & 15);
#pragma unroll
      for (int j = 0; j < C::NB; ++j)
        if (m < n && col0 + 16 * j < a.pitch) *reinterpret_cast<f32x4*>(z + (size_t)m * a.pitch + col0 + 16 * j) = acc[i][j];
    }
  }
  if (!a.part) return;
  float(*red)[C::BM][3] = reinterpret_cast<float(*)[C::BM][3]>(lds);
  static_assert(C::WN * C::BM * 3 <= C::LDS, "the waves' sums fit the operands' place");
  __syncthreads();
#pragma unroll
  for (int i = 0; i < C::MB; ++i) {
    const int m = m0 + wm0 + 16 * i + (lane & 15);
    float mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) mx = fmaxf(mx, acc[i][j][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const int lab = m < n ? (int)((unsigned)a.labels[m] - (unsigned)a.v0) : -1;
    float s = 0.f, equal = 0.f;
#pragma unroll
    for (int j = 0; j < C::NB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v = acc[i][j][e];
        const int c = col0 + 16 * j + e;
        const bool top = v == mx;
        equal += top && c < cols ? 1.f : 0.f;
        s += top ? 0.f : expf(v - mx);
        if (lab == c && c < cols) a.z_label[m] = v;
      }
    s += __shfl_xor(s, 16); s += __shfl_xor(s, 32);
    equal += __shfl_xor(equal, 16); equal += __shfl_xor(equal, 32);
    if (lane < 16) { float* r = red[wn][wm0 + 16 * i + lane]; r[0] = mx; r[1] = s; r[2] = equal; }
  }
  __syncthreads();
  for (int row = threadIdx.x; row < C::BM; row += C::THREADS) {
    if (m0 + row >= n) continue;
    float mx = -INFINITY, s = 0.f, equal = 0.f;
#pragma unroll
    for (int w = 0; w < C::WN; ++w) mx = fmaxf(mx, red[w][row][0]);
#pragma unroll
    for (int w = 0; w < C::WN; ++w) {
      const float mw = red[w][row][0], sw = red[w][row][1], ew = red[w][row][2];
      const bool top = mw == mx;
      s += top || mw == -INFINITY ? sw : (sw + ew) * expf(mw - mx);
      equal += top ? ew : 0.f;
    }
    float* p = a.part + (size_t)(m0 + row) * 2 * a.splits + a.split0 + where.n;
    p[0] = mx;
    p[a.splits] = mx == -INFINITY && !(s != s) ? -1.f : s + (equal - 1.f);
  }
}

// ---------------------------------------------------------------------------------- the last launch of a piece
// dx and dw from their splits, db from the columns of dz (or of its workgroups' sums), the mean loss; each in workgroups of its own.
struct Finish32 {
  const float* dx_sums;
  void* dx;
  const float* dw_sums;
  float* dw;
  const float* columns;          // `rows` rows of `pitch` floats, added up in slabs of kColumnRows
  float* db;
  const float* loss_rows;        // null: no mean
  const int32_t* labels;
  float* loss;
  size_t dx_count, dw_count;
  int dx_splits, dw_splits, rows, pitch, cols, across, n, ignore;
  unsigned dx_blocks, dw_blocks, db_blocks;
};
constexpr int kColumnRows = 1024;
template <class T>
__device__ __forceinline__ void finish32(const Finish32& f, unsigned block) {
  if (block < f.dx_blocks) return join_sums<T>(f.dx_sums, (T*)f.dx, f.dx_count, f.dx_splits, block, f.dx_blocks);
  block -= f.dx_blocks;
  if (block < f.dw_blocks) return join_sums<float>(f.dw_sums, f.dw, f.dw_count, f.dw_splits, block, f.dw_blocks);
  block -= f.dw_blocks;
  if (block >= f.db_blocks) return mean_of_rows<THREADS>(f.loss_rows, f.labels, f.ignore, f.n, nullptr, f.loss);
  // sixty-four columns, a quarter of the slab's rows to each wave
  __shared__ double sh[THREADS];
  const int slab = block / f.across, j = (block - slab * f.across) * 64 + (threadIdx.x & 63);
  const int first = slab * kColumnRows, count = min(kColumnRows, f.rows - first), quarter = (count + 3) / 4;
  int r = first + (int)(threadIdx.x >> 6) * quarter;
  const int end = min(r + quarter, first + count);
  double s = 0.0;
  if (j < f.cols) {
    for (; r + 16 <= end; r += 16) {
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = f.columns[(size_t)(r + u) * f.pitch + j];
#pragma unroll
      for (int u = 0; u < 16; ++u) s += (double)v[u];
    }
    for (; r < end; ++r) s += (double)f.columns[(size_t)r * f.pitch + j];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 64 && j < f.cols) f.db[(size_t)slab * f.pitch + j] = (float)(sh[threadIdx.x] + sh[threadIdx.x + 64] + sh[threadIdx.x + 128] + sh[threadIdx.x + 192]);
}
template <class T>
__global__ __launch_bounds__(THREADS) void finish32_kernel(Finish32 f) { finish32<T>(f, blockIdx.x); }

// dx, dw, db and the mean loss in one launch, 64 x 64 tiles.  They all wait for dz only: where there are few tiles, three launches less (us, all results,
// 64 x 256 x 256 25.6 / 19.5, 200 x 130 x 77 30.2 / 26.3).
typedef Gemm32Cfg<2, 2, 2, 2, false, true, false> Dx64;
typedef Gemm32Cfg<2, 2, 2, 2, true, true, false> Dw64;
__global__ __launch_bounds__(THREADS) void grads32_kernel(Product32 dx, Product32 dw, Finish32 rest, int dx_blocks, int dw_blocks) {
  __shared__ __attribute__((aligned(16))) float lds[Dx64::LDS > Dw64::LDS ? Dx64::LDS : Dw64::LDS];
  const int block = blockIdx.x;                        // (each part begins at a multiple of eight)
  if (block < dx_blocks) {
    const int work = (block & 7) * (dx_blocks >> 3) + (block >> 3);
    if (work < dx.work) product32<Dx64>(dx, work, lds);
  } else if (block < dx_blocks + dw_blocks) {
    const int work = (block & 7) * (dw_blocks >> 3) + ((block - dx_blocks) >> 3);
    if (work < dw.work) product32<Dw64>(dw, work, lds);
  } else {
    finish32<float>(rest, (unsigned)(block - dx_blocks - dw_blocks));
  }
}
// the slabs' sums
__global__ __launch_bounds__(THREADS) void db_kernel(const float* __restrict__ part, float* __restrict__ db, int parts, int pitch, int cols) {
  const int j = blockIdx.x * THREADS + threadIdx.x;
  if (j >= cols) return;
  double s = 0.0;
  for (int k = 0; k < parts; ++k) s += (double)part[(size_t)k * pitch + j];
  db[j] = (float)s;
}

// out (fp32) = in (bf16)
__global__ __launch_bounds__(THREADS) void widen_kernel(const bf16_t* __restrict__ in, float* __restrict__ out, size_t total) {
  for (size_t i = (size_t)blockIdx.x * THREADS + threadIdx.x; i < total; i += (size_t)gridDim.x * THREADS) out[i] = Elem<bf16_t>::load(in + i);
}

// ---------------------------------------------------------------------------------- fp32
constexpr int kRowCols = 8192;                 // columns that a workgroup keeps as a whole row
constexpr int kSplitCols = 2048;               // columns of a row that one workgroup adds up

// out[n][n_out] = in[n][c] * w[n_out][c]^T, as a convolution
ConvGeom product_geom(const float* in, const float* w, float* out, int n, int c, int n_out) {
  ConvGeom g{};
  g.in = in; g.w = w; g.out = out; g.dtype = DT_F32;
  g.n_img = n; g.h = g.wd = g.p = g.q = g.out_h = g.out_w = 1;
  g.c = c; g.n_out = n_out; g.r = g.s = g.stride = g.out_stride = 1;
  return g;
}

struct Plan32 {
  long piece, pieces, splits;    // classes of a piece, pieces, columns of `part`
  int pitch;                     // of z
  bool rows;                     // few rows and classes: a workgroup per row
  bool conv;                     // dx and dw by the convolution kernels
  bool late;                     // the logits' sums and bias in a launch of their own: row_sums_kernel
  bool widen;                    // bf16 operands are copied
  bool together;                 // dx, dw, db and the mean in one launch
  int dz_rows, slabs;            // rows of a workgroup of dz_kernel, and workgroups
  Cut z, dx, dw;
  bool sum_dx;                   // dx from `dx_sums`
  size_t stats, part, logits, x, w, dx_sums, dw_sums, db, wgrad, total;   // offsets of the parts of the workspace, and its size
  size_t wgrad_bytes;
};

Plan32 plan32(int n, int d, int classes, bool grads, int dtype) {
  Plan32 p{};
  // 256 MiB of logits, and of the filter 1 GiB in fp32 where it is copied, 128 classes at least (more than 2^19 rows then have more)
  long most = (1L << 26) / n / 128 * 128;
  if (dtype != DT_F32 && most > (1L << 28) / d / 128 * 128) most = (1L << 28) / d / 128 * 128;
  if (most < 128) most = 128;
  p.piece = classes <= most ? classes : most;
  p.pieces = ceil_div(classes, p.piece);
  p.pitch = (int)up(p.piece, 4);
  // (us, all results, a workgroup per row / sums with the logits: 300 x 64 x 40 24 / 32, 1024 x 512 x 1000 58 / 63, 4096 x 512 x 1000 146 / 150,
  // 16384 x 256 x 1000 235 / 226, 512 x 128 x 8000 71 / 69, 2048 x 64 x 8000 131 / 118, 4096 x 128 x 4000 193 / 172)
  p.rows = p.pieces == 1 && n <= 4096 && p.piece <= (n <= 512 ? kRowCols : kRowCols / 4);
  p.widen = dtype != DT_F32;
  // Few rows and classes of whole widths: the convolution kernels' launches, which deal the sum out among the waves of a workgroup, are faster than cutting it
  // and a launch for the parts' sums.  us, all results, here / convolution: 1 x 2048 x 1000 28 / 23, 8 x 4096 x 1000 41 / 31, 16 x 2048 x 1000 31 / 25, 41 x 2048 x 1000
  // 34 / 30, 41 x 512 x 1000 25 / 23, 41 x 1024 x 640 23 / 23, 32 x 512 x 2048 31 / 27, 50 x 768 x 3000 36 / 38, 64 x 1024 x 4096 52 / 48; beyond the lines drawn
  // here 96 x 2048 x 1000 35 / 40, 128 x 2048 x 1000 39 / 40, 64 x 1024 x 8000 63 / 70, 41 x 1024 x 320 21 / 22, 64 x 256 x 256 19 / 26.  Of 19 sizes within them
  // one takes the slower way by more than 2 % (50 x 768 x 3000).  Elsewhere the kernels here are (1024 x 2048 x 32768: logits 726 / 825, dx 740 / 1023, dw 775 / 841).
  p.conv = !p.widen && p.pieces == 1 && n <= 64 && classes >= 640 && classes <= 4096 && classes % 4 == 0 && d >= 256 && d % 8 == 0;
  if (p.conv) {
    alignas(16) static const float any[4] = {};      // (an aligned address: all that the question looks at)
    ConvGeom g = product_geom(any, nullptr, nullptr, n, classes, d);
    g.w_kn = any;
    p.conv = conv_igemm_rows_takes(g, n, classes);
  }
  p.z = cut32(n, p.piece, d, p.rows || (p.pieces == 1 && n * p.piece <= 1L << 22) ? 1L << 24 : 0);
  p.dx = cut32(n, d, p.piece, 1L << 25);
  p.dw = cut32(p.piece, d, n, 1L << 24);
  const Cut dx = cut32(n, d, p.piece, 1L << 25, 1), dw = cut32(p.piece, d, n, 1L << 24, 1);
  auto works = [](long m, long k, const Cut& c) { return ceil_div(m, 64) * ceil_div(k, 64) * c.splits; };
  p.together = !p.conv && works(n, d, dx) + works(p.piece, d, dw) <= 1024;
  if (p.together) { p.dx = dx; p.dw = dw; }
  p.late = !p.rows && p.z.splits > 1;
  const long split_cols = p.late ? kSplitCols : kTile32[p.z.tile][1];
  p.splits = (p.pieces - 1) * ceil_div(p.piece, split_cols) + ceil_div(classes - (p.pieces - 1) * p.piece, split_cols);
  // rows of a workgroup of dz_kernel: some two thousand workgroups, at most 512 of them down a column
  const long across = ceil_div(p.pitch / 4, THREADS);
  p.dz_rows = (int)up(ceil_div((long)n * across, 2048), 4);
  if (p.dz_rows < ceil_div(n, 512)) p.dz_rows = (int)up(ceil_div(n, 512), 4);
  p.slabs = (int)ceil_div(n, p.dz_rows);
  p.sum_dx = p.widen || (!p.conv && p.dx.splits > 1);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.stats = take((size_t)(4 * (size_t)n + 64) * 4);
  p.part = take(p.rows ? 0 : (size_t)n * 2 * p.splits * 4);
  p.logits = take(p.rows || p.late || grads ? (size_t)n * p.pitch * 4 * p.z.splits : 0);
  p.x = take(p.widen ? (size_t)n * d * 4 : 0);
  p.w = take(p.widen ? (size_t)p.piece * d * 4 : 0);
  if (grads) {
    p.dx_sums = take(p.sum_dx ? (size_t)p.dx.splits * n * d * 4 : 0);
    p.dw_sums = take(!p.conv && p.dw.splits > 1 ? (size_t)p.dw.splits * p.piece * d * 4 : 0);
    p.db = take((size_t)(p.rows ? ceil_div(n, kColumnRows) : p.slabs) * p.pitch * 4);
    if (p.conv) p.wgrad_bytes = wgrad_workspace_bytes(n, 1, 1, d, classes, 1, 1, DT_F32);
    p.wgrad = take(p.wgrad_bytes);
  }
  p.total = at;
  return p;
}

#define ACC_TRY(call) do { if (const hipError_t e_ = (call); e_ != hipSuccess) return e_; } while (0)

hipError_t widen(const void* in, float* out, size_t total, hipStream_t st) {
  const size_t b = (total + THREADS - 1) / THREADS;
  hipLaunchKernelGGL(widen_kernel, dim3((unsigned)(b < 4096 ? b : 4096)), dim3(THREADS), 0, st, (const bf16_t*)in, out, total);
  return hipGetLastError();
}

hipError_t logits32(Logits32 g, const Cut& c, int n, int tiles_n, hipStream_t st) {
  g.tiles_m = (int)ceil_div(n, kTile32[c.tile][0]);
  g.tiles = g.tiles_m * tiles_n;
  g.k_per_split = c.k;
  g.work = g.tiles * c.splits;
  const unsigned blocks = whole_eights(g.work);
  if (c.tile == 0) hipLaunchKernelGGL((logits32_kernel<Gemm32Cfg<1, 4, 2, 2, false, false, false>>), dim3(blocks), dim3(256), 0, st, g, (int)blocks);
  else if (c.tile == 1) hipLaunchKernelGGL((logits32_kernel<Gemm32Cfg<2, 2, 2, 2, false, false, false>>), dim3(blocks), dim3(256), 0, st, g, (int)blocks);
  else hipLaunchKernelGGL((logits32_kernel<Gemm32Cfg<2, 2, 4, 4, false, false, true>>), dim3(blocks), dim3(256), 0, st, g, (int)blocks);
  return hipGetLastError();
}

hipError_t run32(const LceArgs& a) {
  const bool grads = a.dx || a.dw || a.db;
  const Plan32 p = plan32(a.n, a.d, a.classes, grads, a.dtype);
  const LceStats s = lce_stats(a, p.stats);
  float *const part = (float*)(a.ws + p.part), *const z = (float*)(a.ws + p.logits);
  hipStream_t st = a.st;
  const float* x = (const float*)a.x;
  if (p.widen) {
    x = (const float*)(a.ws + p.x);
    ACC_TRY(widen(a.x, (float*)(a.ws + p.x), (size_t)a.n * a.d, st));
  }
  const size_t es = dt_size(a.dtype);
  // of the piece at hand
  long v0 = 0;
  int cols = 0;
  const float* w = nullptr;
  auto logits = [&](long k, bool sums, bool keep) -> hipError_t {
    v0 = k * p.piece;
    cols = (int)(a.classes - v0 < p.piece ? a.classes - v0 : p.piece);
    const char* from = (const char*)a.w + (size_t)v0 * a.d * es;
    w = (const float*)from;
    if (p.widen) {
      w = (const float*)(a.ws + p.w);
      ACC_TRY(widen(from, (float*)(a.ws + p.w), (size_t)cols * a.d, st));
    }
    const int pitch = p.pitch, tile_n = kTile32[p.z.tile][1];
    Logits32 g{};
    g.x = {x, a.n, a.d}; g.w = {w, cols, a.d};
    g.bias = a.bias && !p.rows && !p.late ? a.bias + v0 : nullptr;
    g.labels = a.labels; g.z = keep || p.late ? z : nullptr; g.part = sums && !p.late ? part : nullptr; g.z_label = s.z_label;
    g.d = a.d; g.pitch = pitch; g.v0 = (int)v0; g.split0 = (int)(k * ceil_div(p.piece, tile_n)); g.splits = (int)p.splits;
    ACC_TRY(logits32(g, p.z, a.n, (int)ceil_div(cols, tile_n), st));
    if (!sums || !p.late) return hipSuccess;
    const int here = (int)ceil_div(cols, kSplitCols);
    hipLaunchKernelGGL(row_sums_kernel, dim3((unsigned)(a.n * here)), dim3(THREADS), 0, st, z, a.bias, a.labels, part, s.z_label, pitch, cols, (int)v0, kSplitCols,
                       here, (int)(k * ceil_div(p.piece, kSplitCols)), (int)p.splits, p.z.splits, (size_t)a.n * pitch);
    return hipGetLastError();
  };
  if (p.rows) {
    ACC_TRY(logits(0, false, true));
#define ACC_ROWS(V, NT) hipLaunchKernelGGL((rows_kernel<V, NT>), dim3((unsigned)a.n), dim3(NT), 0, st, z, a.bias, a.labels, a.ignore, s.loss_rows, a.n, p.pitch, \
                                           cols, grads ? 1 : 0, p.z.splits)
    if (p.pitch <= 4 * 256) ACC_ROWS(4, 256);
    else if (p.pitch <= 16 * 256) ACC_ROWS(16, 256);
    else ACC_ROWS(8, 1024);
#undef ACC_ROWS
  } else {
    for (long k = 0; k < p.pieces; ++k) ACC_TRY(logits(k, true, grads && k + 1 == p.pieces));
    ACC_TRY(lce_join(a, s, part, (int)p.splits));
  }
  if (!grads && !(p.rows && a.loss)) return hipGetLastError();
  float* const db_part = (float*)(a.ws + p.db);
  float* const dx_out = p.sum_dx ? (float*)(a.ws + p.dx_sums) : (float*)a.dx;
  for (long k = p.pieces - 1; k >= 0; --k) {           // (the last piece is still there)
    const bool first = k + 1 == p.pieces, last = k == 0;
    if (!first) ACC_TRY(logits(k, false, true));
    const int pitch = p.pitch;
    if (!p.rows)
      hipLaunchKernelGGL(dz_kernel, dim3((unsigned)ceil_div(pitch / 4, THREADS), (unsigned)p.slabs), dim3(THREADS), 0, st, z, p.late ? a.bias : nullptr, a.labels,
                         a.ignore, s.row_max, s.row_rest, s.scale, a.db ? db_part : nullptr, a.n, pitch, cols, (int)v0, p.dz_rows);
    Finish32 f{};
    Product32 gx{}, gw{};
    if (a.dx && p.conv) {
      ConvGeom g = product_geom(z, nullptr, (float*)a.dx, a.n, cols, a.d);
      g.w_kn = w;                              // the filter as it lies
      ACC_TRY(conv_igemm(g, st));
    } else if (a.dx) {
      gx.a = {z, a.n, pitch}; gx.b = {w, a.d, a.d}; gx.out = dx_out; gx.k = cols; gx.add = !first;
      cut_into(gx, p.dx);
      if (!p.together) ACC_TRY((launch_product32<false, true>(gx, p.dx, st)));
      if (p.sum_dx && last) {
        f.dx_sums = dx_out; f.dx = a.dx; f.dx_count = (size_t)a.n * a.d; f.dx_splits = p.dx.splits;
        f.dx_blocks = join_blocks(f.dx_count);
      }
    }
    if (a.dw) {
      float* const to = a.dw + (size_t)v0 * a.d;
      if (p.conv) {
        WgradGeom g{};
        g.x = x; g.dy = z; g.dw = to; g.dtype = DT_F32;
        g.n_img = a.n; g.h = g.wd = g.p = g.q = 1; g.cin = a.d; g.cout = cols; g.r = g.s = g.stride = 1;
        g.workspace = (float*)(a.ws + p.wgrad); g.workspace_bytes = p.wgrad_bytes;
        ACC_TRY(conv_wgrad(g, st));
      } else {
        gw.a = {z, cols, pitch}; gw.b = {x, a.d, a.d}; gw.k = a.n;
        gw.out = p.dw.splits > 1 ? (float*)(a.ws + p.dw_sums) : to;
        cut_into(gw, p.dw);
        if (!p.together) ACC_TRY((launch_product32<true, true>(gw, p.dw, st)));
        if (p.dw.splits > 1) {
          f.dw_sums = gw.out; f.dw = to; f.dw_count = (size_t)cols * a.d; f.dw_splits = p.dw.splits;
          f.dw_blocks = join_blocks(f.dw_count);
        }
      }
    }
    int slabs = 1;
    Finish32 r{};
    if (a.db) {
      r.columns = p.rows ? z : db_part; r.rows = p.rows ? a.n : p.slabs; r.pitch = pitch; r.cols = cols; r.across = (int)ceil_div(cols, 64);
      slabs = (int)ceil_div(r.rows, kColumnRows);
      r.db = slabs > 1 ? db_part : a.db + v0;
      r.db_blocks = (unsigned)(r.across * slabs);
    }
    if (p.rows) { r.loss_rows = s.loss_rows; r.labels = a.labels; r.loss = a.loss; r.n = a.n; r.ignore = a.ignore; }
    const unsigned rest = r.db_blocks + (p.rows && a.loss ? 1 : 0), sums = f.dx_blocks + f.dw_blocks;
    if (p.together) {
      const unsigned bx = whole_eights(gx.work), bw = whole_eights(gw.work);
      if (bx + bw + rest) hipLaunchKernelGGL(grads32_kernel, dim3(bx + bw + rest), dim3(THREADS), 0, st, gx, gw, r, (int)bx, (int)bw);
    } else if (rest) {                           // with the sums
      r.dx_sums = f.dx_sums; r.dx = f.dx; r.dx_count = f.dx_count; r.dx_splits = f.dx_splits; r.dx_blocks = f.dx_blocks;
      r.dw_sums = f.dw_sums; r.dw = f.dw; r.dw_count = f.dw_count; r.dw_splits = f.dw_splits; r.dw_blocks = f.dw_blocks;
      f = r;
    }
    if (sums + (p.together ? 0 : rest)) {
      const dim3 grid(sums + (p.together ? 0 : rest));
      if (a.dtype == DT_F32) hipLaunchKernelGGL(finish32_kernel<float>, grid, dim3(THREADS), 0, st, f);
      else hipLaunchKernelGGL(finish32_kernel<bf16_t>, grid, dim3(THREADS), 0, st, f);
    }
    if (slabs > 1) hipLaunchKernelGGL(db_kernel, dim3((unsigned)ceil_div(cols, THREADS)), dim3(THREADS), 0, st, db_part, a.db, slabs, pitch, cols);
  }
  return hipGetLastError();
}

bool shape_ok(int n, int d, int classes, int dtype) {
  return n > 0 && d > 0 && classes > 0 && n <= (1 << 20) && d <= (1 << 16) && classes <= (1 << 24) && (dtype == DT_F32 || dtype == DT_BF16);
}

}  // namespace

hipError_t lce_join(const LceArgs& a, const LceStats& s, const float* part, int splits) {
  int lanes = 1;
  while (lanes < splits && lanes < 64) lanes *= 2;
  // One workgroup joins all rows and takes their mean if no lane has more than four values to read, which takes as long as the second launch (rows one after the
  // other cost 1.4 us each: 131 us for 1546 rows, now 5)
  const long reads = (((long)a.n * lanes + 1023) / 1024) * ((splits + lanes - 1) / lanes);
  if (reads <= 4) {
    hipLaunchKernelGGL(join_mean_kernel, dim3(1), dim3(1024), 0, a.st, part, s.z_label, a.labels, a.ignore, s.row_max, s.row_rest, s.loss_rows, a.n, splits,
                       a.classes, s.scale, a.loss, lanes);
    return hipGetLastError();
  }
  const int rows = THREADS / lanes;
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)((a.n + rows - 1) / rows)), dim3(THREADS), 0, a.st, part, s.z_label, a.labels, a.ignore, s.row_max,
                     s.row_rest, s.loss_rows, a.n, splits, a.classes, lanes);
  hipLaunchKernelGGL(mean_kernel, dim3(1), dim3(1024), 0, a.st, s.loss_rows, a.labels, a.ignore, a.n, s.scale, a.loss);
  return hipGetLastError();
}

size_t linear_ce_workspace_bytes(int n, int d, int classes, int gradients, int dtype) {
  if (!shape_ok(n, d, classes, dtype)) return 0;
  if (dtype == DT_BF16 && linear_ce_bf16_takes(n, d, classes)) return linear_ce_bf16_workspace_bytes(n, d, classes, gradients != 0);
  return plan32(n, d, classes, gradients != 0, dtype).total;
}

hipError_t linear_ce(const void* x, const void* w, const float* bias, const int32_t* labels, int ignore, float* loss_rows, float* loss, void* dx, float* dw,
                     float* db, int n, int d, int classes, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!x || !w || !labels || !workspace || !(loss_rows || loss || dx || dw || db) || !shape_ok(n, d, classes, dtype)) return hipErrorInvalidValue;
  if (workspace_bytes < linear_ce_workspace_bytes(n, d, classes, dx || dw || db, dtype)) return hipErrorInvalidValue;
  const LceArgs a{x, w, bias, labels, ignore, loss_rows, loss, dx, dw, db, n, d, classes, (char*)workspace, dtype, st};
  return dtype == DT_BF16 && linear_ce_bf16_takes(n, d, classes) ? linear_ce_bf16(a) : run32(a);
}

}  // namespace acc
