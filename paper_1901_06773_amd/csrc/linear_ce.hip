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
// fp32: products of the convolution kernels (a 1x1 convolution of n pixels), logits and dz of a piece in fp32.
#include "kernels.h"
#include "dtype.h"
#include "linear_ce.h"

#include <climits>

namespace acc {
namespace {

constexpr int THREADS = 256;

inline size_t al256(size_t b) { return (b + 255) & ~(size_t)255; }
inline long up(long v, long m) { return (v + m - 1) / m * m; }

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

// m and R of the columns [lo, hi) of a row: part[row][2][splits].  A workgroup's columns are whole splits.
__global__ __launch_bounds__(THREADS) void row_sums_kernel(const float* __restrict__ z, const float* __restrict__ bias, const int32_t* __restrict__ labels,
                                                           float* __restrict__ part, float* __restrict__ z_label, int pitch, int cols, int v0,
                                                           int per_split, int splits_here, int split0, int splits) {
  __shared__ float sh[THREADS / 64];
  const int row = blockIdx.x / splits_here, sp = blockIdx.x - row * splits_here;
  const int lo = sp * per_split, hi = min(lo + per_split, cols);
  const float* zr = z + (size_t)row * pitch;
  float mx = -INFINITY;
  for (int j = lo + threadIdx.x; j < hi; j += THREADS) mx = fmaxf(mx, zr[j] + (bias ? bias[v0 + j] : 0.f));
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
    const long at = (long)labels[row] - v0;
    if (at >= lo && at < hi) z_label[row] = zr[at] + (bias ? bias[v0 + at] : 0.f);
  }
}

// One wave per row: the splits' m and R joined.
__device__ __forceinline__ float join_row(const float* __restrict__ part, const float* __restrict__ z_label, const int32_t* __restrict__ labels, int ignore,
                                          float* __restrict__ row_max, float* __restrict__ row_rest, int row, int splits, int classes) {
  const int lane = threadIdx.x & 63;
  const float* p = part + (size_t)row * 2 * splits;
  float mx = -INFINITY;
  for (int i = lane; i < splits; i += 64) mx = fmaxf(mx, p[i]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  float s = 0.f, equal = 0.f;
  for (int i = lane; i < splits; i += 64) {
    const bool top = p[i] == mx;
    equal += top ? 1.f : 0.f;
    s += top ? p[splits + i] : (1.f + p[splits + i]) * expf(p[i] - mx);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { s += __shfl_xor(s, o); equal += __shfl_xor(equal, o); }
  const float rest = mx == -INFINITY ? NAN : s + (equal - 1.f);     // (every class ruled out: no distribution)
  const int lab = labels[row];
  const bool skip = ignore != INT_MIN && lab == ignore, known = (unsigned)lab < (unsigned)classes;
  if (lane == 0) {
    row_max[row] = mx;
    row_rest[row] = rest;
  }
  return skip ? 0.f : known ? log1pf(rest) - (z_label[row] - mx) : NAN;
}
__global__ __launch_bounds__(THREADS) void join_kernel(const float* __restrict__ part, const float* __restrict__ z_label, const int32_t* __restrict__ labels,
                                                       int ignore, float* __restrict__ row_max, float* __restrict__ row_rest, float* __restrict__ loss_rows,
                                                       int n, int splits, int classes) {
  const int row = blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
  if (row >= n) return;
  const float l = join_row(part, z_label, labels, ignore, row_max, row_rest, row, splits, classes);
  if ((threadIdx.x & 63) == 0) loss_rows[row] = l;
}

// scale[0] = 1 / rows that count (0 if there is none), loss = their mean, of NT threads and in a fixed order.  Either may be null.
template <int NT>
__device__ __forceinline__ void mean_of_rows(const float* loss_rows, const int32_t* __restrict__ labels, int ignore, int n, float* __restrict__ scale,
                                             float* __restrict__ loss) {
  __shared__ double sh[NT / 64];
  __shared__ int counts[NT / 64];
  double s = 0.0;
  int k = 0;
  for (int i = threadIdx.x; i < n; i += NT) {
    s += (double)loss_rows[i];
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
__global__ __launch_bounds__(1024) void mean_kernel(const float* __restrict__ loss_rows, const int32_t* __restrict__ labels, int ignore, int n,
                                                    float* __restrict__ scale, float* __restrict__ loss) {
  mean_of_rows<1024>(loss_rows, labels, ignore, n, scale, loss);
}
// both, in one workgroup
__global__ __launch_bounds__(1024) void join_mean_kernel(const float* __restrict__ part, const float* __restrict__ z_label, const int32_t* __restrict__ labels,
                                                         int ignore, float* __restrict__ row_max, float* __restrict__ row_rest, float* loss_rows, int n,
                                                         int splits, int classes, float* __restrict__ scale, float* __restrict__ loss) {
  for (int row = threadIdx.x >> 6; row < n; row += 16) {
    const float l = join_row(part, z_label, labels, ignore, row_max, row_rest, row, splits, classes);
    if ((threadIdx.x & 63) == 0) loss_rows[row] = l;
  }
  __threadfence_block();
  __syncthreads();
  mean_of_rows<1024>(loss_rows, labels, ignore, n, scale, loss);
}

// A whole row of logits at once, one workgroup per row, up to V values in a thread's registers: the loss, and with `grads` z -> dz in place, columns beyond
// the classes zero.  The rows that count are counted by every workgroup, while its logits are on their way.
template <int V, int NT>
__global__ __launch_bounds__(NT) void rows_kernel(float* __restrict__ z, const float* __restrict__ bias, const int32_t* __restrict__ labels, int ignore,
                                                  float* __restrict__ loss_rows, int n, int pitch, int cols, int grads) {
  __shared__ float sh[3][NT / 64];
  __shared__ int counted;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float* const zr = z + (size_t)row * pitch;
  float v[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int j = tid + u * NT;
    v[u] = j < cols ? zr[j] : -INFINITY;
  }
  if (bias) {
#pragma unroll
    for (int u = 0; u < V; ++u) {
      const int j = tid + u * NT;
      if (j < cols) v[u] += bias[j];
    }
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

// The columns' sums of dz over `per` rows each (straight to db where that is all of them), and in a workgroup of its own the mean loss.
__global__ __launch_bounds__(THREADS) void columns_kernel(const float* __restrict__ dz, float* __restrict__ out, int n, int pitch, int cols, int per, int blocks,
                                                          int stride, const float* __restrict__ loss_rows, const int32_t* __restrict__ labels, int ignore,
                                                          float* __restrict__ loss) {
  if ((int)blockIdx.x >= blocks) {
    mean_of_rows<THREADS>(loss_rows, labels, ignore, n, nullptr, loss);
    return;
  }
  const int across = (cols + THREADS - 1) / THREADS, slab = blockIdx.x / across, j = (blockIdx.x - slab * across) * THREADS + threadIdx.x;
  if (j >= cols) return;
  double s = 0.0;
  int r = slab * per;
  const int end = min(r + per, n);
  for (; r + 16 <= end; r += 16) {
    float v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = dz[(size_t)(r + u) * pitch + j];
#pragma unroll
    for (int u = 0; u < 16; ++u) s += (double)v[u];
  }
  for (; r < end; ++r) s += (double)dz[(size_t)r * pitch + j];
  out[(size_t)slab * stride + j] = (float)s;
}

// z -> dz in place, columns beyond the classes zero, and the columns' sums over the rows of a workgroup: db_part[workgroup][pitch].
constexpr int DZ_ROWS = 32;
__global__ __launch_bounds__(THREADS) void dz_kernel(float* __restrict__ z, const float* __restrict__ bias, const int32_t* __restrict__ labels, int ignore,
                                                     const float* __restrict__ row_max, const float* __restrict__ row_rest, const float* __restrict__ scale,
                                                     float* __restrict__ db_part, int n, int pitch, int cols, int v0) {
  const int j = (blockIdx.x * THREADS + threadIdx.x) * 4;
  if (j >= pitch) return;
  const int r0 = blockIdx.y * DZ_ROWS, r1 = min(r0 + DZ_ROWS, n);
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
  *reinterpret_cast<float4*>(db_part + (size_t)blockIdx.y * pitch + j) = make_float4(sum[0], sum[1], sum[2], sum[3]);
}

__global__ __launch_bounds__(THREADS) void db_kernel(const float* __restrict__ part, float* __restrict__ db, int parts, int pitch, int cols) {
  const int j = blockIdx.x * THREADS + threadIdx.x;
  if (j >= cols) return;
  double s = 0.0;
  for (int k = 0; k < parts; ++k) s += (double)part[(size_t)k * pitch + j];
  db[j] = (float)s;
}

// ---------------------------------------------------------------------------------- copies that make widths whole
// out[r][c] (fp32, rows x cols, pitch = cols) = in[r][c] where that exists, else 0
template <class T>
__global__ __launch_bounds__(THREADS) void widen_kernel(const T* __restrict__ in, float* __restrict__ out, int rows_in, int cols_in, size_t total, int cols) {
  for (size_t i = (size_t)blockIdx.x * THREADS + threadIdx.x; i < total; i += (size_t)gridDim.x * THREADS) {
    const size_t r = i / cols, c = i - r * cols;
    out[i] = r < (size_t)rows_in && c < (size_t)cols_in ? Elem<T>::load(in + r * cols_in + c) : 0.f;
  }
}
template <class T>
__global__ __launch_bounds__(THREADS) void narrow_kernel(const float* __restrict__ in, T* __restrict__ out, size_t total, int cols_out, int cols_in) {
  for (size_t i = (size_t)blockIdx.x * THREADS + threadIdx.x; i < total; i += (size_t)gridDim.x * THREADS) {
    const size_t r = i / cols_out, c = i - r * cols_out;
    Elem<T>::store(out + i, in[r * cols_in + c]);
  }
}
inline unsigned grid_for(size_t total) {
  const size_t b = (total + THREADS - 1) / THREADS;
  return (unsigned)(b < 256 * 16 ? b : 256 * 16);
}

// ---------------------------------------------------------------------------------- fp32
constexpr int kRowCols = 8192;                 // columns that a workgroup keeps as a whole row
constexpr int kColumnRows = 256;               // rows that one workgroup adds up per column
constexpr int kSplitCols = 4096;               // columns of a row that one workgroup adds up

inline long whole(long v) { return v < 16 ? 16 : up(v, 4); }   // widths that the fast kernels take

struct Plan32 {
  long dp, piece, pieces, splits, row_parts;   // width of x as it is multiplied, classes of a piece, ...
  bool rows;                                   // one piece of at most kRowCols classes
  bool own_x, own_w;                           // x resp. the filter of some piece is copied to make its widths whole (or to fp32)
  size_t part, stats, z, x, w, wt, dx, dw, db, wgrad, total;   // offsets of the parts of the workspace, and its size
  size_t wgrad_bytes;
  long cols(long k, int classes) const { return classes - k * piece < piece ? classes - k * piece : piece; }
};

Plan32 plan32(int n, int d, int classes, bool grads, int dtype) {
  Plan32 p{};
  p.dp = whole(d);
  // 256 MiB of logits, 1 GiB of filter, and what the transposing launch takes
  long most = (1L << 26) / n / 64 * 64;
  if (most > (1L << 28) / p.dp / 64 * 64) most = (1L << 28) / p.dp / 64 * 64;
  if (most > 1L << 20) most = 1L << 20;
  if (most < 64) most = 64;
  p.piece = classes <= most ? classes : most;
  p.pieces = (classes + p.piece - 1) / p.piece;
  const long last = p.cols(p.pieces - 1, classes), widest = whole(p.piece);
  p.splits = p.pieces * ((p.piece + kSplitCols - 1) / kSplitCols);
  p.row_parts = (n + DZ_ROWS - 1) / DZ_ROWS;
  p.rows = p.pieces == 1 && p.piece <= kRowCols && n <= 16384;
  p.own_x = dtype != DT_F32 || p.dp != d;
  p.own_w = p.own_x || whole(last) != last;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.stats = take((size_t)(4 * (size_t)n + 64) * 4);
  p.part = take((size_t)n * 2 * p.splits * 4);
  p.z = take((size_t)n * widest * 4);
  p.x = take(p.own_x ? (size_t)n * p.dp * 4 : 0);
  p.w = take(p.own_w ? (size_t)widest * p.dp * 4 : 0);
  if (grads) {
    p.wt = take((size_t)widest * p.dp * 4);
    p.dx = take(p.own_x ? (size_t)n * p.dp * 4 : 0);
    p.dw = take(p.dp != d || whole(last) != last ? (size_t)widest * p.dp * 4 : 0);
    p.db = take((size_t)p.row_parts * widest * 4);
    p.wgrad_bytes = wgrad_workspace_bytes(n, 1, 1, (int)p.dp, (int)widest, 1, 1, DT_F32);
    const size_t tail = wgrad_workspace_bytes(n, 1, 1, (int)p.dp, (int)whole(last), 1, 1, DT_F32);
    if (tail > p.wgrad_bytes) p.wgrad_bytes = tail;
    p.wgrad = take(p.wgrad_bytes);
  }
  p.total = at;
  return p;
}

#define ACC_TRY(call) do { if (const hipError_t e_ = (call); e_ != hipSuccess) return e_; } while (0)

// out[n][n_out] (+)= in[n][c] * w[n_out][c]^T
ConvGeom product_geom(const float* in, const float* w, float* out, int n, int c, int n_out, bool accumulate) {
  ConvGeom g{};
  g.in = in; g.w = w; g.out = out; g.dtype = DT_F32;
  g.n_img = n; g.h = g.wd = g.p = g.q = g.out_h = g.out_w = 1;
  g.c = c; g.n_out = n_out; g.r = g.s = g.stride = g.out_stride = 1; g.accumulate = accumulate ? 1 : 0;
  return g;
}

hipError_t widen(const void* in, int dtype, float* out, int rows_in, int cols_in, long rows, long cols, hipStream_t st) {
  const size_t total = (size_t)rows * cols;
  if (dtype == DT_F32)
    hipLaunchKernelGGL(widen_kernel<float>, dim3(grid_for(total)), dim3(THREADS), 0, st, (const float*)in, out, rows_in, cols_in, total, (int)cols);
  else
    hipLaunchKernelGGL(widen_kernel<bf16_t>, dim3(grid_for(total)), dim3(THREADS), 0, st, (const bf16_t*)in, out, rows_in, cols_in, total, (int)cols);
  return hipGetLastError();
}

hipError_t run32(const LceArgs& a) {
  const bool grads = a.dx || a.dw || a.db;
  const Plan32 p = plan32(a.n, a.d, a.classes, grads, a.dtype);
  const LceStats s = lce_stats(a, p.stats);
  float *const part = (float*)(a.ws + p.part), *const z = (float*)(a.ws + p.z);
  const int dp = (int)p.dp;
  hipStream_t st = a.st;
  const float* x = (const float*)a.x;
  if (p.own_x) {
    x = (const float*)(a.ws + p.x);
    ACC_TRY(widen(a.x, a.dtype, (float*)(a.ws + p.x), a.n, a.d, a.n, dp, st));
  }
  const size_t es = dt_size(a.dtype);
  // of the piece at hand
  long v0 = 0;
  int cols = 0, pitch = 0;
  const float* w = nullptr;
  auto logits = [&](long k) -> hipError_t {
    v0 = k * p.piece;
    cols = (int)p.cols(k, a.classes);
    pitch = (int)whole(cols);
    const char* from = (const char*)a.w + (size_t)v0 * a.d * es;
    w = (const float*)from;
    if (p.own_x || pitch != cols) {
      w = (const float*)(a.ws + p.w);
      ACC_TRY(widen(from, a.dtype, (float*)(a.ws + p.w), cols, a.d, pitch, dp, st));
    }
    return conv_igemm(product_geom(x, w, z, a.n, dp, pitch, false), st);
  };
  float* const db_part = (float*)(a.ws + p.db);
  float* const dx = p.own_x ? (float*)(a.ws + p.dx) : (float*)a.dx;
  if (p.rows) {
    ACC_TRY(logits(0));
#define ACC_ROWS(V, NT) hipLaunchKernelGGL((rows_kernel<V, NT>), dim3((unsigned)a.n), dim3(NT), 0, st, z, a.bias, a.labels, a.ignore, s.loss_rows, a.n, pitch, \
                                           cols, grads ? 1 : 0)
    if (pitch <= 4 * 256) ACC_ROWS(4, 256);
    else if (pitch <= 16 * 256) ACC_ROWS(16, 256);
    else ACC_ROWS(8, 1024);
#undef ACC_ROWS
    const int across = (cols + THREADS - 1) / THREADS, slabs = (a.n + kColumnRows - 1) / kColumnRows, blocks = a.db ? across * slabs : 0;
    if (a.db || a.loss)
      hipLaunchKernelGGL(columns_kernel, dim3((unsigned)(blocks + (a.loss ? 1 : 0))), dim3(THREADS), 0, st, z, slabs > 1 ? db_part : a.db, a.n, pitch, cols, kColumnRows,
                         blocks, pitch, s.loss_rows, a.labels, a.ignore, a.loss);
    if (a.db && slabs > 1)
      hipLaunchKernelGGL(db_kernel, dim3((unsigned)across), dim3(THREADS), 0, st, db_part, a.db, slabs, pitch, cols);
    ACC_TRY(hipGetLastError());
    if (!grads) return hipSuccess;
  } else {
    const int splits_piece = (int)((p.piece + kSplitCols - 1) / kSplitCols);
    for (long k = 0; k < p.pieces; ++k) {
      ACC_TRY(logits(k));
      hipLaunchKernelGGL(row_sums_kernel, dim3((unsigned)(a.n * splits_piece)), dim3(THREADS), 0, st, z, a.bias, a.labels, part, s.z_label, pitch, cols,
                         (int)v0, kSplitCols, splits_piece, (int)(k * splits_piece), (int)p.splits);
    }
    ACC_TRY(lce_join(a, s, part, (int)p.splits));
    if (!grads) return hipSuccess;
  }
  for (long k = 0; k < p.pieces; ++k) {
    if (p.pieces > 1) ACC_TRY(logits(k));
    if (!p.rows) {
      hipLaunchKernelGGL(dz_kernel, dim3((unsigned)((pitch / 4 + THREADS - 1) / THREADS), (unsigned)p.row_parts), dim3(THREADS), 0, st, z, a.bias, a.labels,
                         a.ignore, s.row_max, s.row_rest, s.scale, db_part, a.n, pitch, cols, (int)v0);
      if (a.db)
        hipLaunchKernelGGL(db_kernel, dim3((unsigned)((cols + THREADS - 1) / THREADS)), dim3(THREADS), 0, st, db_part, a.db + v0, (int)p.row_parts, pitch,
                           cols);
    }
    if (a.dx) {
      ConvGeom g = product_geom(z, nullptr, dx, a.n, pitch, dp, k > 0);
      g.w_kn = w;                              // few rows: the filter as it lies
      if (!conv_igemm_rows_takes(g, a.n, pitch)) {
        float* const wt = (float*)(a.ws + p.wt);
        ACC_TRY(filter_flip_transpose(w, wt, pitch, dp, 1, 1, DT_F32, st));
        g = product_geom(z, wt, dx, a.n, pitch, dp, k > 0);
      }
      ACC_TRY(conv_igemm(g, st));
    }
    if (a.dw) {
      float* const to = a.dw + (size_t)v0 * a.d;
      const bool own = dp != a.d || pitch != cols;
      WgradGeom g{};
      g.x = x; g.dy = z; g.dw = own ? (float*)(a.ws + p.dw) : to; g.dtype = DT_F32;
      g.n_img = a.n; g.h = g.wd = g.p = g.q = 1; g.cin = dp; g.cout = pitch; g.r = g.s = g.stride = 1;
      g.workspace = (float*)(a.ws + p.wgrad); g.workspace_bytes = p.wgrad_bytes;
      ACC_TRY(conv_wgrad(g, st));
      const size_t total = (size_t)cols * a.d;
      if (own) hipLaunchKernelGGL(narrow_kernel<float>, dim3(grid_for(total)), dim3(THREADS), 0, st, g.dw, to, total, a.d, dp);
    }
  }
  if (a.dx && p.own_x) {
    const size_t total = (size_t)a.n * a.d;
    if (a.dtype == DT_F32)
      hipLaunchKernelGGL(narrow_kernel<float>, dim3(grid_for(total)), dim3(THREADS), 0, st, dx, (float*)a.dx, total, a.d, dp);
    else
      hipLaunchKernelGGL(narrow_kernel<bf16_t>, dim3(grid_for(total)), dim3(THREADS), 0, st, dx, (bf16_t*)a.dx, total, a.d, dp);
  }
  return hipGetLastError();
}

bool shape_ok(int n, int d, int classes, int dtype) {
  return n > 0 && d > 0 && classes > 0 && n <= (1 << 20) && d <= (1 << 16) && classes <= (1 << 24) && (dtype == DT_F32 || dtype == DT_BF16);
}

}  // namespace

hipError_t lce_join(const LceArgs& a, const LceStats& s, const float* part, int splits) {
  if ((long)a.n * splits <= 16384) {          // a few rows for each of sixteen waves: one launch
    hipLaunchKernelGGL(join_mean_kernel, dim3(1), dim3(1024), 0, a.st, part, s.z_label, a.labels, a.ignore, s.row_max, s.row_rest, s.loss_rows, a.n, splits,
                       a.classes, s.scale, a.loss);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(join_kernel, dim3((a.n + THREADS / 64 - 1) / (THREADS / 64)), dim3(THREADS), 0, a.st, part, s.z_label, a.labels, a.ignore, s.row_max,
                     s.row_rest, s.loss_rows, a.n, splits, a.classes);
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
