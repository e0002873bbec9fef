// Norm over all values of a list of tensors, and the tensors scaled so that it does not exceed a bound:
//
//   N = (sum over all tensors of g^2)^(1/2),   out = g * (N <= bound ? 1 : bound / N).
//
// Bound by memory: every value is read for the norm, and read again and written for the scaled tensors.  Gradients of ResNet-152 (311 tensors, 241 MB): 36 us
// for the norm (part of them still in the memory-side cache), 73 for the scaling (6.6 TB/s with the same help); 117 in all.
//
// The list is a table in the caller's device memory, written once (tensor_list): the tensors cut into pieces of 16384 values at most,
// so that a launch covers hundreds of tensors of any size, and every workgroup finds its next piece with one load.  Pieces are dealt
// out in turn to as many workgroups as there are pieces, 2048 at most; a workgroup leaves one sum in fp64, and the scaling launch
// adds these in a fixed order in every workgroup: no atomics, the same bits on every run.  Squares are exact in fp64 and their sums
// neither overflow nor lose small tensors beside large ones.
#include "kernels.h"
#include "dtype.h"

namespace acc {
namespace {

constexpr int THREADS = 256;
constexpr uint32_t kMagic = 0x61636c31u;
constexpr int kMaxSums = 2048;                 // workgroups of a launch = sums in the workspace

struct ListHeader {
  uint32_t magic, pieces;
  uint32_t pad[14];
};
static_assert(sizeof(ListHeader) == 64, "pieces start on a line");
struct Piece {
  const void* src;
  void* dst;
  uint32_t count, dtype;
};
static_assert(sizeof(Piece) == 24, "table layout");

// One batch of tensors, handed over in the launch's arguments: the table needs no copy from the host and may be written under capture.
constexpr int kBatch = 96;
struct ListBatch {
  const void* src[kBatch];
  void* dst[kBatch];
  uint64_t count[kBatch];
  uint32_t first[kBatch + 1];                  // first piece of every tensor, counted from the batch's
  uint32_t bf16[(kBatch + 31) / 32];
  int tensors;
  uint32_t at, total;                          // the batch's first piece, pieces of the whole list
};
static_assert(sizeof(ListBatch) <= 3800, "arguments of a launch");

__global__ __launch_bounds__(THREADS) void tensor_list_kernel(ListBatch b, char* list) {
  ListHeader* h = reinterpret_cast<ListHeader*>(list);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    h->magic = kMagic;
    h->pieces = b.total;
  }
  Piece* out = reinterpret_cast<Piece*>(list + sizeof(ListHeader)) + b.at;
  for (uint32_t i = blockIdx.x * THREADS + threadIdx.x; i < b.first[b.tensors]; i += gridDim.x * THREADS) {
    int lo = 0, hi = b.tensors;                // the last tensor whose first piece is not behind i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (b.first[mid] <= i) lo = mid; else hi = mid;
    }
    const uint64_t from = (uint64_t)(i - b.first[lo]) * kPieceValues, left = b.count[lo] - from;
    const bool half = (b.bf16[lo >> 5] >> (lo & 31)) & 1u;
    const uint64_t es = half ? 2 : 4;
    out[i] = Piece{static_cast<const char*>(b.src[lo]) + from * es, static_cast<char*>(b.dst[lo]) + from * es,
                   (uint32_t)(left < (uint64_t)kPieceValues ? left : (uint64_t)kPieceValues), half ? (uint32_t)DT_BF16 : (uint32_t)DT_F32};
  }
}

// Sixteen bytes at the alignment of one element: tensors of a list may start anywhere.
// NT: stores that leave nothing in the caches (see grad_clip()).
template <class T> struct Wide;
template <> struct Wide<float> {
  static constexpr int V = 4;
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
    const vec q = *reinterpret_cast<const vec*>(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  }
  template <bool NT> static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
    const vec q{v[0], v[1], v[2], v[3]};
    if constexpr (NT) __builtin_nontemporal_store(q, reinterpret_cast<vec*>(p)); else *reinterpret_cast<vec*>(p) = q;
  }
};
template <> struct Wide<bf16_t> {
  static constexpr int V = 8;
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void load(const bf16_t* p, float (&v)[8]) {
    const vec q = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(q[i] << 16);
      v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
    }
  }
  template <bool NT> static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[8]) {
    vec q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    if constexpr (NT) __builtin_nontemporal_store(q, reinterpret_cast<vec*>(p)); else *reinterpret_cast<vec*>(p) = q;
  }
};

constexpr int U = 4;                           // loads of a thread in flight

template <class T>
__device__ __forceinline__ double piece_squares(const Piece& pc) {
  constexpr int V = Wide<T>::V;
  const T* src = static_cast<const T*>(pc.src);
  const uint32_t whole = pc.count / V * V;
  double s = 0.0;
  uint32_t i = threadIdx.x * V;
  for (; i + (U - 1) * THREADS * V < whole; i += U * THREADS * V) {
    float v[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) Wide<T>::load(src + i + u * THREADS * V, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) s += (double)v[u][j] * (double)v[u][j];
  }
  for (; i < whole; i += THREADS * V) {
    float v[V];
    Wide<T>::load(src + i, v);
#pragma unroll
    for (int j = 0; j < V; ++j) s += (double)v[j] * (double)v[j];
  }
  if (whole + threadIdx.x < pc.count) {        // fewer than V values
    const double g = (double)Elem<T>::load(src + whole + threadIdx.x);
    s += g * g;
  }
  return s;
}

// The sum over the workgroup, in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double sh[THREADS / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  double r = sh[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) r += sh[w];
  return r;
}

// Pieces of a list; none (and a sum that is no number) where the memory holds no list.
__device__ __forceinline__ uint32_t list_pieces(const char* list, uint32_t room, bool* valid) {
  const ListHeader* h = reinterpret_cast<const ListHeader*>(list);
  *valid = h->magic == kMagic && h->pieces <= room;
  return *valid ? h->pieces : 0;
}

__global__ __launch_bounds__(THREADS) void square_sums_kernel(const char* __restrict__ list, uint32_t room, double* __restrict__ sums) {
  bool valid;
  const uint32_t pieces = list_pieces(list, room, &valid);
  const Piece* at = reinterpret_cast<const Piece*>(list + sizeof(ListHeader));
  double s = valid ? 0.0 : (double)NAN;
  for (uint32_t p = blockIdx.x; p < pieces; p += gridDim.x) {
    const Piece pc = at[p];
    s += pc.dtype == DT_BF16 ? piece_squares<bf16_t>(pc) : piece_squares<float>(pc);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__device__ __forceinline__ double total_norm(const double* __restrict__ sums, int count) {
  double v[kMaxSums / THREADS];
#pragma unroll
  for (int u = 0; u < kMaxSums / THREADS; ++u) {
    const int i = threadIdx.x + u * THREADS;
    v[u] = sums[i < count ? i : 0];
  }
  double s = 0.0;
#pragma unroll
  for (int u = 0; u < kMaxSums / THREADS; ++u) s += (int)threadIdx.x + u * THREADS < count ? v[u] : 0.0;
  return sqrt(block_sum(s));
}

// a norm that is no number makes the factor none either: it shows in every value
__device__ __forceinline__ float clip_factor(double norm, float bound) { return norm <= (double)bound ? 1.f : (float)((double)bound / norm); }

__global__ __launch_bounds__(THREADS) void norm_kernel(const double* __restrict__ sums, int count, float* __restrict__ norm) {
  const double n = total_norm(sums, count);
  if (threadIdx.x == 0) *norm = (float)n;
}

template <class T, bool NT>
__device__ __forceinline__ void piece_scale(const Piece& pc, float f) {
  constexpr int V = Wide<T>::V;
  const T* src = static_cast<const T*>(pc.src);
  T* dst = static_cast<T*>(pc.dst);
  const uint32_t whole = pc.count / V * V;
  uint32_t i = threadIdx.x * V;
  for (; i + (U - 1) * THREADS * V < whole; i += U * THREADS * V) {
    float v[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) Wide<T>::load(src + i + u * THREADS * V, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int j = 0; j < V; ++j) v[u][j] *= f;
      Wide<T>::template store<NT>(dst + i + u * THREADS * V, v[u]);
    }
  }
  for (; i < whole; i += THREADS * V) {
    float v[V];
    Wide<T>::load(src + i, v);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= f;
    Wide<T>::template store<NT>(dst + i, v);
  }
  if (whole + threadIdx.x < pc.count) Elem<T>::store(dst + whole + threadIdx.x, Elem<T>::load(src + whole + threadIdx.x) * f);
}

template <bool NT>
__global__ __launch_bounds__(THREADS) void clip_kernel(const char* list, uint32_t room, const double* __restrict__ sums, int count,
                                                       float bound, float* __restrict__ norm) {
  const double n = total_norm(sums, count);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const float f = clip_factor(n, bound);
  bool valid;
  const uint32_t pieces = list_pieces(list, room, &valid);
  const Piece* at = reinterpret_cast<const Piece*>(list + sizeof(ListHeader));
  for (uint32_t p = blockIdx.x; p < pieces; p += gridDim.x) {
    const Piece pc = at[p];
    if (f == 1.f && pc.src == pc.dst) continue;          // nothing would change
    if (pc.dtype == DT_BF16) piece_scale<bf16_t, NT>(pc, f); else piece_scale<float, NT>(pc, f);
  }
}

// The same over one contiguous region, and an SGD step with the scaled gradient, which is not stored.  60.2 M parameters: 42 us (5.7 TB/s) more than the plain step of 118, one more
// reading of the gradient.
__global__ __launch_bounds__(THREADS) void region_sums_kernel(const float* __restrict__ g, size_t count, double* __restrict__ sums) {
  double s = 0.0;
  for (size_t at = (size_t)blockIdx.x * kPieceValues; at < count; at += (size_t)gridDim.x * kPieceValues) {
    const Piece pc{g + at, nullptr, (uint32_t)(count - at < (size_t)kPieceValues ? count - at : (size_t)kPieceValues), DT_F32};
    s += piece_squares<float>(pc);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}
__global__ __launch_bounds__(THREADS) void clipped_sgd_kernel(float* __restrict__ w, const float* __restrict__ g, float lr, size_t count, bf16_t* __restrict__ w16,
                                                              const double* __restrict__ sums, int sum_count, float bound, float* __restrict__ norm) {
  const double n = total_norm(sums, sum_count);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const float f = clip_factor(n, bound);
  for (size_t i = (size_t)blockIdx.x * THREADS + threadIdx.x; i < count; i += (size_t)gridDim.x * THREADS) {
    const float v = fmaf(-lr, g[i] * f, w[i]);
    w[i] = v;
    if (w16) w16[i] = float_to_bf16(v);
  }
}

// From 1024 pieces on (64 MB of fp32) the results are written past the caches, which then still hold more of what the norm has read (us, gradients of
// ResNet-152, 241 MB, 145 -> 117; 140 MB of bf16 90 -> 73; 40 MB of fp32 22.1 -> 22.5, and there the update that follows finds the results in the
// caches).  Pieces taken from the last to the first gain nothing more (118), nor do eight loads in flight (117).
constexpr uint32_t kManyPieces = 1024;
inline uint32_t list_room(size_t list_bytes) {
  const size_t pieces = (list_bytes - sizeof(ListHeader)) / sizeof(Piece);
  return pieces < (1u << 30) ? (uint32_t)pieces : (1u << 30);
}
inline int workgroups(uint32_t room) { return room < 1 ? 1 : room < (uint32_t)kMaxSums ? (int)room : kMaxSums; }
}  // namespace

size_t tensor_list_bytes(const size_t* counts, int n) {
  size_t pieces = 0;
  for (int i = 0; i < n; ++i) {
    pieces += counts[i] / kPieceValues + (counts[i] % kPieceValues != 0);
    if (pieces > (1u << 30)) return 0;
  }
  return sizeof(ListHeader) + pieces * sizeof(Piece);
}

hipError_t tensor_list(const void* const* src, void* const* dst, const size_t* counts, const int32_t* dtypes, int n, void* list, hipStream_t st) {
  const size_t bytes = tensor_list_bytes(counts, n);
  if (!bytes) return hipErrorInvalidValue;
  ListBatch b{};
  b.total = (uint32_t)((bytes - sizeof(ListHeader)) / sizeof(Piece));
  for (int i = 0; i < n;) {
    const int from = i;
    uint32_t pieces = 0;
    for (uint32_t& w : b.bf16) w = 0;
    for (; i < n && i - from < kBatch; ++i) {
      const int k = i - from;
      b.src[k] = src[i];
      b.dst[k] = dst ? dst[i] : const_cast<void*>(src[i]);
      b.count[k] = counts[i];
      b.first[k] = pieces;
      if (dtypes[i] == DT_BF16) b.bf16[k >> 5] |= 1u << (k & 31);
      pieces += (uint32_t)(counts[i] / kPieceValues + (counts[i] % kPieceValues != 0));
    }
    b.tensors = i - from;
    b.first[b.tensors] = pieces;
    const unsigned blocks = pieces / THREADS + 1 < 1024 ? pieces / THREADS + 1 : 1024;
    hipLaunchKernelGGL(tensor_list_kernel, dim3(blocks), dim3(THREADS), 0, st, b, static_cast<char*>(list));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    b.at += pieces;
  }
  return hipSuccess;
}

size_t grad_norm_workspace_bytes() { return kMaxSums * sizeof(double); }

hipError_t sgd_update_clipped(float* w, const float* g, float lr, float max_norm, size_t count, void* w_bf16, float* norm, void* scratch,
                              size_t scratch_bytes, hipStream_t st) {
  if (!w || !g || !norm || !scratch || scratch_bytes < 256 || !(max_norm >= 0.f)) return hipErrorInvalidValue;
  const size_t room = scratch_bytes / sizeof(double), pieces = (count + kPieceValues - 1) / kPieceValues;
  size_t sums = room < (size_t)kMaxSums ? room : (size_t)kMaxSums;
  if (sums > pieces) sums = pieces ? pieces : 1;
  hipLaunchKernelGGL(region_sums_kernel, dim3((unsigned)sums), dim3(THREADS), 0, st, g, count, static_cast<double*>(scratch));
  const size_t blocks = (count + THREADS - 1) / THREADS;
  hipLaunchKernelGGL(clipped_sgd_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks < 4096 ? blocks : 4096)), dim3(THREADS), 0, st, w, g, lr, count, (bf16_t*)w_bf16,
                     static_cast<const double*>(scratch), (int)sums, max_norm, norm);
  return hipGetLastError();
}

hipError_t grad_norm(const void* list, size_t list_bytes, float* norm, void* workspace, hipStream_t st) {
  if (!list || !norm || !workspace || list_bytes < sizeof(ListHeader)) return hipErrorInvalidValue;
  const uint32_t room = list_room(list_bytes);
  const int wgs = workgroups(room);
  hipLaunchKernelGGL(square_sums_kernel, dim3(wgs), dim3(THREADS), 0, st, static_cast<const char*>(list), room, static_cast<double*>(workspace));
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(THREADS), 0, st, static_cast<const double*>(workspace), wgs, norm);
  return hipGetLastError();
}

hipError_t grad_clip(const void* list, size_t list_bytes, float bound, float* norm, void* workspace, hipStream_t st) {
  if (!list || !norm || !workspace || list_bytes < sizeof(ListHeader) || !(bound >= 0.f)) return hipErrorInvalidValue;
  const uint32_t room = list_room(list_bytes);
  const int wgs = workgroups(room);
  hipLaunchKernelGGL(square_sums_kernel, dim3(wgs), dim3(THREADS), 0, st, static_cast<const char*>(list), room, static_cast<double*>(workspace));
  if (room >= kManyPieces)
    hipLaunchKernelGGL(clip_kernel<true>, dim3(wgs), dim3(THREADS), 0, st, static_cast<const char*>(list), room, static_cast<const double*>(workspace), wgs,
                       bound, norm);
  else
    hipLaunchKernelGGL(clip_kernel<false>, dim3(wgs), dim3(THREADS), 0, st, static_cast<const char*>(list), room, static_cast<const double*>(workspace), wgs,
                       bound, norm);
  return hipGetLastError();
}

}  // namespace acc
