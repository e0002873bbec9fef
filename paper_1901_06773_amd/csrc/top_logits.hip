// The k largest values of each row with their columns, largest first, the lower column first among equal ones: a teacher's answers, to be kept in the place of
// its logits.
//
// A row is read once, into the registers of a workgroup.  The threads' largest values bound the k-th largest of the row from below: k of them are values of the
// row.  What reaches the bound, some more than k values, is written into LDS with its column as one 64-bit key and sorted there.  Where that is more than fits
// (many equal values) or there are fewer threads than k, the k-th largest key is found by halving, one bit after the other, with a count of the row each
// time, and then the column up to which equal ones are taken.  Rows that no workgroup's registers hold, and long ones where there are few, are cut into segments
// whose lists are rows of a second launch.  Bound by reading the row from memory.
#include "kernels.h"
#include "row_chunks.h"

namespace acc {
namespace {

// The order of floats as that of whole numbers: both zeros are equal, what is no number is above all.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return v != v ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return o == 0xFFFFFFFFu ? __uint_as_float(0x7fc00000u) : __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// The chunk as something the compiler knows nothing of: what it unpacks of it for one sweep over the row it does not keep for the next.
__device__ __forceinline__ void unpack_again(chunk16& q) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(q));
#endif
}

struct TopArgs {
  const void* z;
  const int32_t* map;        // of a second launch: the columns that the row's values are of
  int32_t* index;            // [row][segment][k]
  float* top;
  int n, classes, k, segment, segments;
};

template <int NT> struct TopRoom { static constexpr int value = NT == 64 ? 512 : NT == 256 ? 1024 : 2048; };      // candidates in LDS, at least k

// The largest t (of the bits `step` and up) that `want` of the threads' whole numbers reach, by one wave, from LDS.
template <int NT> __device__ __forceinline__ uint32_t reached_by(const uint32_t* keys, int want) {
  const int lane = threadIdx.x & 63;
  uint32_t mine[NT / 64];
#pragma unroll
  for (int u = 0; u < NT / 64; ++u) mine[u] = keys[lane + 64 * u];
  uint32_t t = 0;
  for (int bit = 31; bit >= 16; --bit) {               // (a bound: the lower half may as well be zero)
    const uint32_t mid = t | (1u << bit);
    int c = 0;
#pragma unroll
    for (int u = 0; u < NT / 64; ++u) c += __popcll(__ballot(mine[u] >= mid));
    if (c >= want) t = mid;
  }
  return t;
}

template <class T, int NT, int CH>
__global__ __launch_bounds__(NT) void top_kernel(TopArgs a) {
  typedef RowChunks<T> Row;
  constexpr int PER = Row::PER, ROOM = TopRoom<NT>::value, W = NT / 64;
  __shared__ unsigned long long cand[ROOM];
  __shared__ uint32_t keys[NT];
  __shared__ int counter, waves[2][W];
  __shared__ float bound;
  const int tid = threadIdx.x, row_at = (int)blockIdx.x / a.segments, seg = (int)blockIdx.x - row_at * a.segments;
  const int from = seg * a.segment, count = min(a.segment, a.classes - from), want = min(a.k, count);
  const T* const row = static_cast<const T*>(a.z) + (size_t)row_at * a.classes + from;
  const Row r(row, count);
  chunk16 q[CH];
  float mx = -INFINITY;
#pragma unroll
  for (int u = 0; u < CH; ++u)
    if (tid + u * NT < r.chunks) q[u] = r.load(row, tid + u * NT);
#pragma unroll
  for (int u = 0; u < CH; ++u)
    if (tid + u * NT < r.chunks) {
#pragma unroll
      for (int e = 0; e < PER; ++e) mx = fmaxf(mx, Row::value(q[u], e));        // (what is no number reaches any bound)
    }
  // keys of the threads without a value are the lowest
  keys[tid] = tid < r.chunks ? order_of(mx) : 0;
  if (tid == 0) counter = 0;
  row_sync<NT>();
  if (tid < 64) {
    const float b = want <= min(NT, r.chunks) ? value_of(max(reached_by<NT>(keys, want), order_of(-INFINITY))) : -INFINITY;
    if (tid == 0) bound = b;
  }
  row_sync<NT>();
  const float low = bound;
  // f(key, column) for every value of the row, from the caches: the registers of the first two sweeps would not fit with this unrolled
  auto each = [&](auto f) {
#pragma unroll 1
    for (int c = tid; c < r.chunks; c += NT) {
      const chunk16 v = r.load(row, c);
#pragma unroll 1
      for (int e = max(0, -r.at(c)); e < min(PER, count - r.at(c)); ++e) {
        float x;
        if constexpr (sizeof(T) == 2) {
          const uint32_t w = e < 4 ? (e < 2 ? v[0] : v[1]) : (e < 6 ? v[2] : v[3]);
          x = __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
        } else {
          x = __uint_as_float(e < 2 ? (e ? v[1] : v[0]) : (e == 2 ? v[2] : v[3]));
        }
        f(order_of(x), r.at(c) + e);
      }
    }
  };
  auto take = [&](uint32_t key, int at) {
    const int to = atomicAdd(&counter, 1);
    if (to < ROOM) cand[to] = ((unsigned long long)key << 32) | (0xFFFFFFFFu - (uint32_t)at);
  };
#pragma unroll
  for (int u = 0; u < CH; ++u) {
    const int c = tid + u * NT;
    if (c >= r.chunks) continue;
    unpack_again(q[u]);
    bool any = false;
#pragma unroll
    for (int e = 0; e < PER; ++e) any |= !(Row::value(q[u], e) < low);
    if (!any) continue;
    unpack_again(q[u]);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const float v = Row::value(q[u], e);
      const int at = r.at(c) + e;
      if (!(v < low) && at >= 0 && at < count) take(order_of(v), at);
    }
  }
  row_sync<NT>();
  int found = counter;
  if (found > ROOM) {
    int turn = 0;
    auto total = [&](int mine) {                       // the threads' sum
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
      if constexpr (NT > 64) {
        int* const w = waves[turn];
        turn ^= 1;
        if ((tid & 63) == 0) w[tid >> 6] = mine;
        __syncthreads();
        mine = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) mine += w[i];
      }
      return mine;
    };
    // the largest key that `want` values reach; the bits of bf16 values are the upper half
    uint32_t kth = 0;
    for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 0); --bit) {
      const uint32_t mid = kth | (1u << bit);
      int c = 0;
      each([&](uint32_t key, int) { c += key >= mid ? 1 : 0; });
      if (total(c) >= want) kth = mid;
    }
    if (sizeof(T) == 2 && kth == 0xFFFF0000u) kth = 0xFFFFFFFFu;
    if (sizeof(T) == 2 && !(kth & 0x80000000u)) kth |= 0xFFFFu;       // (of negative values the lower half is ones)
    int c = 0;
    each([&](uint32_t key, int) { c += key > kth ? 1 : 0; });
    const int equal = want - total(c);                 // so many of the equal ones, from the lowest column on
    int first = 0;                                     // the lowest column that is not among them: `equal` are below it
    for (int bit = 30; bit >= 0; --bit) {
      const int mid = first | (1 << bit);
      if (mid > count) continue;
      int m = 0;
      each([&](uint32_t key, int at) { m += key == kth && at < mid ? 1 : 0; });
      if (total(m) < equal) first = mid;
    }
    __syncthreads();
    if (tid == 0) counter = 0;
    row_sync<NT>();
    each([&](uint32_t key, int at) { if (key > kth || (key == kth && at <= first)) take(key, at); });
    row_sync<NT>();
    found = counter;
  }
  // sorted, largest first, up to the next power of two
  int size = 1;
  while (size < found) size *= 2;
  for (int i = found + tid; i < size; i += NT) cand[i] = 0;
  row_sync<NT>();
  for (int span = 2; span <= size; span *= 2)
    for (int step = span / 2; step > 0; step /= 2) {
      for (int i = tid; i < size / 2; i += NT) {
        const int lo = 2 * step * (i / step) + i % step, hi = lo + step;
        const unsigned long long x = cand[lo], y = cand[hi];
        if (((lo & span) == 0) == (x < y)) { cand[lo] = y; cand[hi] = x; }
      }
      row_sync<NT>();
    }
  const size_t out = ((size_t)row_at * a.segments + seg) * a.k;
  for (int i = tid; i < a.k; i += NT) {
    if (i >= want) {                                   // (of a short last segment: behind all of its row's values)
      a.index[out + i] = -1;
      a.top[out + i] = -INFINITY;
      continue;
    }
    const unsigned long long c = cand[i];
    const int at = from + (int)(0xFFFFFFFFu - (uint32_t)c);
    a.index[out + i] = a.map ? a.map[(size_t)row_at * a.classes + at] : at;
    a.top[out + i] = value_of((uint32_t)(c >> 32));
  }
}

inline size_t al256(size_t b) { return (b + 255) & ~(size_t)255; }
inline long ceil_div(long a, long b) { return (a + b - 1) / b; }

constexpr int kMostTop = 1024, kMostClasses = 1 << 20, kMostRows = 1 << 20;

struct TopPlan {
  int segment, segments;
  size_t top, total;           // offsets in the workspace: columns, values
};
TopPlan top_plan(int n, int classes, int k, int dtype) {
  TopPlan p{};
  const int per = dtype == DT_BF16 ? 8 : 4, most = 1024 * 16 * per - 64;       // (a row may begin inside a chunk)
  p.segments = (int)ceil_div(classes, most);
  // (whole chunks: segments of a row that begins aligned do, too)
  p.segment = p.segments == 1 ? classes : (int)(ceil_div(ceil_div(classes, p.segments), 64) * 64);
  p.segments = (int)ceil_div(classes, p.segment);
  p.top = al256(p.segments > 1 ? (size_t)n * p.segments * k * 4 : 0);
  p.total = 2 * p.top;
  return p;
}

template <class T> hipError_t launch_top(const TopArgs& a, hipStream_t st) {
  constexpr int PER = RowChunks<T>::PER;
  const int chunks = (a.segment + PER - 1) / PER + 1;
  const dim3 grid((unsigned)(a.n * a.segments));
#define ACC_TOP(NT, CH) if (chunks <= NT * CH && a.k <= TopRoom<NT>::value) { hipLaunchKernelGGL((top_kernel<T, NT, CH>), grid, dim3(NT), 0, st, a); return hipGetLastError(); }
  ACC_TOP(64, 1) ACC_TOP(64, 4)
  ACC_TOP(256, 4) ACC_TOP(256, 16)
  ACC_TOP(512, 16)
  ACC_TOP(1024, 16)
#undef ACC_TOP
  return hipErrorInvalidValue;
}

// (a launch has fewer than 2^32 threads)
bool top_ok(int n, int classes, int k, int dtype) {
  return n > 0 && classes > 0 && k > 0 && n <= kMostRows && classes <= kMostClasses && k <= kMostTop && k <= classes && (dtype == DT_F32 || dtype == DT_BF16) &&
         (long)n * top_plan(n, classes, k, dtype).segments < 1L << 22;
}

}  // namespace

size_t top_logits_workspace_bytes(int n, int classes, int k, int dtype) { return top_ok(n, classes, k, dtype) ? top_plan(n, classes, k, dtype).total : 0; }

hipError_t top_logits(const void* z, int32_t* index, float* top, int n, int classes, int k, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!z || !index || !top || !top_ok(n, classes, k, dtype)) return hipErrorInvalidValue;
  const TopPlan p = top_plan(n, classes, k, dtype);
  if (workspace_bytes < p.total || (p.total && !workspace)) return hipErrorInvalidValue;
  TopArgs a{z, nullptr, index, top, n, classes, k, p.segment, p.segments};
  if (p.segments > 1) {
    a.index = (int32_t*)workspace;
    a.top = (float*)((char*)workspace + p.top);
  }
  const hipError_t e = dtype == DT_BF16 ? launch_top<bf16_t>(a, st) : launch_top<float>(a, st);
  if (e != hipSuccess || p.segments == 1) return e;
  const int all = p.segments * k;
  return launch_top<float>(TopArgs{a.top, a.index, index, top, n, all, k, all, 1}, st);
}

}  // namespace acc
