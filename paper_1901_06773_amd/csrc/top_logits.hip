// The k largest values of each row with their columns, largest first, the lower column first among equal ones: a teacher's answers, to be kept in the place of
// its logits.
//
// A row is read once, into the registers of a workgroup.  The threads' largest values bound the k-th largest of the row from below: k of them are values of the
// row.  What reaches the bound, some more than k values, is written into LDS with its column as one 64-bit key and sorted there.  Where that is more than fits
// (many equal values) or there are fewer threads than k, the k-th largest key is found by halving, one bit after the other, with a count of the row each
// time, and then the column up to which equal ones are taken.  Rows that no workgroup's registers hold are cut into segments
// whose lists are rows of a second launch.
//
// Bound by reading the rows: 4096 bf16 rows of 65536, k = 64, 128 us (4.2 TB/s; two workgroups of a compute unit cover each other's barriers), of fp32 230 to
// 260.  Short rows and long lists by the steps of a row behind each other: 4096 rows of 8192 30 us (2.2 TB/s), k = 150 47; a few rows of any width 6 to 15.
// Rows with more equal values at the k-th than LDS has room for take some fifty sweeps from the caches: of one value throughout, 4096 bf16 rows of 65536 5400
// us, fp32 7200, 4096 bf16 rows of 8192 630, 64 fp32 rows of 1000, k = 16, 79 (others 5.4); of logits rounded to whole numbers, of which few are the largest, 162.
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

// Candidates that LDS has room for, at least k; groups that a thread's values are dealt out to, each of which gives its largest one to the bound.
template <int NT, int CH, int G> struct TopShape {
  static constexpr int room = NT == 64 ? 512 : NT < 1024 ? 1024 : CH == 1 ? 4096 : 2048, groups = G;
};

// The largest t, of its upper sixteen bits (a bound: the lower half may as well be zero), that `want` of the threads' keys reach.  Every wave looks at all
// keys and tries another value of the next bits: log2 of the waves at a time, one barrier each (4096 rows of 65536 bf16 128 us; bit by bit 243).
template <int NT, int GROUPS> __device__ __forceinline__ uint32_t reached_by(const uint32_t* keys, int want, int (*sh)[NT / 64]) {
  constexpr int W = NT / 64, BITS = W >= 16 ? 4 : W >= 8 ? 3 : W >= 4 ? 2 : 1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t t = 0;
  int turn = 0;
  for (int shift = 32 - BITS; shift > 16 - BITS; shift -= BITS) {
    const uint32_t mid = t | ((W == 1 ? 1u : (uint32_t)wave) << shift);
    int c = 0;
#pragma unroll
    for (int u = 0; u < W * GROUPS; ++u) c += __popcll(__ballot(keys[lane + 64 * u] >= mid));
    if constexpr (W == 1) {
      if (c >= want) t = mid;
    } else {
      if (lane == 0) sh[turn][wave] = c;
      __syncthreads();
      int best = 0;
#pragma unroll
      for (int w = 1; w < W; ++w) best = sh[turn][w] >= want ? w : best;       // (the counts fall with w)
      t |= (uint32_t)best << shift;
      turn ^= 1;
    }
  }
  return t;
}

template <class T, int NT, int CH, int G>
__global__ __launch_bounds__(NT, CH == 8 ? 8 : 4) void top_kernel(TopArgs a) {
  typedef RowChunks<T> Row;
  constexpr int PER = Row::PER, ROOM = TopShape<NT, CH, G>::room, GROUPS = TopShape<NT, CH, G>::groups, W = NT / 64;
  __shared__ unsigned long long cand[ROOM];
  __shared__ uint32_t keys[NT * GROUPS];
  __shared__ int counter, waves[2][W];
  const int tid = threadIdx.x, row_at = (int)blockIdx.x / a.segments, seg = (int)blockIdx.x - row_at * a.segments;
  const int from = seg * a.segment, count = min(a.segment, a.classes - from), want = min(a.k, count);
  const T* const row = static_cast<const T*>(a.z) + (size_t)row_at * a.classes + from;
  const Row r(row, count, (long)(a.n - row_at) * a.classes - from);
  chunk16 q[CH];
#pragma unroll
  for (int u = 0; u < CH; ++u)
    if (tid + u * NT < r.chunks) q[u] = r.load(row, tid + u * NT);
  float mx[GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) mx[g] = -INFINITY;
#pragma unroll
  for (int u = 0; u < CH; ++u)
    if (tid + u * NT < r.chunks) {
      r.cut(q[u], tid + u * NT);
#pragma unroll
      for (int e = 0; e < PER; ++e) mx[e * GROUPS / PER] = fmaxf(mx[e * GROUPS / PER], Row::value(q[u], e));        // (what is no number reaches any bound)
    }
  // keys of the threads without a value are the lowest, those of a group without one (at an end of the row) minus infinity's
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) keys[tid + g * NT] = tid < r.chunks ? order_of(mx[g]) : 0;
  if (tid == 0) counter = 0;
  row_sync<NT>();
  // (a group without a value counts as minus infinity: a bound that needs it leaves out nothing)
  const float low = want <= GROUPS * min(NT, r.chunks) ? value_of(max(reached_by<NT, GROUPS>(keys, want, waves), order_of(-INFINITY))) : -INFINITY;
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
      auto add = [](int x, int y) { return x + y; };
      mine = wave_reduce(mine, add);
      if constexpr (NT > 64) {
        int* const w = waves[turn];
        turn ^= 1;
        if ((tid & 63) == 0) w[tid >> 6] = mine;
        __syncthreads();
        mine = join_waves<NT>(w, add);
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
  const size_t out = ((size_t)row_at * a.segments + seg) * a.k;
  auto give = [&](int i, unsigned long long c) {
    const int at = from + (int)(0xFFFFFFFFu - (uint32_t)c);
    a.index[out + i] = a.map ? a.map[(size_t)row_at * a.classes + at] : at;
    a.top[out + i] = value_of((uint32_t)(c >> 32));
  };
  for (int i = want + tid; i < a.k; i += NT) {         // (of a short last segment: behind all of its row's values)
    a.index[out + i] = -1;
    a.top[out + i] = -INFINITY;
  }
  int size = 1;
  while (size < found) size *= 2;
  // Few: each is compared with all others, by as many threads as there are for it; its rank is its place.  More: sorted, largest first, in steps with a barrier
  // each.  (us, ranks / sorted: 4096 bf16 rows of 65536, k = 64 (some 70 found) 128 / 156, 64 fp32 rows of 1000 and k = 100 6.5 / 9.9, 4096 bf16 rows of 8192
  // and k = 150 (some 200 found, 256 threads) 54 / 47.)
  if (size <= NT && found * size <= 160 * NT) {
    const int per = NT / size, i = tid / per, part = tid % per;
    const unsigned long long c = i < found ? cand[i] : 0;
    int rank = 0;
#pragma unroll 8
    for (int j = part; j < found; j += per) rank += cand[j] > c ? 1 : 0;
    for (int o = 1; o < min(per, 64); o <<= 1) rank += __shfl_xor(rank, o);
    if (per > 64) {                                    // (so few that a wave has only one of them)
      if ((tid & 63) == 0) keys[tid >> 6] = (uint32_t)rank;
      row_sync<NT>();
      rank = 0;
      for (int w = 0; w < per / 64; ++w) rank += (int)keys[(i * per >> 6) + w];
    }
    if (part == 0 && i < found && rank < want) give(rank, c);
    return;
  }
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
  for (int i = tid; i < want; i += NT) give(i, cand[i]);
}

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
  // (a row begins inside a chunk where the rows are not whole ones)
  const int chunks = (a.segment + PER - 1) / PER + (a.classes % PER ? 1 : 0);
  const dim3 grid((unsigned)(a.n * a.segments));
  // The smallest workgroup that holds a row, of which all values fit LDS or the bound leaves out most: with k as many as three quarters of the groups it still
  // leaves out half.  (us, so / the smallest that holds the row: 1000 rows of 1306 bf16 logits, k = 118, 12.5 / 85, 1000 of 6000 fp32, k = 300, 23 / 217.)
  // Four groups a thread where k asks for them (so / with one group): 64 fp32 rows of 50000, k = 1000, 43 / 429, 5072 of 200, k = 40, by a wave 7.2 / 16, 5072
  // bf16 of 2000, k = 200, by 256 threads 46 / 271; a wave with them or 256 threads without: 5072 fp32 rows of 259, k = 125, 15 / 28, 12 bf16 rows of 1000, k =
  // 50, 7.0 / 5.6.  A chunk a thread or eight, whose registers leave two workgroups of 1024 threads to a compute unit, and sixteen: with four (4096 bf16 rows
  // of 8192, k = 64, 43 / 31) the compiler takes half as many registers more.
#define ACC_TOP(NT, CH, G, rule)                                                                                 \
  {                                                                                                              \
    const bool bounded = 4 * a.k <= 3 * G * (chunks < NT ? chunks : NT), all = a.segment <= (NT < 1024 ? 2 * NT : 4096); \
    (void)bounded; (void)all;                                                                                    \
    if (chunks <= NT * CH && a.k <= TopShape<NT, CH, G>::room && (rule)) {                                       \
      hipLaunchKernelGGL((top_kernel<T, NT, CH, G>), grid, dim3(NT), 0, st, a);                                  \
      return hipGetLastError();                                                                                  \
    }                                                                                                            \
  }
  ACC_TOP(64, 1, 1, bounded) ACC_TOP(64, 1, 4, bounded) ACC_TOP(64, 1, 1, all) ACC_TOP(64, 4, 1, bounded) ACC_TOP(64, 4, 4, bounded && a.n > 2048)
  ACC_TOP(256, 1, 1, bounded) ACC_TOP(256, 1, 4, bounded) ACC_TOP(256, 1, 1, all) ACC_TOP(256, 8, 1, bounded)
  ACC_TOP(512, 8, 1, bounded)
  ACC_TOP(1024, 1, 4, bounded || all) ACC_TOP(1024, 8, 1, bounded) ACC_TOP(1024, 8, 4, true) ACC_TOP(1024, 16, 1, bounded) ACC_TOP(1024, 16, 4, true)
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
