// Distillation: the loss of a student's logits against a list of a teacher's largest ones, and its gradient.  Of row i, with the teacher's logits t_j of the
// classes c_j of its list, temperature T and, where there are labels, their share:
//
//   p = softmax(t / T) over the list,  q = softmax(z / T) over all classes,  s = softmax(z)
//   loss_i = alpha T^2 sum_j p_j (log p_j - log q_cj) + (1 - alpha) (lse(z) - z_label),   loss = mean over the rows that count
//   dz = (alpha T (q - p) + (1 - alpha) (s - onehot)) / rows that count
//
// A row is read once, into the registers of a wave or a workgroup, and its gradient written from there: memory bounds it.  Rows that no registers hold, and few
// long ones, are cut: a launch leaves the sums of each part, the next joins them and writes the gradient.  The list's probabilities are worked out by the same
// threads, an entry each, while the row is on its way; the few classes of the list (and the label) are written again, behind a barrier, with their own terms.
//
// Sums of exponentials go without the largest one, which is 1: with R the sum of the others', log(1 + R) and, of a class that both give more than a half,
// q - p = (1 - p) - (1 - q) keep R where a class is all but certain.
//
// At high temperatures, where the list holds nearly all that the row has, T^2 sum p (log p - log q) and T (q - p) are what T^2 and T make of the roundings of
// numbers near one.  They are worked out by differences there (Warm).
//
// us: 4096 bf16 rows of 65536, lists of 64, 223 (4.8 TB/s read and written, as a copy; with labels 254: a second exponential for each logit; the loss alone
// 106), of fp32 455; 777 of 50001 59 (512 workgroups run at a time, so two rounds); 4096 of 8192 40 (3.4 TB/s); 64 rows of 10^6, cut, 92.
#include "kernels.h"
#include "row_chunks.h"

#include <climits>

namespace acc {
namespace {

constexpr float LOG2E = 1.44269504088896341f;
__device__ __forceinline__ float exp2_fast(float t) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_exp2f(t);
#else
  return t;
#endif
}

struct DistillArgs {
  const void* z;
  const int32_t* index;
  const float* top;
  const int32_t* labels;       // null: the teacher alone
  int ignore;
  float inv_t, soft, hard, soft_slope, alpha, t2;      // 1 / T, alpha T^2, 1 - alpha, alpha T, alpha, T^2
  float *loss_rows, *loss;
  void* dz;                    // null: the loss alone
  int n, classes, k;
  const int* counts;           // rows that count, in parts; null: counted here
  int count_parts;
  // cut rows
  float *part, *at_list;       // part[row][3][splits]: the largest logit and R at both temperatures; at_list[row][k + 1]: logits of the list and of the label
  unsigned long long* shares;  // shares[row][splits]: sums of shares()
  int splits, chunks_per_split;
};

__device__ __forceinline__ bool row_counts(const DistillArgs& a, int row) {
  return a.labels ? a.ignore == INT_MIN || a.labels[row] != a.ignore : a.index[(size_t)row * a.k] >= 0;
}
// Rows that count among all: a thread's part of NT threads'
template <int NT> __device__ __forceinline__ int count_part(const DistillArgs& a) {
  int c = 0;
  if (a.counts) {
    for (int i = threadIdx.x % NT; i < a.count_parts; i += NT) c += a.counts[i];
  } else {
#pragma unroll 4
    for (int i = threadIdx.x % NT; i < a.n; i += NT) c += row_counts(a, i) ? 1 : 0;
  }
  return c;
}
struct Add {
  template <class V> __device__ __forceinline__ V operator()(V x, V y) const { return x + y; }
};
struct Larger {
  __device__ __forceinline__ float operator()(float x, float y) const { return fmaxf(x, y); }
};
struct Lower {
  __device__ __forceinline__ int operator()(int x, int y) const { return min(x, y); }
};
template <int NT> struct RowShared {
  float v[8][NT / 64];
  int n[2][NT / 64];
};

// The list of a row in LDS, four arrays of list_pitch(k) words; entry j is its thread's, j modulo NT.
struct List {
  int32_t* cls;                // -1 from `length` on
  float *t, *p, *z;            // the teacher's logits, probabilities; the student's logits of these classes
  int length;                  // entries before the first negative class
  float max, rest, inv, log_sum;
};
__host__ __device__ __forceinline__ int list_pitch(int k) { return (k + 3) & ~3; }
__device__ __forceinline__ List list_in(float* lds, int k) {
  const int pitch = list_pitch(k);
  return List{reinterpret_cast<int32_t*>(lds), lds + pitch, lds + 2 * pitch, lds + 3 * pitch, 0, 0.f, 0.f, 0.f, 0.f};
}
// entries, and the student's logits by z_at(entry, class); returns the thread's idea of the length
template <int NT, class F> __device__ __forceinline__ int list_read(const DistillArgs& a, int row, const List& l, F z_at) {
  const int32_t* const index = a.index + (size_t)row * a.k;
  const float* const top = a.top + (size_t)row * a.k;
  int length = a.k;
  for (int j = threadIdx.x % NT; j < list_pitch(a.k); j += NT) {
    const int c = j < a.k ? index[j] : -1;
    const float t = j < a.k ? top[j] : 0.f;
    const float z = (unsigned)c < (unsigned)a.classes ? z_at(j, c) : NAN;
    if (c < 0) length = min(length, j);
    l.cls[j] = c;
    l.t[j] = t;
    l.z[j] = z;
  }
  return length;
}
// behind its end, and the largest logit before it
template <int NT> __device__ __forceinline__ float list_end(const DistillArgs& a, const List& l) {
  float mx = -INFINITY;
  for (int j = threadIdx.x % NT; j < list_pitch(a.k); j += NT) {
    if (j >= l.length) l.cls[j] = -1;
    else mx = fmaxf(mx, l.t[j]);
  }
  return mx;
}
template <int NT> __device__ __forceinline__ void list_sum(const DistillArgs& a, const List& l, float& s, float& equal) {
  s = equal = 0.f;
  for (int j = threadIdx.x % NT; j < l.length; j += NT) {
    const bool top = l.t[j] == l.max;
    equal += top ? 1.f : 0.f;
    s += top ? 0.f : exp2_fast((l.t[j] - l.max) * (a.inv_t * LOG2E));
  }
}
__device__ __forceinline__ void list_known(List& l, float s, float equal) {
  l.rest = fabsf(l.max) == INFINITY ? NAN : s + (equal - 1.f);
  l.inv = 1.f / (1.f + l.rest);
  l.log_sum = log1pf(l.rest);
}
// probabilities; the thread's part of sum p (log p - z / T)
template <int NT> __device__ __forceinline__ float list_loss(const DistillArgs& a, const List& l, float max) {
  float d = 0.f;
  for (int j = threadIdx.x % NT; j < l.length; j += NT) {
    const float v = (l.t[j] - l.max) * a.inv_t, p = exp2_fast(v * LOG2E) * l.inv;
    l.p[j] = p;
    if (l.cls[j] >= a.classes) d = NAN;
    else if (p != 0.f) d += p * (v - l.log_sum) - p * ((l.z[j] - max) * a.inv_t);
  }
  return d;
}

// What a row's sums come to
struct RowSums {
  float max, rest, rest1;      // the largest logit; R at the temperature and at 1
};

// High temperatures.  With x_j = (t_j - t_max) - (z_j - z_max), m = sum p x, y = (x - m) / T, E and P the sums of the row's and the list's exponentials
//
//   sum p (log p - log q) = sum p x / T + log(E / P) = log(1 + sum p (e^-y - 1 + y) + U e^(m / T) / P),   q_j / p_j = e^(-y_j - that)
//
// (sum p y = 0), U the exponentials of the classes that are not listed.  Nothing in it cancels but U, the difference of E and of the listed ones' sum: both are
// added up in whole numbers, of the same roundings of the same exponentials, so that a list of all classes leaves exactly 0.  Relative error of the loss of 512
// fp32 rows of 100 classes, all listed, so / by the plain formula: T = 4 - / 7e-6, 20 1e-7 / 2e-4, 100 8e-8 / 6e-3, 1000 and more 7e-8 / nothing right.  Up to
// 4 the plain formula loses less than T^2 2^-24 log 2^20 = 2e-5, and where the two are half a nat apart or more its roundings are little beside the result.
constexpr float kWarm = 4.f;
struct Warm {
  bool near;                   // less than half a nat apart
  float mean, kl, loss;        // m; the sum above; alpha T^2 times it
};
// The exponential of a logit, and in units of 2^-47.  (A row's sum may pass 2^64; the difference of two that is looked at does not.)
__device__ __forceinline__ float share(float z, float max, float inv_t2) { return exp2_fast((z - max) * inv_t2); }
__device__ __forceinline__ unsigned long long whole(float share) {
  const float v = fmaxf(share, 0.f) * 2147483648.f;    // (no number counts as 0)
  const uint32_t hi = (uint32_t)v, lo = (uint32_t)((v - (float)hi) * 65536.f);
  return ((unsigned long long)hi << 16) + lo;
}
// KL >= log E - (the entropy of p) >= log E - log(entries): less than half a nat asks for as much
__device__ __forceinline__ bool may_be_near(const RowSums& r, int length) { return 1.f + r.rest < 1.7f * (float)length; }
// A thread's part of the whole() of chunks [c0, c1), from memory
template <int NT, class Row, class T> __device__ __forceinline__ unsigned long long wholes(const Row& r, const T* z, int c0, int c1, float max, float inv_t2) {
  unsigned long long all = 0;
#pragma unroll 1
  for (int c = c0 + (int)threadIdx.x % NT; c < c1; c += NT) {
    chunk16 q = r.load(z, c);
    r.cut(q, c);
#pragma unroll
    for (int e = 0; e < Row::PER; ++e) all += whole(share(Row::value(q, e), max, inv_t2));
  }
  return all;
}
template <int NT> struct WarmShared {
  float v[3][NT / 64];
  unsigned long long n[2][NT / 64];
};
// d: the plain formula's sum of the list's parts; all: of the row's whole(); both known to everybody, as the result
template <int NT> __device__ __forceinline__ Warm warm_of(const DistillArgs& a, const List& l, float d, const RowSums& r, unsigned long long all, WarmShared<NT>& sh) {
  const float inv_t2 = a.inv_t * LOG2E;
  float mean = 0.f;
  unsigned long long listed = 0;
  for (int j = threadIdx.x % NT; j < l.length; j += NT)
    if (l.p[j] != 0.f && l.cls[j] < a.classes) {
      mean += l.p[j] * ((l.t[j] - l.max) - (l.z[j] - r.max));
      listed += whole(share(l.z[j], r.max, inv_t2));
    }
  mean = row_reduce<NT>(mean, sh.v[0], Add());
  listed = row_reduce<NT>(listed, sh.n[1], Add());
  const float scale = exp2_fast(mean * inv_t2) * l.inv;
  float bent = 0.f;            // T^2 sum p (e^-y - 1 + y)
  for (int j = threadIdx.x % NT; j < l.length; j += NT)
    if (l.p[j] != 0.f && l.cls[j] < a.classes) {
      const float x = (l.t[j] - l.max) - (l.z[j] - r.max) - mean, y = x * a.inv_t, p = l.p[j];
      if (fabsf(y) < 0.5f) {
        const float series = 0.5f - y * (1.f / 6 - y * (1.f / 24 - y * (1.f / 120 - y * (1.f / 720 - y * (1.f / 5040 - y * (1.f / 40320 - y * (1.f / 362880)))))));
        bent += p * (x * x) * series;
      } else if (y > 0.f) {
        bent += p * a.t2 * (expm1f(-y) + y);
      } else {                 // (p e^-y is q times e^KL: no overflow)
        bent += a.t2 * (share(l.z[j], r.max, inv_t2) * scale + p * (y - 1.f));
      }
    }
  bent = row_reduce<NT>(bent, sh.v[1], Add());
  Warm w;
  const float rest = (float)(long long)(all - listed) * 0x1p-47f * scale, v = bent * a.inv_t * a.inv_t + rest;
  w.near = fabsf(d + log1pf(r.rest)) < 0.5f;           // (false for what is no number)
  w.mean = mean;
  w.kl = log1pf(v);
  // (T^2 v, where v itself may be below fp32's smallest value)
  w.loss = fabsf(v) > 0x1p-12f ? a.soft * w.kl : (a.alpha * bent + a.soft * rest) * (1.f - v * (0.5f - v * (1.f / 3)));
  return w;
}
// d: the list's parts together
__device__ __forceinline__ float loss_of(const DistillArgs& a, int length, float d, const RowSums& r, const Warm& w, int label, float z_label) {
  float loss = length ? (w.near ? w.loss : a.soft * (d + log1pf(r.rest))) : 0.f * r.rest;      // (no list, and no distribution of z: none of the loss either)
  if (a.hard > 0.f) loss += (unsigned)label < (unsigned)a.classes ? a.hard * (log1pf(r.rest1) - (z_label - r.max)) : NAN;
  return loss;
}

// What the gradient of any class is made of
struct Slope {
  float inv_t2, soft, hard, max;      // log2 e / T; alpha T / rows / (1 + R), 0 without a list; (1 - alpha) / rows / (1 + R1)
  template <bool HARD> __device__ __forceinline__ float of(float z) const {
    const float d = z - max;
    float v = exp2_fast(d * inv_t2) * soft;
    if (HARD) v += exp2_fast(d * LOG2E) * hard;
    return v;
  }
};
__device__ __forceinline__ Slope slope_of(const DistillArgs& a, const RowSums& r, int length, float inv_rows) {
  return Slope{a.inv_t * LOG2E, length ? a.soft_slope * inv_rows / (1.f + r.rest) : 0.f, a.hard * inv_rows / (1.f + r.rest1), r.max};
}

// The gradient of the classes [lo, hi) that are in the list, and of the label, by NT threads: their own terms.
template <class T, int NT, bool HARD, bool WARM>
__device__ __forceinline__ void write_listed(const DistillArgs& a, T* dz, int lo, int hi, const List& l, const RowSums& r, const Warm& w, int label, float z_label,
                                             float inv_rows) {
  const float inv = 1.f / (1.f + r.rest), inv1 = 1.f / (1.f + r.rest1);
  for (int j = threadIdx.x % NT; j <= l.length; j += NT) {
    const bool entry = j < l.length;
    const int c = entry ? l.cls[j] : label;
    if (!entry && (!HARD || (unsigned)label >= (unsigned)a.classes)) continue;
    if (c < lo || c >= hi) continue;
    // a class that is listed more than once has all of its entries' probabilities, by the first one
    float sum = entry ? l.p[j] : 0.f;
    int times = 0;
#pragma unroll 4
    for (int i = 0; i < l.length; i += 4) {
      const int4 q = *reinterpret_cast<const int4*>(l.cls + i);
      times += (q.x == c ? 1 : 0) + (q.y == c ? 1 : 0) + (q.z == c ? 1 : 0) + (q.w == c ? 1 : 0);
    }
    if (!entry && times) continue;                     // (a listed label is its entry's)
    if (times > 1) {
      bool first = true;
      for (int i = 0; i < l.length; ++i) {
        const bool same = l.cls[i] == c;
        first = first && !(same && i < j);
        if (same && i > j) sum += l.p[i];
      }
      if (!first) continue;
    }
    const float d = (entry ? l.z[j] : z_label) - r.max;
    float v = 0.f;
    if (l.length) {
      const float u = d * a.inv_t, q = exp2_fast(u * LOG2E) * inv;
      float diff = q - sum;
      const float apart = WARM && entry ? ((l.t[j] - l.max) - d - w.mean) * a.inv_t + w.kl : 0.f;      // log(p / q)
      if (WARM && w.near && entry && times == 1 && sum != 0.f && fabsf(apart) < 0.5f)
        diff = sum * expm1f(-apart);
      else if (entry && times == 1 && q > 0.5f && sum > 0.5f)
        diff = (l.rest - expm1f((l.t[j] - l.max) * a.inv_t)) * l.inv - (r.rest - expm1f(u)) * inv;
      v = a.soft_slope * diff;
    }
    if (HARD) {
      float own = exp2_fast(d * LOG2E) * inv1;
      if (c == label) own = own > 0.5f ? (expm1f(d) - r.rest1) * inv1 : own - 1.f;
      v += a.hard * own;
    }
    Elem<T>::store(dz + c, v * inv_rows);
  }
}

// sums of a thread's chunks about the row's largest logit
template <bool HARD, class Row>
__device__ __forceinline__ void add_chunk(const chunk16& q, float max, float inv_t2, bool careful, float& s, float& s1, float& equal) {
#pragma unroll
  for (int e = 0; e < Row::PER; ++e) {
    const float v = Row::value(q, e), d = v - max;
    const float x = share(v, max, inv_t2), x1 = HARD ? exp2_fast(d * LOG2E) : 0.f;
    if (careful && v == max) equal += 1.f;
    else { s += x; s1 += x1; }
  }
}

// What follows the sums of such a row, from memory: beside the registers that hold a row there is no room for it.  (us, 4096 bf16 rows of 65536 with lists of
// 64, which are none of these, at T = 20, so / from the registers 224 / 298, with labels 293 / 378 and at T = 2 254; 64 fp32 rows of 1000, all listed, at T =
// 20 54, at 2 50)
template <class T, int NT, bool HARD>
__device__ __forceinline__ void near_row(const DistillArgs& a, int row, const RowChunks<T>& r, const T* z, T* dz, const List& l, const RowSums& t, int label, float z_label,
                                         float inv_rows, WarmShared<NT>& sh) {
  typedef RowChunks<T> Row;
  const float inv_t2 = a.inv_t * LOG2E;
  const float d = row_reduce<NT>(list_loss<NT>(a, l, t.max), sh.v[2], Add());
  const unsigned long long all = row_reduce<NT>(wholes<NT, Row>(r, z, 0, r.chunks, t.max, inv_t2), sh.n[0], Add());
  const Warm w = warm_of<NT>(a, l, d, t, all, sh);
  if (threadIdx.x % NT == 0) a.loss_rows[row] = loss_of(a, l.length, d, t, w, label, z_label);
  if (!dz) return;
  const Slope g = slope_of(a, t, l.length, inv_rows);
#pragma unroll 1
  for (int c = threadIdx.x % NT; c < r.chunks; c += NT) {
    const chunk16 q = r.load(z, c);
    float v[Row::PER];
#pragma unroll
    for (int e = 0; e < Row::PER; ++e) v[e] = g.template of<HARD>(Row::value(q, e));
    r.store(dz, c, Row::pack(v));
  }
  row_sync<NT>();
  write_listed<T, NT, HARD, true>(a, dz, 0, a.classes, l, t, w, label, z_label, inv_rows);
}

// A row by NT threads, CH chunks each.  lists: 4 list_pitch(k) words of LDS.
template <class T, int NT, int CH, bool HARD, bool WARM>
__device__ __forceinline__ void distill_row(const DistillArgs& a, int row, float* lists, RowShared<NT>& sh, WarmShared<WARM ? NT : 64>& warm) {
  typedef RowChunks<T> Row;
  const int tid = threadIdx.x % NT;
  const T* const z = static_cast<const T*>(a.z) + (size_t)row * a.classes;
  T* const dz = a.dz ? static_cast<T*>(a.dz) + (size_t)row * a.classes : nullptr;
  const Row r(z, a.classes, (long)(a.n - row) * a.classes);
  chunk16 q[CH];
  // (as a lambda: written out behind the return, the compiler keeps the chunks in scratch memory, and 4096 rows of 65536 take 21 ms in place of 0.22)
  auto ask = [&]() {
#pragma unroll
    for (int u = 0; u < CH; ++u)
      if (tid + u * NT < r.chunks) q[u] = r.load(z, tid + u * NT);
  };
  int rows = dz ? count_part<NT>(a) : 0;
  if (!row_counts(a, row)) {
    if (tid == 0) a.loss_rows[row] = 0.f;
    if (dz)
#pragma unroll
      for (int u = 0; u < CH; ++u)
        if (tid + u * NT < r.chunks) r.store(dz, tid + u * NT, chunk16{0, 0, 0, 0});
    return;
  }
  ask();
  List l = list_in(lists, a.k);
  const int label = HARD ? a.labels[row] : -1;
  float z_label = 0.f;
  if (HARD && (unsigned)label < (unsigned)a.classes) z_label = Elem<T>::load(z + label);
  l.length = row_reduce<NT>(list_read<NT>(a, row, l, [&](int, int c) { return Elem<T>::load(z + c); }), sh.n[0], Lower());
  const float own_top = list_end<NT>(a, l);
  float own = -INFINITY;
#pragma unroll
  for (int u = 0; u < CH; ++u)
    if (tid + u * NT < r.chunks) {
      r.cut(q[u], tid + u * NT);
#pragma unroll
      for (int e = 0; e < Row::PER; ++e) own = fmaxf(own, Row::value(q[u], e));
    }
  RowSums t;
  t.max = wave_reduce(own, Larger());
  l.max = wave_reduce(own_top, Larger());
  if constexpr (NT > 64) {
    if ((tid & 63) == 0) { sh.v[0][tid >> 6] = t.max; sh.v[1][tid >> 6] = l.max; }
    __syncthreads();
    t.max = join_waves<NT>(sh.v[0], Larger());
    l.max = join_waves<NT>(sh.v[1], Larger());
  }
  const float inv_t2 = a.inv_t * LOG2E;
  float s = 0.f, s1 = 0.f, equal = 0.f;
  if (own == t.max) {
#pragma unroll
    for (int u = 0; u < CH; ++u)
      if (tid + u * NT < r.chunks) add_chunk<HARD, Row>(q[u], t.max, inv_t2, true, s, s1, equal);
  } else {
#pragma unroll
    for (int u = 0; u < CH; ++u)
      if (tid + u * NT < r.chunks) add_chunk<HARD, Row>(q[u], t.max, inv_t2, false, s, s1, equal);
  }
  float ls, lequal;
  list_sum<NT>(a, l, ls, lequal);
  s = wave_reduce(s, Add());
  equal = wave_reduce(equal, Add());
  rows = wave_reduce(rows, Add());
  if (HARD) s1 = wave_reduce(s1, Add());
  ls = wave_reduce(ls, Add());
  lequal = wave_reduce(lequal, Add());
  if constexpr (NT > 64) {                             // (one barrier for all of them)
    if ((tid & 63) == 0) {
      const int w = tid >> 6;
      sh.v[2][w] = s; sh.v[3][w] = equal; sh.v[4][w] = s1; sh.v[5][w] = ls; sh.v[6][w] = lequal; sh.n[1][w] = rows;
    }
    __syncthreads();
    s = join_waves<NT>(sh.v[2], Add());
    equal = join_waves<NT>(sh.v[3], Add());
    if (HARD) s1 = join_waves<NT>(sh.v[4], Add());
    ls = join_waves<NT>(sh.v[5], Add());
    lequal = join_waves<NT>(sh.v[6], Add());
    rows = join_waves<NT>(sh.n[1], Add());
  }
  const float inv_rows = rows ? 1.f / (float)rows : 0.f;
  const bool none = fabsf(t.max) == INFINITY;          // no distribution
  t.rest = none ? NAN : s + (equal - 1.f);
  t.rest1 = none ? NAN : s1 + (equal - 1.f);
  list_known(l, ls, lequal);
  if constexpr (WARM) {
    if (may_be_near(t, l.length)) return near_row<T, NT, HARD>(a, row, r, z, dz, l, t, label, z_label, inv_rows, warm);      // (the same for all threads)
  }
  float d = wave_reduce(list_loss<NT>(a, l, t.max), Add());
  if (NT > 64 && (tid & 63) == 0) sh.v[7][tid >> 6] = d;
  if (dz) {
    const Slope g = slope_of(a, t, l.length, inv_rows);
#pragma unroll
    for (int u = 0; u < CH; ++u)
      if (tid + u * NT < r.chunks) {
        float v[Row::PER];
#pragma unroll
        for (int e = 0; e < Row::PER; ++e) v[e] = g.template of<HARD>(Row::value(q[u], e));
        r.store(dz, tid + u * NT, Row::pack(v));
      }
  }
  row_sync<NT>();
  if (NT > 64 && tid < 64) d = join_waves<NT>(sh.v[7], Add());
  if (tid == 0) a.loss_rows[row] = loss_of(a, l.length, d, t, Warm{}, label, z_label);
  if (dz) write_listed<T, NT, HARD, false>(a, dz, 0, a.classes, l, t, Warm{}, label, z_label, inv_rows);
}

template <class T, int NT, int CH, bool HARD, bool WARM>
__global__ __launch_bounds__(NT, CH == 8 ? 8 : 4) void distill_rows_kernel(DistillArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lists[];
  __shared__ RowShared<NT> sh;
  __shared__ WarmShared<WARM ? NT : 64> warm;
  distill_row<T, NT, CH, HARD, WARM>(a, blockIdx.x, lists, sh, warm);
}

// A wave per row; in one workgroup (with all rows, four at most) the mean, too
template <class T, int CH, bool HARD, bool WARM>
__global__ __launch_bounds__(256) void distill_waves_kernel(DistillArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lists[];
  const int wave = threadIdx.x >> 6, row = (int)blockIdx.x * (int)(blockDim.x >> 6) + wave;
  if (row < a.n) {
    RowShared<64> sh;                                  // (one wave needs none of it)
    WarmShared<64> warm;
    distill_row<T, 64, CH, HARD, WARM>(a, row, lists + (size_t)wave * 4 * list_pitch(a.k), sh, warm);
  }
  if (gridDim.x > 1 || !a.loss) return;
  __threadfence_block();
  __syncthreads();
  if (threadIdx.x) return;
  double s = 0.0;
  int rows = 0;
  for (int i = 0; i < a.n; ++i) {
    s += (double)a.loss_rows[i];
    rows += row_counts(a, i) ? 1 : 0;
  }
  *a.loss = rows ? (float)(s / (double)rows) : 0.f;
}

// Cut rows: the sums of a part
template <class T, bool HARD>
__global__ __launch_bounds__(256) void distill_part_kernel(DistillArgs a) {
  typedef RowChunks<T> Row;
  __shared__ float sh[4][4];
  const int row = (int)blockIdx.x / a.splits, sp = (int)blockIdx.x - row * a.splits, tid = threadIdx.x;
  const T* const z = static_cast<const T*>(a.z) + (size_t)row * a.classes;
  if (!row_counts(a, row)) return;
  const Row r(z, a.classes, (long)(a.n - row) * a.classes);
  const int c0 = sp * a.chunks_per_split, c1 = min(c0 + a.chunks_per_split, r.chunks);
  if (sp == 0) {
    float* const at = a.at_list + (size_t)row * (a.k + 1);
    for (int j = tid; j < a.k; j += 256) {
      const int c = a.index[(size_t)row * a.k + j];
      at[j] = (unsigned)c < (unsigned)a.classes ? Elem<T>::load(z + c) : NAN;
    }
    if (HARD && tid == 0) at[a.k] = (unsigned)a.labels[row] < (unsigned)a.classes ? Elem<T>::load(z + a.labels[row]) : NAN;
  }
  float own = -INFINITY, s = 0.f, s1 = 0.f, equal = 0.f;
  const float inv_t2 = a.inv_t * LOG2E;
  for (int c = c0 + tid; c < c1; c += 256) {
    chunk16 q = r.load(z, c);
    r.cut(q, c);
#pragma unroll
    for (int e = 0; e < Row::PER; ++e) own = fmaxf(own, Row::value(q, e));
  }
  const float mx = row_reduce<256>(own, sh[0], Larger());
  for (int c = c0 + tid; c < c1; c += 256) {
    chunk16 q = r.load(z, c);
    r.cut(q, c);
    add_chunk<HARD, Row>(q, mx, inv_t2, own == mx, s, s1, equal);
  }
  s = row_reduce<256>(s, sh[1], Add());
  equal = row_reduce<256>(equal, sh[2], Add());
  if (HARD) s1 = row_reduce<256>(s1, sh[3], Add());
  if (tid == 0) {
    float* const p = a.part + (size_t)row * 3 * a.splits + sp;
    const bool none = mx == -INFINITY && !(s != s);    // (nothing but minus infinity: the other parts decide)
    p[0] = mx;
    p[a.splits] = none ? -1.f : s + (equal - 1.f);
    p[2 * a.splits] = none ? -1.f : s1 + (equal - 1.f);
  }
}

// The parts' sums joined, by every wave
__device__ __forceinline__ RowSums sums_of_parts(const DistillArgs& a, int row, int lane) {
  const float* const at = a.part + (size_t)row * 3 * a.splits;
  const bool mine = lane < a.splits;
  const float m = mine ? at[lane] : -INFINITY, rest = mine ? at[a.splits + lane] : -1.f, rest1 = mine ? at[2 * a.splits + lane] : -1.f;
  RowSums t;
  t.max = wave_reduce(m, Larger());
  const bool top = mine && m == t.max;
  float s = top ? rest : (1.f + rest) * exp2_fast((m - t.max) * (a.inv_t * LOG2E)), s1 = top ? rest1 : (1.f + rest1) * exp2_fast((m - t.max) * LOG2E);
  if (!mine) s = s1 = 0.f;
  const float equal = wave_reduce(top ? 1.f : 0.f, Add());
  s = wave_reduce(s, Add());
  s1 = wave_reduce(s1, Add());
  const bool none = fabsf(t.max) == INFINITY;
  t.rest = none ? NAN : s + (equal - 1.f);
  t.rest1 = none ? NAN : s1 + (equal - 1.f);
  return t;
}

// Cut rows at high temperatures: a part's exponentials about the row's largest logit, in whole numbers
template <class T>
__global__ __launch_bounds__(256) void distill_shares_kernel(DistillArgs a) {
  typedef RowChunks<T> Row;
  __shared__ unsigned long long sh[4];
  const int row = (int)blockIdx.x / a.splits, sp = (int)blockIdx.x - row * a.splits, tid = threadIdx.x, lane = tid & 63;
  if (!row_counts(a, row)) return;
  const RowSums t = sums_of_parts(a, row, lane);
  if (!may_be_near(t, a.k)) return;                    // (no list is longer)
  const T* const z = static_cast<const T*>(a.z) + (size_t)row * a.classes;
  const Row r(z, a.classes, (long)(a.n - row) * a.classes);
  const int c0 = sp * a.chunks_per_split, c1 = min(c0 + a.chunks_per_split, r.chunks);
  const float inv_t2 = a.inv_t * LOG2E;
  const unsigned long long all = row_reduce<256>(wholes<256, Row>(r, z, c0, c1, t.max, inv_t2), sh, Add());
  if (tid == 0) a.shares[(size_t)row * a.splits + sp] = all;
}

// Cut rows: the parts joined (64 at most), the loss by the first workgroup, a part of the gradient by each
template <class T, bool HARD, bool WARM>
__global__ __launch_bounds__(256) void distill_join_kernel(DistillArgs a) {
  typedef RowChunks<T> Row;
  extern __shared__ __attribute__((aligned(16))) float lists[];
  __shared__ WarmShared<256> warm;
  __shared__ int shc[4], shn[4];
  __shared__ float sh[4][4];
  const int row = (int)blockIdx.x / a.splits, sp = (int)blockIdx.x - row * a.splits, tid = threadIdx.x, lane = tid & 63;
  const int rows = row_reduce<256>(count_part<256>(a), shc, Add());
  const float inv_rows = rows ? 1.f / (float)rows : 0.f;
  const T* const z = static_cast<const T*>(a.z) + (size_t)row * a.classes;
  T* const dz = a.dz ? static_cast<T*>(a.dz) + (size_t)row * a.classes : nullptr;
  const Row r(z, a.classes, (long)(a.n - row) * a.classes);
  const int c0 = sp * a.chunks_per_split, c1 = min(c0 + a.chunks_per_split, r.chunks);
  if (!row_counts(a, row)) {
    if (tid == 0 && sp == 0) a.loss_rows[row] = 0.f;
    if (dz)
      for (int c = c0 + tid; c < c1; c += 256) r.store(dz, c, chunk16{0, 0, 0, 0});
    return;
  }
  const bool mine = lane < a.splits;
  const RowSums t = sums_of_parts(a, row, lane);
  const float* const kept = a.at_list + (size_t)row * (a.k + 1);
  const int label = HARD ? a.labels[row] : -1;
  const float z_label = HARD ? kept[a.k] : 0.f;
  List l = list_in(lists, a.k);
  l.length = row_reduce<256>(list_read<256>(a, row, l, [&](int j, int) { return kept[j]; }), shn, Lower());
  l.max = row_reduce<256>(list_end<256>(a, l), sh[0], Larger());
  float ls, lequal;
  list_sum<256>(a, l, ls, lequal);
  ls = row_reduce<256>(ls, sh[1], Add());
  lequal = row_reduce<256>(lequal, sh[2], Add());
  list_known(l, ls, lequal);
  const float d = row_reduce<256>(list_loss<256>(a, l, t.max), sh[3], Add());
  Warm w{};
  if constexpr (WARM) {
    if (may_be_near(t, l.length)) w = warm_of<256>(a, l, d, t, wave_reduce(mine ? a.shares[(size_t)row * a.splits + lane] : 0ull, Add()), warm);
  }
  if (tid == 0 && sp == 0) a.loss_rows[row] = loss_of(a, l.length, d, t, w, label, z_label);
  if (!dz) return;
  const Slope g = slope_of(a, t, l.length, inv_rows);
  for (int c = c0 + tid; c < c1; c += 256) {
    const chunk16 q = r.load(z, c);
    float v[Row::PER];
#pragma unroll
    for (int e = 0; e < Row::PER; ++e) v[e] = g.template of<HARD>(Row::value(q, e));
    r.store(dz, c, Row::pack(v));
  }
  __syncthreads();
  write_listed<T, 256, HARD, WARM>(a, dz, r.at(c0), c1 < r.chunks ? r.at(c1) : a.classes, l, t, w, label, z_label, inv_rows);
}

// loss = sum of loss_rows / rows that count, in a fixed order; `parts` sums of parts, or the rows themselves (0)
__global__ __launch_bounds__(1024) void distill_mean_kernel(DistillArgs a, const double* sums, int parts) {
  __shared__ int sh[16];
  __shared__ double shd[16];
  double s = 0.0;
  if (parts) {
    for (int i = threadIdx.x; i < parts; i += 1024) s += sums[i];
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < a.n; i += 1024) s += (double)a.loss_rows[i];
  }
  const int rows = row_reduce<1024>(count_part<1024>(a), sh, Add());
  s = row_reduce<1024>(s, shd, Add());
  if (threadIdx.x == 0) *a.loss = rows ? (float)(s / (double)rows) : 0.f;
}
// sums of the loss of `each` rows
__global__ __launch_bounds__(256) void distill_sum_kernel(DistillArgs a, double* sums, int each) {
  __shared__ double sh[4];
  double s = 0.0;
  const int first = (int)blockIdx.x * each, end = min(first + each, a.n);
#pragma unroll 4
  for (int i = first + (int)threadIdx.x; i < end; i += 256) s += (double)a.loss_rows[i];
  s = row_reduce<256>(s, sh, Add());
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}
// rows that count, `each` rows to a workgroup
__global__ __launch_bounds__(256) void distill_count_kernel(DistillArgs a, int* counts, int each) {
  __shared__ int sh[4];
  int c = 0;
  const int first = (int)blockIdx.x * each, end = min(first + each, a.n);
#pragma unroll 4
  for (int i = first + (int)threadIdx.x; i < end; i += 256) c += row_counts(a, i) ? 1 : 0;
  c = row_reduce<256>(c, sh, Add());
  if (threadIdx.x == 0) counts[blockIdx.x] = c;
}

struct DistillPlan {
  bool waves;                  // a wave per row, an entry of its list to a lane
  bool one;                    // four rows at most, in one workgroup, with the mean
  int splits, chunks_per_split;      // 1: a workgroup per row
  int chunks;
  int count_parts, count_each; // rows that count: parts of so many rows (256 at most); 0: every workgroup counts them all
  bool sum_parts;              // the loss by parts of as many rows
  size_t rows, counts, sums, part, at_list, shares, total;
};
DistillPlan distill_plan(int n, int classes, int k, int dtype) {
  DistillPlan p{};
  const int per = dtype == DT_BF16 ? 8 : 4;
  p.chunks = (classes + per - 1) / per + (classes % per ? 1 : 0);      // (a row begins inside one where the rows are not whole ones)
  // (us, fp32, a wave per row / a workgroup per row: 41 rows of 500 7.8 / 7.7, of 1000 8.5 / 7.5, 1000 of 250 10.8 / 10.7, of 1000 12.6 / 11.4, 2000 of 1000
  // 12.9 / 14.0, 4096 of 250 12.1 / 18.0, of 1000 16.6 / 20.1; the mean by the same workgroup / by another launch: 1 of 1000 6.3 / 8.3, 4 of 1000 7.7 / 8.4, 16
  // of 1000 11.6 / 8.6)
  p.one = p.chunks <= 64 * 4 && k <= 64 && n <= 4;
  p.waves = p.one || (p.chunks <= (n > 1536 ? 64 * 4 : 64 * 2) && k <= 64);
  p.splits = 1;
  // more than a workgroup's registers: 64 KiB to a part, 64 parts at most; few long rows: 8 KiB  (us, so / in one piece: 3 bf16 rows of 111759 15 / 33, of
  // 33591 13.0 / 14.7, 32 of 54159 15.5 / 20.6, 8 fp32 of 10000, which are in one piece, 12.6 / 10.3)
  const bool few = n <= 32 && p.chunks > 4096;
  if (p.chunks > 1024 * 16 || few) {
    p.splits = few && p.chunks < 64 * 512 ? (int)ceil_div(p.chunks, 512) : few ? 64 : (int)ceil_div(p.chunks, 4112);
    p.chunks_per_split = (int)ceil_div(p.chunks, p.splits);
  }
  p.count_each = n > 65536 ? (int)ceil_div(n, 256) : 256;
  p.count_parts = n > 1024 ? (int)ceil_div(n, p.count_each) : 0;      // (with it / without: 1025 rows 9.6 / 10.5, 2048 10.4 / 16.0, 4096 12.0 / 38.9)
  p.sum_parts = n > 32768;      // (one launch / two, us: 16385 rows 23.0 / 23.8, 65536 66 / 64, 262144 244 / 225)
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.rows = take((size_t)n * 4);
  p.sums = take(p.sum_parts ? (size_t)p.count_parts * 8 : 0);
  p.counts = take((size_t)p.count_parts * 4);
  p.part = take(p.splits > 1 ? (size_t)n * 3 * p.splits * 4 : 0);
  p.at_list = take(p.splits > 1 ? (size_t)n * (k + 1) * 4 : 0);
  p.shares = take(p.splits > 1 ? (size_t)n * p.splits * 8 : 0);
  p.total = at;
  return p;
}
bool distill_ok(int n, int classes, int k, int dtype) {
  return n > 0 && classes > 0 && k > 0 && n <= kMostRows && classes <= kMostClasses && k <= kMostTop && (dtype == DT_F32 || dtype == DT_BF16) &&
         (long)n * distill_plan(n, classes, k, dtype).splits < 1L << 22;       // (a launch has fewer than 2^32 threads)
}

template <class T, bool HARD, bool WARM> hipError_t launch_distill(const DistillArgs& a, const DistillPlan& p, hipStream_t st) {
  const size_t lists = (size_t)4 * list_pitch(a.k) * 4;
  if (p.splits > 1) {
    const dim3 grid((unsigned)(a.n * p.splits));
    hipLaunchKernelGGL((distill_part_kernel<T, HARD>), grid, dim3(256), 0, st, a);
    if (WARM) hipLaunchKernelGGL(distill_shares_kernel<T>, grid, dim3(256), 0, st, a);
    hipLaunchKernelGGL((distill_join_kernel<T, HARD, WARM>), grid, dim3(256), lists, st, a);
  } else if (p.waves) {
    const int threads = p.one ? 64 * a.n : 64;
    const dim3 grid(p.one ? 1u : (unsigned)ceil_div(a.n, threads / 64));
#define ACC_WAVES(CH) hipLaunchKernelGGL((distill_waves_kernel<T, CH, HARD, WARM>), grid, dim3(threads), lists * (threads / 64), st, a)
    if (p.chunks <= 64) ACC_WAVES(1);
    else if (p.chunks <= 128) ACC_WAVES(2);
    else ACC_WAVES(4);
#undef ACC_WAVES
  } else {
#define ACC_ROWS(NT, CH) if (p.chunks <= NT * CH) { hipLaunchKernelGGL((distill_rows_kernel<T, NT, CH, HARD, WARM>), dim3((unsigned)a.n), dim3(NT), lists, st, a); break; }
    do {
      ACC_ROWS(256, 2) ACC_ROWS(256, 4) ACC_ROWS(256, 8) ACC_ROWS(512, 8) ACC_ROWS(1024, 8) ACC_ROWS(1024, 16)
    } while (false);
#undef ACC_ROWS
  }
  return hipGetLastError();
}

}  // namespace

size_t distill_workspace_bytes(int n, int classes, int k, int dtype) { return distill_ok(n, classes, k, dtype) ? distill_plan(n, classes, k, dtype).total : 0; }

hipError_t distill(const void* z, const int32_t* index, const float* top, const int32_t* labels, int ignore, float temperature, float alpha, float* loss_rows,
                   float* loss, void* dz, int n, int classes, int k, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!z || !index || !top || !workspace || !(loss_rows || loss || dz) || !distill_ok(n, classes, k, dtype)) return hipErrorInvalidValue;
  if (!(temperature >= 1e-18f && temperature <= 1e18f) || !(alpha > 0.f && alpha <= 1.f) || (!labels && alpha != 1.f)) return hipErrorInvalidValue;
  const DistillPlan p = distill_plan(n, classes, k, dtype);
  if (workspace_bytes < p.total) return hipErrorInvalidValue;
  char* const ws = (char*)workspace;
  DistillArgs a{};
  a.z = z; a.index = index; a.top = top; a.labels = labels; a.ignore = ignore;
  a.inv_t = 1.f / temperature; a.soft = alpha * temperature * temperature; a.hard = 1.f - alpha; a.soft_slope = alpha * temperature;
  a.alpha = alpha; a.t2 = temperature * temperature;
  a.loss_rows = loss_rows ? loss_rows : (float*)(ws + p.rows);
  a.loss = loss; a.dz = dz; a.n = n; a.classes = classes; a.k = k;
  a.part = (float*)(ws + p.part); a.at_list = (float*)(ws + p.at_list); a.shares = (unsigned long long*)(ws + p.shares);
  a.splits = p.splits; a.chunks_per_split = p.chunks_per_split;
  if (p.count_parts && (dz || loss)) {
    int* const counts = (int*)(ws + p.counts);
    hipLaunchKernelGGL(distill_count_kernel, dim3((unsigned)p.count_parts), dim3(256), 0, st, a, counts, p.count_each);
    a.counts = counts; a.count_parts = p.count_parts;
  }
  const bool hard = alpha < 1.f, warm = temperature > kWarm;
  hipError_t e;
#define ACC_DISTILL(T) \
  e = hard ? warm ? launch_distill<T, true, true>(a, p, st) : launch_distill<T, true, false>(a, p, st) \
           : warm ? launch_distill<T, false, true>(a, p, st) : launch_distill<T, false, false>(a, p, st)
  if (dtype == DT_BF16) ACC_DISTILL(bf16_t);
  else ACC_DISTILL(float);
#undef ACC_DISTILL
  if (e != hipSuccess || !loss || p.one) return e;
  double* const sums = (double*)(ws + p.sums);
  if (p.sum_parts) hipLaunchKernelGGL(distill_sum_kernel, dim3((unsigned)p.count_parts), dim3(256), 0, st, a, sums, p.count_each);
  hipLaunchKernelGGL(distill_mean_kernel, dim3(1), dim3(1024), 0, st, a, sums, p.sum_parts ? p.count_parts : 0);
  return hipGetLastError();
}

}  // namespace acc
