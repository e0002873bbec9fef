// A gated linear layer: two projections of the same rows, of which one, through an activation, scales the other.
//
//   ab = x w^T + bias, w [2 f][d]: rows of the gate a, then of the value b;  h = act(a) b
//   da = dh b act'(a),  db = dh act(a);  with dz = [da | db]:  dx = dz w,  dw = dz^T x,  dbias = sum over the rows of dz
//
// 4 rows d f operations forward, 8 backward and 4 more where the projections were not kept: bound by the matrix cores but for few rows, where reading w is.
// Gate and value are worked out by the same workgroup, so that neither is in memory unless it is to be kept.  The backward pass writes dz (a workspace), as
// two products read it.  Few tiles: the projections' sums are cut, and launches that work value by value add the parts and do the rest.
// Up to three or four rows: every wave takes a few columns and all rows, the layer's weights once through the vector units.
//
// fp32, us: 2009 rows, 2048 to 2 x 1365 (22 GFLOP) forward 144, its two launches' sums 134 (168 TFLOP/s) and h 10; all gradients 313 (143 TFLOP/s).  12544 x
// 1024 x 4096 1037 (203 TFLOP/s) and 2624 (160).  Value by value, bf16, kept projections of 12544 rows of 2 x 4096 and dh, to dz in two values: 112, 6.4
// TB/s.
#include "kernels.h"
#include "glu.h"
#include "product32.h"

#include <type_traits>

namespace acc {
namespace {

typedef uint32_t any16 __attribute__((ext_vector_type(4), aligned(2)));

// V neighbouring values as floats, at any address that the type allows; `left` of them exist
template <class T, int V> __device__ __forceinline__ void get(const T* p, int left, float (&v)[V]) {
  if (V > 1 && left >= V) {
    if constexpr (sizeof(T) == 2) {
      const any16 q = *reinterpret_cast<const any16*>(p);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = __uint_as_float(e & 1 ? q[e >> 1] & 0xffff0000u : q[e >> 1] << 16);
    } else {
      const f32x4_any q = *reinterpret_cast<const f32x4_any*>(p);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = q[e];
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = e < left ? Elem<T>::load(p + e) : 0.f;
}
template <class T, int V> __device__ __forceinline__ void put(T* p, int left, const float (&v)[V]) {
  if (V > 1 && left >= V) {
    if constexpr (sizeof(T) == 2) {
      any16 q;
#pragma unroll
      for (int e = 0; e < V / 2; ++e) q[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
      *reinterpret_cast<any16*>(p) = q;
    } else {
      f32x4_any q;
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = v[e];
      *reinterpret_cast<f32x4_any*>(p) = q;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (e < left) Elem<T>::store(p + e, v[e]);
}

// V values from column c on of a row of f, zeros or values of no use behind its end.  The last ones of a row that is no whole number of them are read with
// their neighbours before them and shifted: one by one, a load waits for the other (22419 rows of kept projections 2 x 1205 to dz in two values 245 us).
template <class T, int V> __device__ __forceinline__ void get_row(const T* row, int c, int f, float (&v)[V]) {
  if (f < V) return get<T, V>(row + c, f - c, v);
  const int over = c - min(c, f - V);
  get<T, V>(row + (c - over), V, v);
  if (f % V == 0) return;
#pragma unroll
  for (int by = V / 2; by > 0; by /= 2)
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = over & by ? (e + by < V ? v[e + by] : 0.f) : v[e];
}

// ---------------------------------------------------------------------------------- value by value
template <class T> struct PointWidth { static constexpr int value = 16 / (int)sizeof(T); };

template <class T, bool BWD, int PARTS, bool SUMS>
__global__ __launch_bounds__(256) void glu_point_kernel(PointArgs a) {
  constexpr int V = PointWidth<T>::value;
  __shared__ float sh[BWD ? 2 * V : 1][256];
  const int tx = threadIdx.x % a.tx, ty = threadIdx.x / a.tx, step = 256 / a.tx;
  const int across = (int)blockIdx.x % a.across, slab = (int)blockIdx.x / a.across;
  const int c = (across * a.tx + tx) * V, left = ty < step ? a.f - c : 0;
  const size_t whole = (size_t)a.rows * 2 * a.half;
  float ba[V], bb[V], sa[V], sb[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    ba[e] = a.bias && e < left ? a.bias[c + e] : 0.f;
    bb[e] = a.bias && e < left ? a.bias[a.f + c + e] : 0.f;
    sa[e] = sb[e] = 0.f;
  }
  const int r1 = min((slab + 1) * a.slab, a.rows);
  for (int r = slab * a.slab + ty; r < r1 && left > 0; r += step) {
    float g[V], v[V];
    if constexpr (SUMS) {
      const float* const from = a.sums + (size_t)r * 2 * a.half;
#pragma unroll
      for (int e = 0; e < V; ++e) { g[e] = ba[e]; v[e] = bb[e]; }
      auto add = [&](int s0, auto several) {           // so many parts on their way at once
        constexpr int U = decltype(several)::value;
        float p[U][V], q[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < V; e += 4) {
            get_row<float, 4>(from + (s0 + u) * whole, c + e, a.half, *reinterpret_cast<float(*)[4]>(&p[u][e]));
            get_row<float, 4>(from + (s0 + u) * whole + a.half, c + e, a.half, *reinterpret_cast<float(*)[4]>(&q[u][e]));
          }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e) { g[e] += p[u][e]; v[e] += q[u][e]; }
      };
      int s = 0;
      for (; s + 4 <= a.splits; s += 4) add(s, std::integral_constant<int, 4>());
      for (; s < a.splits; ++s) add(s, std::integral_constant<int, 1>());
    } else {
      const T* const from = static_cast<const T*>(a.ab_in) + (size_t)r * 2 * a.f;
      get_row<T, V>(from, c, a.f, g);
      get_row<T, V>(from + a.f, c, a.f, v);
    }
    if constexpr (!BWD) {
      float h[V];
#pragma unroll
      for (int e = 0; e < V; ++e) h[e] = glu_act(a.act, g[e]) * v[e];
      put<T, V>(static_cast<T*>(a.h) + (size_t)r * a.f + c, left, h);
      if (a.ab) {
        T* const to = static_cast<T*>(a.ab) + (size_t)r * 2 * a.f + c;
        put<T, V>(to, left, g);
        put<T, V>(to + a.f, left, v);
      }
    } else {
      float dh[V];
      get_row<T, V>(static_cast<const T*>(a.dh) + (size_t)r * a.f, c, a.f, dh);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float da, db;
        glu_slopes(a.act, g[e], v[e], dh[e], da, db);
        g[e] = e < left ? da : 0.f;
        v[e] = e < left ? db : 0.f;
        {
#pragma clang fp contract(off)                         // (the same bits whether dz is written or not)
          sa[e] += g[e];
          sb[e] += v[e];
        }
      }
      // (columns up to a.half exist and are zero from a.f on)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) {
        T* const to = static_cast<T*>(a.dz[part]) + (size_t)r * a.pitch + c;
        put<T, V>(to, a.half - c, g);
        put<T, V>(to + a.half, a.half - c, v);
        if (part + 1 < PARTS) {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const uint32_t p = pack_bf16(g[e], g[e + 1]), q = pack_bf16(v[e], v[e + 1]);
            g[e] -= __uint_as_float(p << 16); g[e + 1] -= __uint_as_float(p & 0xffff0000u);
            v[e] -= __uint_as_float(q << 16); v[e + 1] -= __uint_as_float(q & 0xffff0000u);
          }
        }
      }
    }
  }
  if constexpr (BWD) {
    if (!a.db_part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) { sh[e][threadIdx.x] = sa[e]; sh[V + e][threadIdx.x] = sb[e]; }
    __syncthreads();
    // column e of the tx threads that hold it, row by row of threads
    for (int i = threadIdx.x; i < a.tx * 2 * V; i += 256) {
      const int t = i % a.tx, e = i / a.tx, col = (across * a.tx + t) * V + (e % V);
      if (col >= a.f) continue;
      float s = 0.f;
      for (int y = 0; y < step; ++y) s += sh[e][y * a.tx + t];
      a.db_part[(size_t)slab * a.pitch + col + (e < V ? 0 : a.half)] = s;
    }
  }
}

// ---------------------------------------------------------------------------------- sums of parts
// Many parts of few values: sixty-four values to a workgroup, a quarter of the parts to each wave
template <class T> __device__ __forceinline__ void join_many(const float* __restrict__ sums, T* __restrict__ out, size_t count, int splits, size_t block) {
  __shared__ float sh[256];
  const size_t i = block * 64 + (threadIdx.x & 63);
  const int each = (splits + 3) / 4, k0 = (int)(threadIdx.x >> 6) * each, k1 = min(k0 + each, splits);
  float s = 0.f;
  if (i < count) {
#pragma unroll 8
    for (int k = k0; k < k1; ++k) s += sums[(size_t)k * count + i];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 64 && i < count) Elem<T>::store(out + i, ((s + sh[threadIdx.x + 64]) + sh[threadIdx.x + 128]) + sh[threadIdx.x + 192]);
}
// (us, all gradients, fp32, so / a value to a thread: 196 x 512 x 1024, some eight parts, 36 / 41, 48 x 456 23 / 28; more values 777 x 1160 118 / 114, 1000 x
// 512 51 / 48)
inline bool many_parts(size_t count, int splits) { return splits >= 16 ? count <= 1u << 20 : splits >= 4 && count <= 1u << 18; }
template <class T>
__global__ __launch_bounds__(256) void glu_finish_kernel(GluFinish f, unsigned dx_blocks, unsigned dw_blocks, int many) {
  unsigned block = blockIdx.x;
  if (block < dx_blocks)
    return many & 1 ? join_many<T>(f.dx_sums, (T*)f.dx, f.dx_count, f.dx_splits, block) : join_sums<T>(f.dx_sums, (T*)f.dx, f.dx_count, f.dx_splits, block, dx_blocks);
  block -= dx_blocks;
  if (block < dw_blocks)
    return many & 2 ? join_many<float>(f.dw_sums, f.dw, f.dw_count, f.dw_splits, block) : join_sums<float>(f.dw_sums, f.dw, f.dw_count, f.dw_splits, block, dw_blocks);
  block -= dw_blocks;
  glu_db(f, (int)block);
}

// sixty-four columns of a slab, every fourth of its rows to a wave
__global__ __launch_bounds__(256) void glu_db_slabs_kernel(const float* __restrict__ part, float* __restrict__ slabs, int parts, int each, int pitch, int across) {
  __shared__ double sh[256];
  const int slab = (int)blockIdx.x / across, j = ((int)blockIdx.x - slab * across) * 64 + (threadIdx.x & 63);
  const int first = slab * each, end = min(first + each, parts);
  double s = 0.0;
  if (j < pitch) {
#pragma unroll 8
    for (int r = first + (int)(threadIdx.x >> 6); r < end; r += 4) s += (double)part[(size_t)r * pitch + j];
  }
  sh[threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x < 64 && j < pitch) slabs[(size_t)slab * pitch + j] = (float)(((s + sh[threadIdx.x + 64]) + sh[threadIdx.x + 128]) + sh[threadIdx.x + 192]);
}

// ---------------------------------------------------------------------------------- few rows R rows: a wave's columns one after the other, sixteen bytes of
// gate and value rows of w to a lane, all rows of x against them.  (All loads of four steps are on their way at once: with a test of the row's end around each,
// 4 rows of 2048 to 2 x 8192 took 30 us in place of 16.)
template <class T, int R>
__global__ __launch_bounds__(256) void glu_few_kernel(const T* __restrict__ x, const T* __restrict__ w, const float* __restrict__ bias, T* __restrict__ h,
                                                      T* __restrict__ ab, int d, int f, int act) {
  constexpr int V = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 63, waves = (int)gridDim.x * 4;
  for (int c = (int)blockIdx.x * 4 + (threadIdx.x >> 6); c < f; c += waves) {
    const T *const wa = w + (size_t)c * d, *const wb = w + (size_t)(f + c) * d;
    float a[R], b[R];
#pragma unroll
    for (int r = 0; r < R; ++r) a[r] = b[r] = 0.f;
    auto add = [&](int k, int left) {
      float va[V], vb[V], vx[R][V];
      get<T, V>(wa + k, left, va);
      get<T, V>(wb + k, left, vb);
#pragma unroll
      for (int r = 0; r < R; ++r) get<T, V>(x + (size_t)r * d + k, left, vx[r]);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          a[r] = fmaf(va[e], vx[r][e], a[r]);
          b[r] = fmaf(vb[e], vx[r][e], b[r]);
        }
    };
    int k = lane * V;
#pragma unroll 4
    for (; k + V <= d; k += 64 * V) add(k, V);
    if (k < d) add(k, d - k);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) { a[r] += __shfl_xor(a[r], o); b[r] += __shfl_xor(b[r], o); }
    const float ba = bias ? bias[c] : 0.f, bb = bias ? bias[f + c] : 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (lane == r) {
        const float g = a[r] + ba, v = b[r] + bb;
        Elem<T>::store(h + (size_t)r * f + c, glu_act(act, g) * v);
        if (ab) {
          Elem<T>::store(ab + (size_t)r * 2 * f + c, g);
          Elem<T>::store(ab + (size_t)r * 2 * f + f + c, v);
        }
      }
  }
}
// (us, so / by tiles: 1 row of 512 to 2 x 2048 bf16 3.9 / 5.8, fp32 3.8 / 8.4; 4 rows, bf16, 1024 to 2 x 4096 5.6 / 7.5, 2048 to 2 x 8192 16.0 / 12.8; 3 rows
// of that 13.1 / 12.9; 4 rows of it in fp32 22 / 27; 1 row of 4096 to 2 x 11008 26.7 / 27.9, which is 6.8 TB/s of weights that the caches hold.)
inline bool few_rows(int rows, int d, int f, int dtype) { return rows <= 3 || (rows == 4 && (dtype == DT_F32 || (long)d * f <= 1L << 23)); }
template <class T> hipError_t glu_few(const GluArgs& a) {
  const long blocks = ceil_div(a.f, 4);
  const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
#define ACC_FEW(R) hipLaunchKernelGGL((glu_few_kernel<T, R>), grid, dim3(256), 0, a.st, (const T*)a.x, (const T*)a.w, a.bias, (T*)a.h, (T*)a.ab, a.d, a.f, a.act)
  switch (a.rows) {
    case 1: ACC_FEW(1); break;
    case 2: ACC_FEW(2); break;
    case 3: ACC_FEW(3); break;
    default: ACC_FEW(4);
  }
#undef ACC_FEW
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------- fp32 products
struct Pair32 {
  Gemm32Operand x, w;          // w.second: from the gate's rows to the value's
  const float* bias;
  int rows, d, f, act, tiles_m, tiles;
  float *h, *ab;               // forward
  const float* dh;             // backward
  float *dz, *db_part;         // each may be null
};
template <class C, bool BWD>
__global__ __launch_bounds__(C::THREADS) void glu32_kernel(Pair32 a, int blocks) {
  __shared__ __attribute__((aligned(16))) float lds[C::LDS];
  const int at = xcd_tile(blocks);
  if (at >= a.tiles) return;
  const TileAt where = tile_at(at, a.tiles_m, a.tiles);
  const int m0 = where.m * C::BM, n0 = where.n * (C::BN / 2);
  Gemm32Acc<C> acc;
  gemm32_tile<C>(a.x, a.w, m0, n0, 0, a.d, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm0 = (wave / C::WN) * 16 * C::MB, col0 = n0 + (wave % C::WN) * 8 * C::NB + 4 * (lane >> 4);
  const size_t f = a.f;
#pragma unroll
  for (int j = 0; j < C::NB / 2; ++j) {
    const int c = col0 + 16 * j, left = a.f - c;
    float ba[4], bb[4], sa[4], sb[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ba[e] = a.bias && e < left ? a.bias[c + e] : 0.f;
      bb[e] = a.bias && e < left ? a.bias[f + c + e] : 0.f;
      sa[e] = sb[e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < C::MB; ++i) {
      const int m = m0 + wm0 + 16 * i + (lane & 15);
      if (m >= a.rows || left <= 0) continue;
      float g[4], v[4], o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) { g[e] = acc[i][2 * j][e] + ba[e]; v[e] = acc[i][2 * j + 1][e] + bb[e]; }
      if constexpr (!BWD) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = glu_act(a.act, g[e]) * v[e];
        put<float, 4>(a.h + m * f + c, left, o);
        if (a.ab) {
          put<float, 4>(a.ab + m * 2 * f + c, left, g);
          put<float, 4>(a.ab + m * 2 * f + f + c, left, v);
        }
      } else {
        get<float, 4>(a.dh + m * f + c, left, o);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float da, db;
          glu_slopes(a.act, g[e], v[e], o[e], da, db);
          g[e] = da;
          v[e] = db;
          sa[e] += da;
          sb[e] += db;
        }
        if (a.dz) {
          put<float, 4>(a.dz + m * 2 * f + c, left, g);
          put<float, 4>(a.dz + m * 2 * f + f + c, left, v);
        }
      }
    }
    if (BWD && a.db_part) {
      float* const to = a.db_part + (size_t)(where.m * C::WM + wave / C::WN) * 2 * f + c;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) { sa[e] += __shfl_xor(sa[e], o); sb[e] += __shfl_xor(sb[e], o); }
        if ((lane & 15) == 0 && e < left) { to[e] = sa[e]; to[f + e] = sb[e]; }
      }
    }
  }
}

// dx, dw and db in one launch of 64 x 64 tiles: they all wait for dz only, so where there are few tiles two launches less
typedef Gemm32Cfg<2, 2, 2, 2, false, true, false> GluDx64;
typedef Gemm32Cfg<2, 2, 2, 2, true, true, false> GluDw64;
__global__ __launch_bounds__(256) void glu_grads32_kernel(Product32 dx, Product32 dw, GluFinish f, int dx_blocks, int dw_blocks) {
  __shared__ __attribute__((aligned(16))) float lds[GluDx64::LDS > GluDw64::LDS ? GluDx64::LDS : GluDw64::LDS];
  const int block = blockIdx.x;                        // (each part begins at a multiple of eight)
  if (block < dx_blocks) {
    const int work = (block & 7) * (dx_blocks >> 3) + (block >> 3);
    if (work < dx.work) product32<GluDx64>(dx, work, lds);
  } else if (block < dx_blocks + dw_blocks) {
    const int work = (block & 7) * (dw_blocks >> 3) + ((block - dx_blocks) >> 3);
    if (work < dw.work) product32<GluDw64>(dw, work, lds);
  } else {
    glu_db(f, block - dx_blocks - dw_blocks);
  }
}

constexpr double kSaved = 3.0;         // us: a launch that adds parts

struct GluPlan32 {
  int tile;
  bool cut;
  bool together;
  Cut proj, dx, dw;
  int db_parts;
  size_t sums, dz, dx_sums, dw_sums, db, slabs, total;
};
GluPlan32 glu_plan32(int rows, int d, int f, bool backward, bool kept) {
  GluPlan32 p{};
  const long wide = 2L * f;
  const Cut whole = cut32(rows, wide, d, 0);
  p.tile = whole.tile;
  p.proj = cut32(rows, wide, d, 1L << 24);
  // (us, so / whole: forward 64 x 2048 x 512 12 / 51, 300 x 1024 x 64 9.5 / 26.8, 196 x 512 x 1024 14 / 15)
  p.cut = !kept && p.proj.splits > 1 && p.proj.us + 3.0 < whole.us;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t a = at; at += al256(bytes); return a; };
  p.sums = take(p.cut ? (size_t)p.proj.splits * rows * wide * 4 : 0);
  if (backward) {
    p.dx = cut32(rows, d, wide, 1L << 25);
    p.dw = cut32(wide, d, rows, 1L << 25);
    const Cut dx = cut32(rows, d, wide, 1L << 25, 1), dw = cut32(wide, d, rows, 1L << 25, 1);
    // (us, so / each for itself: 196 x 512 x 1024 23.8 / 30.0, 2009 x 512 x 512 55 / 65, 777 x 1160 x 1003, which is more, 106 / 82)
    p.together = ceil_div(d, 64) * (ceil_div(rows, 64) * dx.splits + ceil_div(wide, 64) * dw.splits) <= 1024;
    if (p.together) {
      p.dx = dx; p.dw = dw;
      // (whole sums save the launch that adds parts)
      const Cut x1 = cut32(rows, d, wide, 0, 1), w1 = cut32(wide, d, rows, 0, 1);
      if (x1.us < dx.us + kSaved && w1.us < dw.us + kSaved) { p.dx = x1; p.dw = w1; }
    }
    p.dz = take((size_t)rows * wide * 4);
    p.dx_sums = take(p.dx.splits > 1 ? (size_t)p.dx.splits * rows * d * 4 : 0);
    p.dw_sums = take(p.dw.splits > 1 ? (size_t)p.dw.splits * wide * d * 4 : 0);
    PointArgs q{};
    q.rows = rows; q.f = f;
    p.db_parts = kept || p.cut ? glu_point_shape(q, DT_F32) : (int)ceil_div(rows, kTile32[p.tile][0]) * (p.tile == 0 ? 1 : 2);
    p.db = take((size_t)p.db_parts * wide * 4);
    p.slabs = take(p.db_parts > kDbMany ? (size_t)kDbSlabs * wide * 4 : 0);
  }
  p.total = at;
  return p;
}
template <class C> void launch_pair32(const Pair32& g, bool backward, hipStream_t st) {
  const unsigned blocks = whole_eights(g.tiles);
  if (backward) hipLaunchKernelGGL((glu32_kernel<C, true>), dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
  else hipLaunchKernelGGL((glu32_kernel<C, false>), dim3(blocks), dim3(C::THREADS), 0, st, g, (int)blocks);
}

hipError_t glu32(const GluArgs& a, bool backward) {
  const bool kept = backward && a.ab_in;
  const GluPlan32 p = glu_plan32(a.rows, a.d, a.f, backward, kept);
  const float *x = (const float*)a.x, *w = (const float*)a.w;
  float *const dz = a.dx || a.dw ? (float*)(a.ws + p.dz) : nullptr, *const db_part = backward && a.db ? (float*)(a.ws + p.db) : nullptr;
  hipStream_t st = a.st;
  const int wide = 2 * a.f;
  if (kept || p.cut) {
    PointArgs q{};
    q.ab_in = a.ab_in; q.dh = a.dh; q.h = a.h; q.ab = a.ab; q.dz[0] = dz; q.db_part = db_part;
    q.rows = a.rows; q.f = a.f; q.act = a.act; q.half = a.f; q.pitch = wide;
    if (!kept) {
      Product32 g{};
      g.a = {x, a.rows, a.d}; g.b = {w, wide, a.d}; g.out = (float*)(a.ws + p.sums); g.k = a.d;
      cut_into(g, p.proj);
      if (const hipError_t e = launch_product32<false, false>(g, p.proj, st); e != hipSuccess) return e;
      q.sums = g.out; q.splits = p.proj.splits; q.bias = a.bias;
    }
    glu_point_shape(q, DT_F32);
    if (const hipError_t e = glu_point(q, backward, dz ? 1 : 0, DT_F32, st); e != hipSuccess || !backward) return e;
  } else {
    Pair32 g{};
    g.x = {x, a.rows, a.d}; g.w = {w, a.f, a.d, (uint32_t)a.f * (uint32_t)a.d};
    g.bias = a.bias; g.rows = a.rows; g.d = a.d; g.f = a.f; g.act = a.act;
    g.tiles_m = (int)ceil_div(a.rows, kTile32[p.tile][0]); g.tiles = g.tiles_m * (int)ceil_div(a.f, kTile32[p.tile][1] / 2);
    g.h = (float*)a.h; g.ab = (float*)a.ab; g.dh = (const float*)a.dh; g.dz = dz; g.db_part = db_part;
    if (p.tile == 0) launch_pair32<Gemm32Cfg<1, 4, 2, 2, false, false, false, true>>(g, backward, st);
    else if (p.tile == 1) launch_pair32<Gemm32Cfg<2, 2, 2, 2, false, false, false, true>>(g, backward, st);
    else launch_pair32<Gemm32Cfg<2, 2, 4, 4, false, false, true, true>>(g, backward, st);
    if (!backward) return hipGetLastError();
  }
  GluFinish f{};
  Product32 gx{}, gw{};
  if (a.dx) {
    gx.a = {dz, a.rows, wide}; gx.b = {w, a.d, a.d}; gx.k = wide;
    gx.out = p.dx.splits > 1 ? (float*)(a.ws + p.dx_sums) : (float*)a.dx;
    cut_into(gx, p.dx);
    if (p.dx.splits > 1) { f.dx_sums = gx.out; f.dx = a.dx; f.dx_count = (size_t)a.rows * a.d; f.dx_splits = p.dx.splits; }
  }
  if (a.dw) {
    gw.a = {dz, wide, wide}; gw.b = {x, a.d, a.d}; gw.k = a.rows;
    gw.out = p.dw.splits > 1 ? (float*)(a.ws + p.dw_sums) : a.dw;
    cut_into(gw, p.dw);
    if (p.dw.splits > 1) { f.dw_sums = gw.out; f.dw = a.dw; f.dw_count = (size_t)wide * a.d; f.dw_splits = p.dw.splits; }
  }
  if (a.db) { f.db_part = db_part; f.db = a.db; f.db_parts = p.db_parts; f.pitch = wide; f.half = a.f; f.f = a.f; }
  if (const hipError_t e = glu_db_slabs(f, (float*)(a.ws + p.slabs), st); e != hipSuccess) return e;
  if (p.together) {
    const unsigned bx = whole_eights(gx.work), bw = whole_eights(gw.work);
    hipLaunchKernelGGL(glu_grads32_kernel, dim3(bx + bw + glu_db_blocks(f)), dim3(256), 0, st, gx, gw, f, (int)bx, (int)bw);
  } else {
    if (a.dx) if (const hipError_t e = launch_product32<false, true>(gx, p.dx, st); e != hipSuccess) return e;
    if (a.dw) if (const hipError_t e = launch_product32<true, true>(gw, p.dw, st); e != hipSuccess) return e;
  }
  return glu_finish(f, !p.together, DT_F32, st);
}

// w takes fewer than 4 GiB as bf16 values, a launch fewer than 2^32 threads
bool glu_ok(int rows, int d, int f, int dtype) {
  return rows > 0 && d > 0 && f > 0 && rows <= (1 << 24) && d <= (1 << 16) && f <= (1 << 16) && (long)up(d, 8) * up(f, 8) < (1L << 30) - (1L << 20) &&
         (long)rows * (d + f) <= 1L << 36 && (dtype == DT_F32 || dtype == DT_BF16);
}

}  // namespace

int glu_point_shape(PointArgs& a, int dtype) {
  const int v = dtype == DT_BF16 ? 8 : 4, chunks = (a.f + v - 1) / v;
  // The fewest workgroups across that leave the fewest threads without work, three more than needed at most.  (us, so / the fewest: 22419 bf16 rows of 2 x 1205
  // 71 / 126, 20000 of 2 x 1200 56 / 76, of 2 x 2600 125 / 140)
  const int least = (int)ceil_div(chunks, 256);
  int most = 0;
  for (int across = least; across <= least + 3 && across <= chunks; ++across) {
    // (of 256 threads; whole lines of 128 bytes)
    const int tx = (int)(across > 1 ? up(ceil_div(chunks, across), 8) : chunks), busy = (int)((long)chunks * (256 / tx) / ceil_div(chunks, tx));
    if (busy <= most + most / 16) continue;            // (a sixteenth more, or it is not worth a shorter piece of a row)
    most = busy;
    a.tx = tx;
    a.across = (int)ceil_div(chunks, tx);
  }
  // some thousand workgroups, which run at the same time, at most 512 of them down a column (bf16, 11810 rows of 2 x 4624, us: 127, with twice as many 156)
  const int step = 256 / a.tx;
  long each = ceil_div((long)a.rows * a.across, 1024);
  if (each < ceil_div(a.rows, 512)) each = ceil_div(a.rows, 512);
  a.slab = (int)up(each, step);
  return (int)ceil_div(a.rows, a.slab);
}

hipError_t glu_point(const PointArgs& a, bool backward, int parts, int dtype, hipStream_t st) {
  const dim3 grid((unsigned)(ceil_div(a.rows, a.slab) * a.across));
#define ACC_POINT(T, BWD, PARTS, SUMS) hipLaunchKernelGGL((glu_point_kernel<T, BWD, PARTS, SUMS>), grid, dim3(256), 0, st, a)
  if (!backward) { if (dtype == DT_F32) ACC_POINT(float, false, 1, true); else ACC_POINT(bf16_t, false, 1, true); }
  else if (dtype == DT_F32 && parts) { if (a.sums) ACC_POINT(float, true, 1, true); else ACC_POINT(float, true, 1, false); }
  else if (dtype == DT_F32) { if (a.sums) ACC_POINT(float, true, 0, true); else ACC_POINT(float, true, 0, false); }
  else if (parts == 3) { if (a.sums) ACC_POINT(bf16_t, true, 3, true); else ACC_POINT(bf16_t, true, 3, false); }
  else if (parts == 2) { if (a.sums) ACC_POINT(bf16_t, true, 2, true); else ACC_POINT(bf16_t, true, 2, false); }
  else { if (a.sums) ACC_POINT(bf16_t, true, 0, true); else ACC_POINT(bf16_t, true, 0, false); }
#undef ACC_POINT
  return hipGetLastError();
}

hipError_t glu_db_slabs(GluFinish& f, float* slabs, hipStream_t st) {
  if (!f.db || f.db_parts <= kDbMany) return hipSuccess;
  const int each = (int)ceil_div(f.db_parts, kDbSlabs), across = (int)ceil_div(f.pitch, 64), count = (int)ceil_div(f.db_parts, each);
  hipLaunchKernelGGL(glu_db_slabs_kernel, dim3((unsigned)(count * across)), dim3(256), 0, st, f.db_part, slabs, f.db_parts, each, f.pitch, across);
  f.db_part = slabs;
  f.db_parts = count;
  return hipGetLastError();
}

hipError_t glu_finish(const GluFinish& f, bool db, int dtype, hipStream_t st) {
  const int many = (many_parts(f.dx_count, f.dx_splits) ? 1 : 0) | (many_parts(f.dw_count, f.dw_splits) ? 2 : 0);
  const unsigned bx = f.dx_splits <= 1 ? 0 : many & 1 ? (unsigned)((f.dx_count + 63) / 64) : join_blocks(f.dx_count);
  const unsigned bw = f.dw_splits <= 1 ? 0 : many & 2 ? (unsigned)((f.dw_count + 63) / 64) : join_blocks(f.dw_count);
  const unsigned blocks = bx + bw + (db ? glu_db_blocks(f) : 0);
  if (blocks) {
    if (dtype == DT_F32) hipLaunchKernelGGL(glu_finish_kernel<float>, dim3(blocks), dim3(256), 0, st, f, bx, bw, many);
    else hipLaunchKernelGGL(glu_finish_kernel<bf16_t>, dim3(blocks), dim3(256), 0, st, f, bx, bw, many);
  }
  return hipGetLastError();
}

size_t glu_workspace_bytes(int rows, int d, int f, int backward, int dtype) {
  if (!glu_ok(rows, d, f, dtype)) return 0;
  if (!backward && few_rows(rows, d, f, dtype)) return 0;
  if (dtype == DT_BF16) return glu_bf16_workspace_bytes(rows, d, f, backward != 0);
  const size_t again = glu_plan32(rows, d, f, backward != 0, false).total, kept = backward ? glu_plan32(rows, d, f, true, true).total : 0;
  return again > kept ? again : kept;
}

hipError_t glu_forward(const void* x, const void* w, const float* bias, void* h, void* ab, int rows, int d, int f, int act, void* workspace,
                       size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!x || !w || !h || act < GLU_NONE || act > GLU_SILU || !glu_ok(rows, d, f, dtype)) return hipErrorInvalidValue;
  const size_t need = glu_workspace_bytes(rows, d, f, 0, dtype);
  if (workspace_bytes < need || (need && !workspace)) return hipErrorInvalidValue;
  GluArgs a{};
  a.x = x; a.w = w; a.bias = bias; a.h = h; a.ab = ab; a.rows = rows; a.d = d; a.f = f; a.act = act; a.ws = (char*)workspace; a.dtype = dtype; a.st = st;
  if (few_rows(rows, d, f, dtype)) return dtype == DT_BF16 ? glu_few<bf16_t>(a) : glu_few<float>(a);
  return dtype == DT_BF16 ? glu_bf16(a, false) : glu32(a, false);
}

hipError_t glu_backward(const void* x, const void* w, const float* bias, const void* ab, const void* dh, void* dx, float* dw, float* db, int rows, int d, int f,
                        int act, void* workspace, size_t workspace_bytes, int dtype, hipStream_t st) {
  if (!x || !w || !dh || !workspace || !(dx || dw || db) || act < GLU_NONE || act > GLU_SILU || !glu_ok(rows, d, f, dtype)) return hipErrorInvalidValue;
  if (workspace_bytes < glu_workspace_bytes(rows, d, f, 1, dtype)) return hipErrorInvalidValue;
  GluArgs a{};
  a.x = x; a.w = w; a.bias = bias; a.ab_in = ab; a.dh = dh; a.dx = dx; a.dw = dw; a.db = db;
  a.rows = rows; a.d = d; a.f = f; a.act = act; a.ws = (char*)workspace; a.dtype = dtype; a.st = st;
  return dtype == DT_BF16 ? glu_bf16(a, true) : glu32(a, true);
}

}  // namespace acc
