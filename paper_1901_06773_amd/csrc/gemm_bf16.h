// One tile of a plain matrix product on the bf16 matrix cores, for kernels that do something of their own with it:
//
//   acc[m][n] = sum_k A[m][k] * B[k][n]  (+ the same with a second and third A),   m in [m0, m0 + BM), n in [n0, n0 + BN), k in [k_lo, k_hi)
//
// Each operand lies in memory with its values of k side by side (rows of m resp. n) or with its values of m resp. n side by side (rows of k).
// Either way 16 bytes at a time go straight into LDS as they lie; of the first kind a lane reads its eight values of k, the second kind is transposed
// by the LDS read.  Rows and columns that don't exist read as zero (offsets beyond the descriptor), so edges and a last part of k need no code of
// their own.  Loads of a later chunk stand among the matrix instructions, and the last step of a chunk is multiplied behind the next chunk's barrier,
// when that chunk's first reads are on their way.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "lds_load.h"

namespace acc {

// WM x WN waves, each MB x NB blocks of 32 x 32; BK values of k per chunk, NS stages in LDS.  AT / BT: the operand lies in rows of k.  PARTS: A is
// the sum of so many matrices of the same layout (their products go to the same accumulators).  SWAP: the accumulators are those of the transposed
// block: register v of a lane holds column 8 * (v / 4) + 4 * (lane / 32) + v % 4 of row lane % 32; otherwise row and column change places.
template <int WM_, int WN_, int MB_, int NB_, int BK_, int NS_, bool AT_, bool BT_, int PARTS_, bool SWAP_> struct GemmCfg {
  static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, BK = BK_, NS = NS_, PARTS = PARTS_;
  static constexpr bool AT = AT_, BT = BT_, SWAP = SWAP_;
  static constexpr int THREADS = 64 * WM * WN, BM = 32 * MB * WM, BN = 32 * NB * WN;
  static constexpr int A_PITCH = AT ? BM * 2 : BK * 2, B_PITCH = BT ? BN * 2 : BK * 2;      // bytes of a staged row
  static constexpr int A_COLS = A_PITCH / 16, B_COLS = B_PITCH / 16;
  static constexpr int A_ROWS = AT ? BK : BM, B_ROWS = BT ? BK : BN;
  static constexpr int A_STEP = THREADS / A_COLS, B_STEP = THREADS / B_COLS;                // rows that one load instruction of the workgroup fills
  static constexpr int AI = A_ROWS / A_STEP, BI = B_ROWS / B_STEP;
  static constexpr int A_PART = A_ROWS * A_PITCH, A_BYTES = A_PART * PARTS, STAGE = A_BYTES + B_ROWS * B_PITCH, LDS = NS * STAGE;
  static_assert(AI * A_STEP == A_ROWS && BI * B_STEP == B_ROWS, "whole load instructions");
  static_assert((AT ? A_STEP % 4 : A_STEP % 16) == 0 && (BT ? B_STEP % 4 : B_STEP % 16) == 0, "a thread's rows are permuted alike");
  static_assert(BK % 32 == 0 && (AT || BK <= 64) && NS >= 2 && NS <= 4 && PARTS <= 3, "an even number of steps of 16; rows of 64 or 128 bytes");
};

struct GemmOperand {
  const void* p;         // 16-byte aligned
  const void* more[2];   // the other parts of A
  long rows;             // of m resp. n, or of k
  int cols;              // what lies side by side; a multiple of 8
  int pitch;             // elements between rows; a multiple of 8
};

// A descriptor of the rows [first, first + count) of an operand (as far as they exist), fewer than 4 GiB of them.
__device__ __forceinline__ srsrc operand_rows(const GemmOperand& o, const void* p, long first, long count) {
  const long left = o.rows - first, take = left < count ? left : count;
  return descriptor(static_cast<const char*>(p) + (size_t)first * o.pitch * 2, take > 0 ? (size_t)take * o.pitch * 2 : 0);
}

template <class C> using GemmAcc = v16f[C::MB][C::NB];

template <class C>
__device__ __forceinline__ void gemm_tile(const GemmOperand& A, const GemmOperand& B, int m0, int n0, int k_lo, int k_hi, char* lds,
                                          GemmAcc<C>& acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int MB = C::MB, NB = C::NB, AI = C::AI, BI = C::BI, NS = C::NS, PARTS = C::PARTS, BK = C::BK;
  constexpr uint32_t OUTSIDE = 0xFFFFFFF0u;           // beyond any descriptor range: reads as zero
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / C::WN) * 32 * MB, wn0 = (wave % C::WN) * 32 * NB;
#pragma unroll
  for (int a = 0; a < MB; ++a)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.f;

  // ---- loads.  Rows of m or n: the lane's 16-byte column of k, permuted by the row; rows of k: its column of m or n, permuted likewise
  auto swz = [](int row) { return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3; };
  const int arow = tid / C::A_COLS, brow = tid / C::B_COLS;
  const int acol = C::AT ? (tid % C::A_COLS) ^ (row_xor<C::A_PITCH>(arow) << 2) : (tid % C::A_COLS) ^ swz(arow);
  const int bcol = C::BT ? (tid % C::B_COLS) ^ (row_xor<C::B_PITCH>(brow) << 2) : (tid % C::B_COLS) ^ swz(brow);
  srsrc rs_a[PARTS], rs_b;
  uint32_t a_voff[AI], b_voff[BI];
#pragma unroll
  for (int part = 0; part < PARTS; ++part)
    rs_a[part] = operand_rows(A, part == 0 ? A.p : A.more[part - 1], C::AT ? 0 : m0, C::AT ? A.rows : C::BM);
  rs_b = operand_rows(B, B.p, C::BT ? 0 : n0, C::BT ? B.rows : C::BN);
  const uint32_t a_pitch = (uint32_t)A.pitch * 2u, b_pitch = (uint32_t)B.pitch * 2u;
#pragma unroll
  for (int i = 0; i < AI; ++i) {
    const int row = arow + C::A_STEP * i;
    const bool ok = C::AT ? m0 + acol * 8 < A.cols : m0 + row < A.rows;
    a_voff[i] = ok ? (uint32_t)row * a_pitch + (uint32_t)(C::AT ? m0 * 2 : 0) + (uint32_t)acol * 16u : OUTSIDE;
  }
#pragma unroll
  for (int i = 0; i < BI; ++i) {
    const int row = brow + C::B_STEP * i;
    const bool ok = C::BT ? n0 + bcol * 8 < B.cols : n0 + row < B.rows;
    b_voff[i] = ok ? (uint32_t)row * b_pitch + (uint32_t)(C::BT ? n0 * 2 : 0) + (uint32_t)bcol * 16u : OUTSIDE;
  }
  const uint32_t lds0 = (uint32_t)(size_t)lds, lds_w = lds0 + wave * 1024;
  constexpr int LA = AI * PARTS, L = LA + BI, MF = MB * NB * PARTS;
  int k_next = k_lo;                                  // first value of k of the next chunk to be loaded
  const int ka_hi = C::AT ? (int)(A.rows < k_hi ? A.rows : k_hi) : k_hi, kb_hi = C::BT ? (int)(B.rows < k_hi ? B.rows : k_hi) : k_hi;
  // load u of a chunk, which goes to the stage at `at`
  auto load = [&](int u, uint32_t at) {
    if (u < LA) {
      const int part = u / AI, i = u - part * AI;
      const bool ok = C::AT ? k_next + arow + C::A_STEP * i < ka_hi : k_next + acol * 8 < ka_hi;
      load_lds16(rs_a[part], ok ? a_voff[i] : OUTSIDE, C::AT ? (uint32_t)k_next * a_pitch : (uint32_t)k_next * 2u,
                 at + part * C::A_PART + i * (C::THREADS * 16));
    } else {
      const int i = u - LA;
      const bool ok = C::BT ? k_next + brow + C::B_STEP * i < kb_hi : k_next + bcol * 8 < kb_hi;
      load_lds16(rs_b, ok ? b_voff[i] : OUTSIDE, C::BT ? (uint32_t)k_next * b_pitch : (uint32_t)k_next * 2u, at + C::A_BYTES + i * (C::THREADS * 16));
    }
    if (u == L - 1) k_next += BK;
  };
  // ---- fragments: row (of m or n) lane % 32, values of k 8 * (lane / 32) .. + 7 of a step of 16
  typedef short v4s __attribute__((ext_vector_type(4)));
  typedef unsigned v2u __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) v4s* tr_ptr;
  auto* const lds3 = (__attribute__((address_space(3))) char*)lds;
  const int t16 = lane & 15, frow = 8 * (lane >> 5) + (t16 >> 2), fcol = 32 * ((lane >> 4) & 1) + 8 * (t16 & 3);
  auto read_tr = [&](uint32_t at, int pitch4) {
    const v2u lo = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(lds3 + at)));
    const v2u hi = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(lds3 + at + pitch4)));
    return v4u{lo.x, lo.y, hi.x, hi.y};
  };
  uint32_t a_at[C::AT ? MB : 1], b_at[C::BT ? NB : 1];
  const int ra = wm0 + (lane & 31), rb = wn0 + (lane & 31), xa = swz(ra), xb = swz(rb);
  if constexpr (C::AT) {
#pragma unroll
    for (int i = 0; i < MB; ++i) a_at[i] = frow * C::A_PITCH + (((wm0 / 32 + i) ^ row_xor<C::A_PITCH>(frow)) << 6) + fcol;
  }
  if constexpr (C::BT) {
#pragma unroll
    for (int j = 0; j < NB; ++j) b_at[j] = C::A_BYTES + frow * C::B_PITCH + (((wn0 / 32 + j) ^ row_xor<C::B_PITCH>(frow)) << 6) + fcol;
  }
  constexpr int NG = BK / 16;
  struct Frags { v4u a[PARTS][MB], b[NB]; } F[2];
  typedef __attribute__((address_space(3))) const v4u* frag_ptr;
  auto rd = [&](Frags& f, uint32_t st, int g) {
    const int c16 = g * 2 + (lane >> 5);
#pragma unroll
    for (int part = 0; part < PARTS; ++part)
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        if constexpr (C::AT) f.a[part][i] = read_tr(a_at[i] + st + part * C::A_PART + g * 16 * C::A_PITCH, 4 * C::A_PITCH);
        else f.a[part][i] = *(frag_ptr)(lds3 + st + part * C::A_PART + (ra + 32 * i) * C::A_PITCH + ((c16 ^ xa) << 4));
      }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      if constexpr (C::BT) f.b[j] = read_tr(b_at[j] + st + g * 16 * C::B_PITCH, 4 * C::B_PITCH);
      else f.b[j] = *(frag_ptr)(lds3 + st + C::A_BYTES + (rb + 32 * j) * C::B_PITCH + ((c16 ^ xb) << 4));
    }
  };
  auto mm1 = [&](const Frags& f, int u) {
    const int part = u / (MB * NB), w = u - part * (MB * NB);
    if constexpr (C::SWAP) acc[w / NB][w % NB] = mfma_bf16(f.b[w % NB], f.a[part][w / NB], acc[w / NB][w % NB]);
    else acc[w / NB][w % NB] = mfma_bf16(f.a[part][w / NB], f.b[w % NB], acc[w / NB][w % NB]);
  };
  auto chunk = [&](int stage, int to, bool first, bool more) {
    const uint32_t st = stage * C::STAGE, at = lds_w + to * C::STAGE;
    __builtin_amdgcn_sched_barrier(0);
    rd(F[0], st, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (first) {
      if (more) {
#pragma unroll
        for (int l = 0; l < L; ++l) load(l, at);
      }
    } else if (more) {
#pragma unroll
      for (int u = 0; u < MF; ++u) {
        mm1(F[1], u);
#pragma unroll
        for (int l = u * L / MF; l < (u + 1) * L / MF; ++l) load(l, at);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int u = 0; u < MF; ++u) mm1(F[1], u);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g + 1 < NG; ++g) {
      rd(F[(g + 1) & 1], st, g + 1);
#pragma unroll
      for (int u = 0; u < MF; ++u) mm1(F[g & 1], u);
      constexpr int RD = PARTS * MB * (C::AT ? 2 : 1) + NB * (C::BT ? 2 : 1);
#pragma unroll
      for (int u = 0; u < MF; ++u) {
        __builtin_amdgcn_sched_group_barrier(0x100, (RD + MF - 1) / MF, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    static_assert(NG % 2 == 0, "the held-back step is F[1]");
  };
  const int chunks = k_hi > k_lo ? (k_hi - k_lo + BK - 1) / BK : 0;
  // what opens chunk j: this wave's loads of it have landed, then a barrier: everybody's have, and everybody is done with the chunk
  // whose stage the next loads overwrite
  auto open = [&](int j) {
    __builtin_amdgcn_sched_barrier(0);
    const int later = chunks - 1 - j;                 // chunks behind this one that have been issued, NS - 2 at most
    if (NS > 3 && later >= 2) wait_loads<(NS > 3 ? 2 * L : 0)>();
    else if (NS > 2 && later >= 1) wait_loads<(NS > 2 ? L : 0)>();
    else wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  if (chunks == 0) return;
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < chunks) {
#pragma unroll
      for (int l = 0; l < L; ++l) load(l, lds_w + s * C::STAGE);
    }
  open(0);
  chunk(0, NS - 1, true, NS - 1 < chunks);
  int stage = 1, to = 0, j = 1;
  for (; j + NS - 1 < chunks; ++j) {
    open(j);
    chunk(stage, to, false, true);
    stage = stage + 1 == NS ? 0 : stage + 1;
    to = to + 1 == NS ? 0 : to + 1;
  }
  for (; j < chunks; ++j) {
    open(j);
    chunk(stage, to, false, false);
    stage = stage + 1 == NS ? 0 : stage + 1;
  }
#pragma unroll
  for (int u = 0; u < MF; ++u) mm1(F[1], u);
  __builtin_amdgcn_s_waitcnt(0xc07f);                 // this wave's LDS reads are done
  __builtin_amdgcn_s_barrier();                       // everybody's: the caller may use LDS
  asm volatile("" ::: "memory");
#endif
}

}  // namespace acc
