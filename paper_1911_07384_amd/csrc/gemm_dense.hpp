// The product of two binary16 operands with float32 sums,
//   D[q][p] = sum_k P(p, k) Q(q, k),
// as the inner part of a workgroup's tile of the dense layers.  An operand's rows run
// along k in memory, or (PS, QS) its columns do: P[k][p].
//
// Matrix instructions are the 16 x 16 x 32 ones: the card is bound by its power, and on
// random operands in registers they sustain 1930 TFLOP/s, 32 x 32 x 16 ones 1650.
//
// A workgroup owns BP x BQ outputs, WP x WQ waves TP x TQ tiles of 16 x 16 each, and G such
// groups of waves a range of the reduction each, with LDS of their own.  Slices
// of 64 of the reduction go through S stages of LDS, loaded past the registers (1 KB an
// instruction and wave) S slices ahead, in the sub-step (32 of the reduction) behind the
// barrier that frees their stage.  A sub-step's fragments are read from LDS between the
// products of the one before.
//
// Which rows a tile holds is free, and chosen so that the sums need no exchange between
// lanes before they are stored: tile t of a wave's 8 takes rows 8 c + t, and its rows
// are in such an order that a lane's sums are 8 consecutive p of chunks 4 i + l / 16,
// i = 0 .. 3: four lanes store 64 bytes of one q.
//
// LDS, an operand along k: a line of 128 bytes a row, in the order of the tiles, its
// 16-byte chunk c at c ^ ((line / 2) % 8): the 16 lines a read touches at a time lie in
// different banks.  An operand along its rows: a line of the tile's rows for each k.  A
// lane reads T consecutive rows at its eight k and permutes bytes into the fragments of
// T tiles, 4 permutes each (gfx950's transposing read would need none, but through the
// compiler's builtin each waits for all loads in flight).
#pragma once

#include "common.hpp"

#include <type_traits>
#include <utility>

namespace fp16k {

template <int WP_, int WQ_, int TP_, int TQ_, int S_, int OCC_, bool PS_ = false, bool QS_ = false,
          int G_ = 1>
struct DenseCfg {
  static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, S = S_, OCC = OCC_, G = G_;
  static constexpr bool PS = PS_, QS = QS_;
  static constexpr int WAVES = WP * WQ, THREADS = 64 * WAVES * G;
  static constexpr int BP = 16 * TP * WP, BQ = 16 * TQ * WQ;
  static constexpr int STAGE = (BP + BQ) * 128, LDS = S * STAGE;  // of a group
  static constexpr int IP = BP / (8 * WAVES), IQ = BQ / (8 * WAVES);  // loads of a wave
  static_assert(TP == 8, "a lane's chunks of 8 rows");
  static_assert(IP % 2 == 0 && IQ % 2 == 0, "the chunks' order");
  static_assert(IP * 8 * WAVES == BP && IQ * 8 * WAVES == BQ, "whole loads");
  static_assert(G * LDS * OCC <= 160 * 1024, "LDS");
  static_assert((G - 1) * BP * BQ * 4 <= G * LDS, "the groups' sums");
  static_assert(!QS || ((TQ == 2 || TQ == 4 || TQ == 8) && 512 % BQ == 0), "lines of whole loads");
  static_assert(!PS || 512 % BP == 0, "lines of whole loads");
  // Threads for __launch_bounds__: two waves a SIMD, also where there is one, keep the
  // compiler to 256 registers, with the sums among them (with accumulator registers it
  // copied them to and fro within the loop, 96 moves for 64 products).
  static constexpr int BOUND = THREADS > 512 / OCC ? THREADS : 512 / OCC;
};

// One 16-byte-per-lane load from a buffer resource into LDS (1 KB a wave).
__device__ __forceinline__ void dense_load(__amdgpu_buffer_rsrc_t rs, char* lds_dst, uint32_t voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds_dst, 16,
                                           voff, 0, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t dense_rsrc(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, 0x00020000);
}

// f(0), f(1), .. with compile-time indexes (the compiler unrolls no loop of this size).
template <class F, int... N>
__device__ __forceinline__ void dense_each(F&& f, std::integer_sequence<int, N...>) {
  (f(std::integral_constant<int, N>{}), ...);
}

// The rows of one tile, each operand from the tile's first row (and k = 0).
struct DenseTile {
  const h16 *p, *q;
  uint32_t ldp, ldq;  // bytes from row to row (from k to k along rows), multiples of 16
  int prows, qrows;   // rows there are from the tile's first; others read as zeros
  int nk;             // a multiple of 8 for an operand along k
  int part, parts;    // which of so many ranges of the slices
};

// The chunk of 8 rows that row m of a wave's tiles of P belongs to.
__device__ __forceinline__ int dense_chunk(int m) { return 4 * (m & 3) + (m >> 2); }

// T rows at a lane's eight k as they were read.
template <int T>
struct DenseRaw {
  uint32_t d[8][T / 2];
};
template <int T>
__device__ __forceinline__ half8 dense_rows(const DenseRaw<T>& r, int t) {
  const uint32_t sel = t & 1 ? 0x07060302u : 0x05040100u;
  V8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v.d[i] = __builtin_amdgcn_perm(r.d[2 * i + 1][t >> 1], r.d[2 * i][t >> 1], sel);
  return v.h;
}

// One group's sums; lds: its own.  Every group passes the same number of barriers.
template <class C>
__device__ __forceinline__ void dense_loop(const DenseTile& t, char* lds, int wave,
                                           floatx4 (&acc)[C::TP][C::TQ]) {
  constexpr int TP = C::TP, TQ = C::TQ, S = C::S, IP = C::IP, IQ = C::IQ, I = IP + IQ;
  constexpr uint32_t OOB = 0x80000000u;
  const int lane = threadIdx.x & 63;
  const int wp = wave / C::WQ, wq = wave % C::WQ;
  const int m = lane & 15, g = lane >> 4;

  // this part's range of the reduction
  const int slices = (t.nk + 63) / 64, KT = (slices + t.parts - 1) / t.parts;
  int k0 = t.part * KT * 64;
  const int kend = t.nk < k0 + KT * 64 ? t.nk : k0 + KT * 64;

  // loads of an operand along k: an instruction fills 8 lines, lane l the 16 bytes l % 8
  // of line l / 8; of line 16 t + m of a wave's block the row is 8 chunk(m) + t (P) or
  // the line itself (Q)
  const int prec = (t.prows < C::BP ? t.prows : C::BP) * (int)t.ldp;
  const int qrec = (t.qrows < C::BQ ? t.qrows : C::BQ) * (int)t.ldq;
  int ck[2];  // element of the chunk in its row's slice, even and odd instructions
  uint32_t pv[2], qv[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    ck[h] = ((lane & 7) ^ ((h * 4 + (lane >> 4)) & 7)) * 8;
    pv[h] = (uint32_t)(8 * dense_chunk(h * 8 + (lane >> 3))) * t.ldp + (uint32_t)ck[h] * 2u;
    qv[h] = (uint32_t)(wave * IQ * 8 + (lane >> 3)) * t.ldq + (uint32_t)ck[h] * 2u;
  }
  // .. along its rows: an instruction fills the lines of PK (QK) k
  constexpr int PK = 512 / C::BP, QK = 512 / C::BQ;
  const char* ps = reinterpret_cast<const char*>(t.p);
  const char* qs = reinterpret_cast<const char*>(t.q);
  if (C::PS) ps += (uint64_t)k0 * t.ldp;
  if (C::QS) qs += (uint64_t)k0 * t.ldq;
  // bytes of a slice of it, up to its last k's last chunk
  auto slice_bytes = [&](uint32_t ld, int rows) {
    const int n = kend - k0;
    return n <= 0 ? 0 : ((n < 64 ? n : 64) - 1) * (int)ld + ((rows + 7) & ~7) * 2;
  };
  bool in[2];
  auto begin = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) in[h] = k0 + ck[h] < kend;
  };
  auto load = [&](char* buf, int i) {
    if (i < IP) {
      const int n = wave * IP + i;
      if constexpr (C::PS) {
        dense_load(dense_rsrc(ps, slice_bytes(t.ldp, t.prows)), buf + n * 1024,
                   (uint32_t)(n * PK + lane / (64 / PK)) * t.ldp + (lane % (64 / PK)) * 16u);
      } else {
        const uint32_t row = (uint32_t)(n / 16 * 128 + n / 2 % 8);
        dense_load(dense_rsrc(t.p, prec), buf + n * 1024,
                   in[i & 1] ? pv[i & 1] + (row * t.ldp + (uint32_t)k0 * 2u) : OOB);
      }
    } else {
      const int j = i - IP, n = wave * IQ + j;
      char* const to = buf + C::BP * 128 + n * 1024;
      if constexpr (C::QS) {
        dense_load(dense_rsrc(qs, slice_bytes(t.ldq, t.qrows)), to,
                   (uint32_t)(n * QK + lane / (64 / QK)) * t.ldq + (lane % (64 / QK)) * 16u);
      } else {
        dense_load(dense_rsrc(t.q, qrec), to,
                   in[j & 1] ? qv[j & 1] + ((uint32_t)(j * 8) * t.ldq + (uint32_t)k0 * 2u) : OOB);
      }
    }
  };
  auto advance = [&]() {
    k0 += 64;
    if (C::PS) ps += 64ull * t.ldp;
    if (C::QS) qs += 64ull * t.ldq;
  };

#pragma unroll
  for (int a = 0; a < TP; ++a)
#pragma unroll
    for (int b = 0; b < TQ; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[a][b][e] = 0.0f;

  // an operand along its rows is held as it was read until its products
  half8 fp[2][TP], fq[2][TQ];
  DenseRaw<TP> rp[2];
  DenseRaw<C::QS ? TQ : 2> rq[2];
  const int line = m * 128, swz = (m >> 1) & 7;
  auto along = [&](const char* block, int tile, int ks) {
    return *reinterpret_cast<const half8*>(block + tile * 2048 + line + (((ks * 4 + g) ^ swz) * 16));
  };
  auto across = [&](const char* from, auto& raw, int j) {
    constexpr int W = sizeof(raw.d[0]);
    if constexpr (W == 16) {
      const V8 v = load16(from);
#pragma unroll
      for (int k = 0; k < 4; ++k) raw.d[j][k] = v.d[k];
    } else if constexpr (W == 8) {
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      const u32x2 v = *reinterpret_cast<const u32x2*>(from);
      raw.d[j][0] = v[0];
      raw.d[j][1] = v[1];
    } else {
      raw.d[j][0] = *reinterpret_cast<const uint32_t*>(from);
    }
  };
  // read r of the fragments of sub-step ks: all of Q, then P in the order of its use
  constexpr int RQ = C::QS ? 8 : TQ, RP = C::PS ? 8 : TP, R = RP + RQ, M = TP * TQ;
  auto fetch = [&](const char* buf, int ks, int r, int set) {
    if (r < RQ) {
      const char* const from = buf + C::BP * 128;
      if constexpr (C::QS)
        across(from + (ks * 32 + g * 8 + r) * C::BQ * 2 + (wq * 16 + m) * TQ * 2, rq[set], r);
      else
        fq[set][r < TQ ? r : 0] = along(from + wq * TQ * 2048, r, ks);
    } else {
      if constexpr (C::PS)
        across(buf + (ks * 32 + g * 8 + r - RQ) * C::BP * 2 + (wp * 16 + dense_chunk(m)) * 16,
               rp[set], r - RQ);
      else
        fp[set][r - RQ] = along(buf + wp * TP * 2048, r - RQ, ks);
    }
  };
  // One sub-step: the products of one set of fragments, between them the reads of the
  // other set (sub-step ks of `from`), done by three quarters of it, and a slice's loads
  // into `to`, spread evenly: a burst of them holds the wave's products up (in the first
  // quarter 834 us for 8192 x 8192 x 8192, spread 817, with half of them in the sub-step
  // after, where they have less time to land, 866).  The scheduling barriers keep them
  // there.
  auto substep = [&](auto which, const char* from, int ks, char* to, auto loads) {
    constexpr int set = decltype(which)::value;
    constexpr bool LOADS = decltype(loads)::value;
    dense_each(
        [&](auto n) __attribute__((always_inline)) {
          constexpr int i = decltype(n)::value, a = i / TQ, b = i % TQ;
          if constexpr (C::PS && b == 0) fp[set][a] = dense_rows(rp[set], a);
          if constexpr (C::QS && a == 0) fq[set][b] = dense_rows(rq[set], b);
          acc[a][b] =
              __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[set][a], fq[set][b], acc[a][b], 0, 0, 0);
          constexpr int F = M * 3 / 4;
          if constexpr (i < F) {
#pragma unroll
            for (int r = R * i / F; r < R * (i + 1) / F; ++r) fetch(from, ks, r, set ^ 1);
          }
          if constexpr (LOADS) {
#pragma unroll
            for (int v = I * i / M; v < I * (i + 1) / M; ++v) load(to, v);
          }
          if constexpr (i % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        },
        std::make_integer_sequence<int, M>{});
  };

#pragma unroll
  for (int s = 0; s < S; ++s) {
    begin();
#pragma unroll
    for (int i = 0; i < I; ++i) load(lds + s * C::STAGE, i);
    advance();
  }
  // the stage used next has landed once at most the S - 2 later ones are out
  static_assert(S >= 2 && I * (S - 1) < 64, "the wait's counter");
  auto wait = [](auto n) {  // (and for this wave's LDS reads)
    constexpr int N = decltype(n)::value;
    __builtin_amdgcn_s_waitcnt((0x0 << 8) | (0x7 << 4) | (N & 0xF) | ((N >> 4) << 14));
  };
  // a barrier without the implied memory fence
  auto barrier = []() { __asm__ volatile("s_barrier" ::: "memory"); };
  wait(std::integral_constant<int, I * (S - 1)>{});
  barrier();
#pragma unroll
  for (int r = 0; r < R; ++r) fetch(lds, 0, r, 0);
  int rd = 0;
  for (int kt = 0; kt < KT; ++kt) {
    char* const freed = lds + rd * C::STAGE;
    substep(std::integral_constant<int, 0>{}, freed, 1, nullptr, std::false_type{});
    begin();
    // this wave's reads of the stage are complete and its part of the next one has
    // landed: publish it, and free this stage
    wait(std::integral_constant<int, I * (S - 2)>{});
    barrier();
    rd = rd + 1 == S ? 0 : rd + 1;
    substep(std::integral_constant<int, 1>{}, lds + rd * C::STAGE, 0, freed, std::true_type{});
    advance();
  }
  __builtin_amdgcn_s_waitcnt(0);  // (loads past the end are still to land in LDS)
}

// The groups' sums added in their order, in the first one's.
template <class C>
__device__ __forceinline__ void dense_groups(char* lds, int group, int wave,
                                             floatx4 (&acc)[C::TP][C::TQ]) {
  constexpr int N = C::TP * C::TQ * 64;
  floatx4* const sums = reinterpret_cast<floatx4*>(lds) + wave * N + (threadIdx.x & 63);
  __syncthreads();  // (the last reads of what is written over)
  if (group > 0) {
#pragma unroll
    for (int a = 0; a < C::TP; ++a)
#pragma unroll
      for (int b = 0; b < C::TQ; ++b)
        sums[(group - 1) * C::WAVES * N + (a * C::TQ + b) * 64] = acc[a][b];
  }
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int g = 0; g < C::G - 1; ++g)
#pragma unroll
    for (int a = 0; a < C::TP; ++a)
#pragma unroll
      for (int b = 0; b < C::TQ; ++b) acc[a][b] += sums[g * C::WAVES * N + (a * C::TQ + b) * 64];
}

// A wave's outputs to memory: its tile's first p and q, and for a lane 8 consecutive p
// of one q at a time, with the interface
//   epi.column(p)                  what compute needs for any q
//   epi.load(p, q)                 .. for this q, read a group of q ahead
//   epi.compute(p, q, v, col, pre, out) out[OUTS] from the sums v[8]; any p, q
//   epi.store(p, q, out)           out, if p and q are within
template <class C, class Epi>
__device__ __forceinline__ void dense_store(const floatx4 (&acc)[C::TP][C::TQ], int p0, int q0,
                                            const Epi& epi) {
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  typename Epi::Col col[4];
  typename Epi::Pre pre[4];
  auto row = [&](int b) { return q0 + (C::QS ? C::TQ * m + b : 16 * b + m); };
  auto load = [&](int b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) pre[i] = epi.load(p0 + 8 * (4 * i + g), row(b));
  };
  load(0);
#pragma unroll
  for (int i = 0; i < 4; ++i) col[i] = epi.column(p0 + 8 * (4 * i + g));
#pragma unroll 1
  for (int b = 0; b < C::TQ; ++b) {
    typename Epi::Pre now[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) now[i] = pre[i];
    if (b + 1 < C::TQ) load(b + 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[2][8];
#pragma unroll
      for (int s = 0; s < C::TQ; ++s) {
        if (s != b) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) v[i][k] = acc[k][s][2 * h + i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int p = p0 + 8 * (4 * (2 * h + i) + g);
        V8 out[Epi::OUTS];
        epi.compute(p, row(b), v[i], col[2 * h + i], now[2 * h + i], out);
        epi.store(p, row(b), out);
      }
      __builtin_amdgcn_sched_barrier(0);  // (two chunks' registers at a time)
    }
  }
}

// Workgroup b of a grid of 8 * ceil(n / 8): the workgroups that one XCD takes (every
// eighth) get neighbouring tiles, which share rows in its L2.
__device__ __forceinline__ int dense_xcd(int b, int n) {
  return (b & 7) * ((n + 7) >> 3) + (b >> 3);
}

}  // namespace fp16k
