// The product of two row-major operands over their rows' common length,
//   D[p][q] = sum_k P[p][k] * Q[q][k],
// for binary16 rows (float32 sums) and 8-bit integer rows (32-bit sums), as the
// inner part of a workgroup's tile.  Both element types take the same bytes the
// same way: a lane's fragment is 16 bytes of one row (8 halves or 16 integers),
// a slice of the reduction is 128 bytes of every row.
//
// A workgroup owns BP x BQ outputs, WP x WQ waves TP x TQ tiles of 32 x 32 each, over
// the whole reduction or one of several parts of it.  The slices go through S stages
// of LDS, loaded past the registers (8 rows of one slice, 1 KB, an instruction and
// wave) S - 1 slices ahead and a few between the products of every sub-step, one
// barrier a slice.  Rows of LDS
// are whole 128-byte lines; the 16-byte chunk c of row r lies at c ^ ((r/2) % 8),
// so that the 16 rows a fragment read touches at a time lie in different banks.
//
// What bounds it: each sub-step reads (TP + TQ) KB of LDS a wave for TP * TQ
// products of 32 cycles, of 128 bytes a cycle that the LDS gives: 96 with eight waves
// of 2 x 4 tiles (Nt256), 85 with four of 3 x 3 (Nt192), all of them with 2 x 2, and
// the 64 x 64 tiles' loads take what the L2 gives (17 to 20 TB/s over all CUs).
// 8-bit, m x n x k = 8192 x 4096 x 4096: 126 us with its epilogue, 2180 TOP/s; 4096
// each: 65.6 us (a library product of 4096: 67.0).  Binary16: about 1500 TFLOP/s in
// the loop of the 4096 x 4096 x 4096 product, 900 with a float32 epilogue.
#pragma once

#include "common.hpp"

namespace fp16k {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));

struct NtHalf {  // binary16 elements, float32 sums
  typedef half8 Frag;
  typedef floatx16 Acc;
  static __device__ __forceinline__ Acc mma(const Frag& p, const Frag& q, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(p, q, c, 0, 0, 0);
  }
};

struct NtByte {  // 8-bit integers, 32-bit sums (exact below 2^31)
  typedef intx4 Frag;
  typedef intx16 Acc;
  static __device__ __forceinline__ Acc mma(const Frag& p, const Frag& q, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(p, q, c, 0, 0, 0);
  }
};

// H = 2: operands in a high and a low part each (see nt_product).
template <int WP_, int WQ_, int TP_, int TQ_, int SB_, int S_, int OCC_, int H_ = 1>
struct NtCfg {
  static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, SB = SB_, S = S_, OCC = OCC_, H = H_;
  static constexpr int WAVES = WP * WQ, THREADS = 64 * WAVES;
  static constexpr int BP = 32 * TP * WP, BQ = 32 * TQ * WQ;
  static constexpr int PART = (BP + BQ) * SB, STAGE = H * PART, LDS = S * STAGE;
  static constexpr int IP = BP * SB / (1024 * WAVES), IQ = BQ * SB / (1024 * WAVES);  // loads
  static_assert(SB == 64 || (SB == 128 && IP % 2 == 0 && IQ % 2 == 0), "the chunks' order");
  static_assert(IP * 1024 * WAVES == BP * SB && IQ * 1024 * WAVES == BQ * SB, "whole loads");
  static_assert(LDS * OCC <= 160 * 1024, "LDS");
};

// One 16-byte-per-lane load from a buffer resource into LDS (1 KB a wave).
__device__ __forceinline__ void nt_load(__amdgpu_buffer_rsrc_t rs, char* lds_dst, uint32_t voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds_dst, 16,
                                           voff, 0, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t nt_rsrc(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, 0x00020000);
}
// workgroup barrier without the implied memory fence; callers wait first
__device__ __forceinline__ void nt_barrier() { __asm__ volatile("s_barrier" ::: "memory"); }

// The rows of one tile, each operand from the tile's first row (with H = 2 its high
// and its low part).
struct NtTile {
  const void* p[2];
  const void* q[2];
  uint32_t ldp, ldq;   // bytes from row to row, multiples of 16
  int prows, qrows;    // rows there are from the tile's first; others read as zeros
  int kbytes;          // of a row; a last chunk's bytes past it are multiplied too
  int part, parts;     // which of so many ranges of the slices
};

// acc = the sums of P[p][k] Q[q][k]; with H = 2 of Ph Ql + Pl Qh + Ph Qh, every part
// loaded once for the three products.
template <class T, class C>
__device__ __forceinline__ void nt_product(const NtTile& t, char* lds,
                                           typename T::Acc (&acc)[C::TP][C::TQ]) {
  typedef typename T::Frag Frag;
  constexpr int TP = C::TP, TQ = C::TQ, S = C::S, SB = C::SB, H = C::H, IP = C::IP, IQ = C::IQ;
  constexpr int I1 = IP + IQ, I = H * I1;
  constexpr uint32_t OOB = 0x80000000u;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave / C::WQ, wq = wave % C::WQ;
  const int lrow = lane & 31, lhi = lane >> 5;

  // loads: an instruction fills 8 lines of 128 bytes, lane l the 16 bytes l % 8 of
  // line l / 8: rows RI (wave * I. + i) .. + RI - 1 (see the layout above)
  constexpr int RI = 1024 / SB;
  const int prec = (t.prows < C::BP ? t.prows : C::BP) * (int)t.ldp;
  const int qrec = (t.qrows < C::BQ ? t.qrows : C::BQ) * (int)t.ldq;
  int ck[2];           // byte of the chunk in its row's slice, even and odd instructions
  uint32_t pv[2], qv[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int row;
    if (SB == 128) {
      row = lane >> 3;
      ck[h] = ((lane & 7) ^ ((h * 4 + (lane >> 4)) & 7)) * 16;
    } else {
      const int c = (lane & 7) ^ ((lane >> 4) & 3);
      row = (lane >> 3) * 2 + (c >> 2);
      ck[h] = (c & 3) * 16;
    }
    pv[h] = (uint32_t)(wave * IP * RI + row) * t.ldp + (uint32_t)ck[h];
    qv[h] = (uint32_t)(wave * IQ * RI + row) * t.ldq + (uint32_t)ck[h];
  }
  // this part's range of the slices: its length, and the one loaded next
  const int slices = (t.kbytes + SB - 1) / SB, KT = (slices + t.parts - 1) / t.parts;
  int k0 = t.part * KT * SB;
  const int kend = t.kbytes < k0 + KT * SB ? t.kbytes : k0 + KT * SB;
  bool in[2];
  auto begin = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) in[h] = k0 + ck[h] < kend;
  };
  auto load = [&](char* buf, int n) {
    const int h = n / I1, i = n % I1;
    buf += h * C::PART;
    if (i < IP) {
      const uint32_t off = pv[i & 1] + ((uint32_t)(i * RI) * t.ldp + (uint32_t)k0);
      nt_load(nt_rsrc(t.p[h], prec), buf + (wave * IP + i) * 1024, in[i & 1] ? off : OOB);
    } else {
      const int j = i - IP;
      const uint32_t off = qv[j & 1] + ((uint32_t)(j * RI) * t.ldq + (uint32_t)k0);
      nt_load(nt_rsrc(t.q[h], qrec), buf + C::BP * SB + (wave * IQ + j) * 1024,
              in[j & 1] ? off : OOB);
    }
  };
  auto advance = [&]() { k0 += SB; };

#pragma unroll
  for (int a = 0; a < TP; ++a)
#pragma unroll
    for (int b = 0; b < TQ; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[a][b][e] = 0;

  Frag fp[2][H][TP], fq[2][H][TQ];
  // byte of this lane's fragment of sub-step ks in a block of 32 rows
  auto place = [&](int ks) {
    if (SB == 128) return lrow * 128 + ((ks * 2 + lhi) ^ ((lrow >> 1) & 7)) * 16;
    return (lrow >> 1) * 128 + (((lrow & 1) * 4 + ks * 2 + lhi) ^ ((lrow >> 2) & 3)) * 16;
  };
  // read r of the fragments of sub-step ks, in the order they are used in
  auto fetch = [&](const char* buf, int ks, int r, Frag (&p)[H][TP], Frag (&q)[H][TQ]) {
    const bool isq = r < TQ || r >= TQ + H * TP;
    const int h = H == 1 ? 0 : r < TQ ? 1 : r < TQ + TP ? 0 : r < TQ + 2 * TP ? 1 : 0;
    const int i = r < TQ ? r : r < TQ + TP ? r - TQ : r < TQ + 2 * TP ? r - TQ - TP : r - TQ - 2 * TP;
    const Frag* from = reinterpret_cast<const Frag*>(
        buf + h * C::PART + (isq ? C::BP * SB + (wq * TQ + i) * 32 * SB : (wp * TP + i) * 32 * SB) +
        place(ks));
    if (isq)
      q[h][i < TQ ? i : 0] = *from;
    else
      p[h][i < TP ? i : 0] = *from;
  };
  constexpr int R = H * (TP + TQ), M = (H == 2 ? 3 : 1) * TP * TQ;  // reads, products
  // One sub-step: the products of one set of fragments, between them the reads of
  // the next set (sub-step ks of `from`) and loads L0 .. L1 - 1 into `to`, an
  // instruction or two after each product (kept there by the scheduling barriers;
  // left to itself the compiler issues them in bursts that hold the products up).
  auto substep = [&](const Frag (&p)[H][TP], const Frag (&q)[H][TQ], const char* from, int ks,
                     Frag (&np)[H][TP], Frag (&nq)[H][TQ], char* to, auto l0, auto l1) {
    constexpr int L0 = decltype(l0)::value, V = decltype(l1)::value - L0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int a = i / TQ % TP, b = i % TQ, term = i / (TP * TQ);
      acc[a][b] = T::mma(p[H == 2 && term == 1][a], q[H == 2 && term == 0][b], acc[a][b]);
#pragma unroll
      for (int r = R * i / M; r < R * (i + 1) / M; ++r) fetch(from, ks, r, np, nq);
#pragma unroll
      for (int v = V * i / M; v < V * (i + 1) / M; ++v) load(to, L0 + v);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

#pragma unroll
  for (int s = 0; s < S - 1; ++s) {
    begin();
#pragma unroll
    for (int i = 0; i < I; ++i) load(lds + s * C::STAGE, i);
    advance();
  }
  // the stage used next has landed once at most the S - 2 later ones are out
  constexpr int OUT = I * (S - 2);
  static_assert(OUT < 64, "the wait's counter");
  constexpr int WAIT = (0x0 << 8) | (0x7 << 4) | (OUT & 0xF) | ((OUT >> 4) << 14);
  __builtin_amdgcn_s_waitcnt(WAIT);
  nt_barrier();
#pragma unroll
  for (int r = 0; r < R; ++r) fetch(lds, 0, r, fp[0], fq[0]);
  int rd = 0, wr = S - 1;
  for (int kt = 0; kt < KT; ++kt) {
    const char* cur = lds + rd * C::STAGE;
    char* nxt = lds + wr * C::STAGE;
    constexpr std::integral_constant<int, 0> L0{};
    constexpr std::integral_constant<int, SB == 64 ? I : (I + 1) / 2> L1{};
    constexpr std::integral_constant<int, I> L2{};
    begin();
    substep(fp[0], fq[0], cur, 1, fp[1], fq[1], nxt, L0, L1);
    if constexpr (SB == 128) {
      substep(fp[1], fq[1], cur, 2, fp[0], fq[0], nxt, L1, L2);
      substep(fp[0], fq[0], cur, 3, fp[1], fq[1], nxt, L2, L2);
    }
    advance();
    // this wave's reads of the stage are complete and its part of the next one
    // has landed: publish it, and free this stage
    __builtin_amdgcn_s_waitcnt(WAIT);
    nt_barrier();
    rd = rd + 1 == S ? 0 : rd + 1;
    wr = wr + 1 == S ? 0 : wr + 1;
    substep(fp[1], fq[1], lds + rd * C::STAGE, 0, fp[0], fq[0], nxt, L2, L2);
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();  // every load has landed and every read is done: LDS is free
}

// Workgroup b of a grid of 8 * ceil(n / 8): the workgroups that one XCD takes
// (every eighth) get neighbouring tiles, which share rows in its L2.
__device__ __forceinline__ int nt_xcd(int b, int n) { return (b & 7) * ((n + 7) >> 3) + (b >> 3); }

// LDS written by this wave's lanes visible to all of them (LDS operations of one
// wave complete in order; this keeps the compiler from moving them)
__device__ __forceinline__ void nt_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wave's outputs to memory, 32 columns q of its 32 TP rows p at a time.  The
// products leave rows p = 8 (e/4) + 4 (l/32) + e%4 of column q = l%32 in lane l, so
// that memory would see runs of 32 bytes; through LDS each lane gets 8 consecutive
// p of one q and 4 TP lanes a whole run of 32 TP:
//   epi.load(p, q)                what compute needs of memory, read a group of
//                                 passes ahead; any p, q (reads within bounds)
//   epi.compute(p, q, v, pre, out) out[OUTS] from the sums v[8]; any p, q
//   epi.store(p, q, out)          what goes out[q][p ..], if p and q are within
//   epi.diagonal(q, v)            (DIAGONAL) the sum of p = q
// With `mirror`, out[0 .. PARTS - 1] are also stored transposed, mir[s][p * ldm + q]
// (their 16-byte chunks in LDS exclusive-ored with the row, since the writes step 8
// rows a lane), where p < plim and q < qlim.
// A workgroup runs this once, at one wave a SIMD for the large tiles: the passes of
// a group are done side by side without branches, so that they hide each other's
// latency (one at a time with a test each: 4 us a pass of a 256 x 256 tile; twice as
// many side by side no longer fit the registers of two workgroups a CU: the 8-bit
// product of 4096 each 65 -> 81 us).
template <class C, int PARTS>
struct NtEpi {
  static constexpr int TP = C::TP, TQ = C::TQ, U = TP;
  static constexpr int FLD = 32 * TP + 4, MLD = 40;  // floats, halves
  static constexpr int WAVE = 32 * FLD * 4 + PARTS * 32 * TP * MLD * 2;
  static constexpr int LDS = WAVE * C::WAVES > C::LDS ? WAVE * C::WAVES : C::LDS;
  static_assert(LDS * C::OCC <= 160 * 1024, "LDS");
};

template <class C, int PARTS, class Acc, class Epi>
__device__ __forceinline__ void nt_store(const Acc (&acc)[C::TP][C::TQ], char* lds, int p0, int q0,
                                         int plim, int qlim, bool mirror, h16* const (&mir)[PARTS],
                                         int ldm, const Epi& epi) {
  typedef NtEpi<C, PARTS> E;
  constexpr int TP = E::TP, TQ = E::TQ, U = E::U, FLD = E::FLD, MLD = E::MLD;
  constexpr int CPR = 4 * TP;  // chunks of a run; 2 TP passes a block, U at a time
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lrow = lane & 31, lhi = lane >> 5;
  typedef decltype(acc[0][0][0] + 0) V;
  typedef V V4 __attribute__((ext_vector_type(4)));
  V* const f = reinterpret_cast<V*>(lds + wave * E::WAVE);
  h16* const m = reinterpret_cast<h16*>(f + 32 * FLD);
  typename Epi::Pre pre[U];
  // passes n U .. n U + U - 1 of the wave's 2 TP TQ: columns and chunks' first rows
  auto load = [&](int n) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = (n % 2) * U + u;
      pre[u] = epi.load(p0 + 8 * ((i * 64 + lane) % CPR), q0 + 32 * (n / 2) + (i * 64 + lane) / CPR);
    }
  };
  load(0);
#pragma unroll 1
  for (int b = 0; b < TQ; ++b) {
#pragma unroll
    for (int s = 0; s < TQ; ++s) {
      if (s != b) continue;
#pragma unroll
      for (int a = 0; a < TP; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const V4 v = {acc[a][s][4 * e], acc[a][s][4 * e + 1], acc[a][s][4 * e + 2],
                        acc[a][s][4 * e + 3]};
          *reinterpret_cast<V4*>(f + lrow * FLD + 32 * a + 8 * e + 4 * lhi) = v;
        }
    }
    nt_wave_sync();
    const int qb = q0 + 32 * b;
    if constexpr (Epi::DIAGONAL) {
      if (qb >= p0 && qb < p0 + 32 * TP) {
        if (lane < 32) epi.diagonal(qb + lane, f[lane * FLD + qb - p0 + lane]);
      }
    }
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      typename Epi::Pre now[U];
      V v[U][8];
      V8 out[U][Epi::OUTS];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = ((h * U + u) * 64 + lane) / CPR, c = ((h * U + u) * 64 + lane) % CPR;
        const V4* from = reinterpret_cast<const V4*>(f + r * FLD + 8 * c);
        const V4 x = from[0], y = from[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[u][k] = x[k];
          v[u][4 + k] = y[k];
        }
        now[u] = pre[u];
      }
      if (2 * b + h + 1 < 2 * TQ) load(2 * b + h + 1);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = ((h * U + u) * 64 + lane) / CPR, c = ((h * U + u) * 64 + lane) % CPR;
        epi.compute(p0 + 8 * c, qb + r, v[u], now[u], out[u]);
        if (mirror) {
#pragma unroll
          for (int s = 0; s < PARTS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              m[s * 32 * TP * MLD + (8 * c + e) * MLD + ((r / 8) ^ ((c >> 1) & 3)) * 8 + r % 8] =
                  out[u][s].h[e];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = ((h * U + u) * 64 + lane) / CPR, c = ((h * U + u) * 64 + lane) % CPR;
        epi.store(p0 + 8 * c, qb + r, out[u]);
      }
    }
    nt_wave_sync();
    if (mirror) {
#pragma unroll
      for (int s = 0; s < PARTS; ++s) {
        V8 w[2 * TP];
#pragma unroll
        for (int i = 0; i < 2 * TP; ++i) {
          const int r = (i * 64 + lane) / 4, c = (i * 64 + lane) % 4;
          w[i] = load16(m + s * 32 * TP * MLD + r * MLD + 8 * (c ^ ((r >> 4) & 3)));
        }
#pragma unroll
        for (int i = 0; i < 2 * TP; ++i) {
          const int r = (i * 64 + lane) / 4, q = qb + 8 * ((i * 64 + lane) % 4);
          if (p0 + r < plim && q < qlim) store16(mir[s] + (int64_t)(p0 + r) * ldm + q, w[i]);
        }
      }
      nt_wave_sync();
    }
  }
}

// The sums of a workgroup as they lie in registers, to memory and back, for a
// reduction split over workgroups: 1 KB a wave and instruction.
template <class C, class Acc>
__device__ __forceinline__ void nt_put(const Acc (&acc)[C::TP][C::TQ], floatx4* to) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int a = 0; a < C::TP; ++a)
#pragma unroll
    for (int b = 0; b < C::TQ; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const floatx4 v = {acc[a][b][4 * e], acc[a][b][4 * e + 1], acc[a][b][4 * e + 2],
                           acc[a][b][4 * e + 3]};
        to[(((wave * C::TP + a) * C::TQ + b) * 4 + e) * 64 + lane] = v;
      }
}
// One 32 x 32 tile (wave, a, b) of the sums that `parts` workgroups put there.
template <class C>
__device__ __forceinline__ floatx16 nt_get(const floatx4* from, int parts, int wave, int a, int b) {
  const int lane = threadIdx.x & 63;
  floatx16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
#pragma unroll 4
  for (int s = 0; s < parts; ++s) {
    const floatx4* f = from + (size_t)s * (C::BP * C::BQ / 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const floatx4 v = f[(((wave * C::TP + a) * C::TQ + b) * 4 + e) * 64 + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[4 * e + i] += v[i];
    }
  }
  return acc;
}

//            waves  tile  slice  stages  workgroups a CU
typedef NtCfg<4, 2, 2, 4, 128, 2, 1> Nt256;   // 256 x 256
typedef NtCfg<2, 2, 3, 3, 128, 3, 1> Nt192;   // 192 x 192
typedef NtCfg<2, 2, 2, 2, 128, 2, 2> Nt128;   // 128 x 128, two workgroups
typedef NtCfg<2, 2, 2, 2, 128, 4, 1> Nt128d;  // 128 x 128, one, loads further ahead
typedef NtCfg<2, 2, 1, 1, 128, 5, 2> Nt64;    // 64 x 64

}  // namespace fp16k
