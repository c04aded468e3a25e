// The product of two row-major operands over their rows' common length,
//   D[p][q] = sum_k P[p][k] * Q[q][k],
// for binary16 rows (float32 sums) and 8-bit integer rows (32-bit sums), as the
// inner part of a workgroup's tile.  Both element types take the same bytes the
// same way: a lane's fragment is 16 bytes of one row (8 halves or 16 integers),
// a slice of the reduction is 128 bytes of every row.
//
// A workgroup of WP x WQ waves owns BP x BQ outputs, each wave TP x TQ tiles of
// 32 x 32.  The slices go through S stages of LDS, loaded past the registers
// (8 rows of one slice, 1 KB, an instruction and wave) S - 1 slices ahead and a
// few between the products of every sub-step, one barrier a slice.  Rows of LDS
// are whole 128-byte lines; the 16-byte chunk c of row r lies at c ^ ((r/2) % 8),
// so that the 16 rows a fragment read touches at a time lie in different banks.
//
// What bounds it: each sub-step reads (TP + TQ) KB of LDS a wave for TP * TQ
// products of 32 cycles.  At TP = TQ = 4 with four waves that is 64 bytes a cycle
// (and 32 written) of the 128 that the LDS gives, at TP = TQ = 2 all of them.
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

template <int WP_, int WQ_, int TP_, int TQ_, int S_, int OCC_>
struct NtCfg {
  static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, S = S_, OCC = OCC_;
  static constexpr int WAVES = WP * WQ, THREADS = 64 * WAVES;
  static constexpr int BP = 32 * TP * WP, BQ = 32 * TQ * WQ;
  static constexpr int IP = BP / (8 * WAVES), IQ = BQ / (8 * WAVES);  // loads a wave and slice
  static constexpr int STAGE = (BP + BQ) * 128, LDS = S * STAGE;
  static_assert(IP % 2 == 0 && IQ % 2 == 0, "the chunk order goes by pairs of loads");
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

// The rows of one tile: NSEG pairs of operands whose products add up (the parts
// of split operands), each from the tile's first row.
template <int NSEG>
struct NtTile {
  const void* p[NSEG];
  const void* q[NSEG];
  uint32_t ldp, ldq;   // bytes from row to row, multiples of 16
  int prows, qrows;    // rows there are from the tile's first; others read as zeros
  int kbytes;          // of a row; a last chunk's bytes past it are multiplied too
};

template <class T, class C, int NSEG>
__device__ __forceinline__ void nt_product(const NtTile<NSEG>& t, char* lds,
                                           typename T::Acc (&acc)[C::TP][C::TQ]) {
  typedef typename T::Frag Frag;
  constexpr int TP = C::TP, TQ = C::TQ, S = C::S, IP = C::IP, IQ = C::IQ, I = IP + IQ;
  constexpr uint32_t OOB = 0x80000000u;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave / C::WQ, wq = wave % C::WQ;
  const int lrow = lane & 31, lhi = lane >> 5;

  // loads: instruction i of a wave takes rows 8 * (wave * I. + i) .. + 7, lane l
  // row l / 8 of them and the chunk that lies at l % 8 of that row
  const int prec = (t.prows < C::BP ? t.prows : C::BP) * (int)t.ldp;
  const int qrec = (t.qrows < C::BQ ? t.qrows : C::BQ) * (int)t.ldq;
  int ck[2];           // byte of the chunk in its row's slice, even and odd instructions
  uint32_t pv[2], qv[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    ck[h] = ((lane & 7) ^ ((h * 4 + (lane >> 4)) & 7)) * 16;
    pv[h] = (uint32_t)(wave * IP * 8 + (lane >> 3)) * t.ldp + (uint32_t)ck[h];
    qv[h] = (uint32_t)(wave * IQ * 8 + (lane >> 3)) * t.ldq + (uint32_t)ck[h];
  }
  int k0 = 0, seg = 0;  // the slice loaded next
  const void *pp = t.p[0], *qp = t.q[0];
  bool in[2];
  auto begin = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) in[h] = k0 + ck[h] < t.kbytes;
  };
  auto load = [&](char* buf, int i) {
    if (i < IP) {
      const uint32_t off = pv[i & 1] + ((uint32_t)(i * 8) * t.ldp + (uint32_t)k0);
      nt_load(nt_rsrc(pp, prec), buf + (wave * IP + i) * 1024, in[i & 1] ? off : OOB);
    } else {
      const int j = i - IP;
      const uint32_t off = qv[j & 1] + ((uint32_t)(j * 8) * t.ldq + (uint32_t)k0);
      nt_load(nt_rsrc(qp, qrec), buf + C::BP * 128 + (wave * IQ + j) * 1024,
              in[j & 1] ? off : OOB);
    }
  };
  auto advance = [&]() {
    k0 += 128;
    if (NSEG > 1 && k0 >= t.kbytes && seg + 1 < NSEG) {
      k0 = 0;
      ++seg;
#pragma unroll
      for (int s = 1; s < NSEG; ++s)
        if (seg == s) {
          pp = t.p[s];
          qp = t.q[s];
        }
    }
  };

#pragma unroll
  for (int a = 0; a < TP; ++a)
#pragma unroll
    for (int b = 0; b < TQ; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[a][b][e] = 0;

  const int swz = (lrow >> 1) & 7;
  Frag fp[2][TP], fq[2][TQ];
  auto fetch = [&](const char* buf, int ks, Frag (&p)[TP], Frag (&q)[TQ]) {
    const int pos = ((ks * 2 + lhi) ^ swz) * 16;
#pragma unroll
    for (int b = 0; b < TQ; ++b)
      q[b] = *reinterpret_cast<const Frag*>(buf + C::BP * 128 + ((wq * TQ + b) * 32 + lrow) * 128 + pos);
#pragma unroll
    for (int a = 0; a < TP; ++a)
      p[a] = *reinterpret_cast<const Frag*>(buf + ((wp * TP + a) * 32 + lrow) * 128 + pos);
  };
  auto mma = [&](const Frag (&p)[TP], const Frag (&q)[TQ]) {
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
      for (int b = 0; b < TQ; ++b) acc[a][b] = T::mma(p[a], q[b], acc[a][b]);
  };

  const int KT = NSEG * ((t.kbytes + 127) / 128);
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
  fetch(lds, 0, fp[0], fq[0]);
  int rd = 0, wr = S - 1;
  for (int kt = 0; kt < KT; ++kt) {
    const char* cur = lds + rd * C::STAGE;
    char* nxt = lds + wr * C::STAGE;
    constexpr int Q1 = (I + 2) / 3, Q2 = 2 * Q1 < I ? 2 * Q1 : I;
    begin();
    fetch(cur, 1, fp[1], fq[1]);
#pragma unroll
    for (int i = 0; i < Q1; ++i) load(nxt, i);
    mma(fp[0], fq[0]);
    __builtin_amdgcn_sched_barrier(0);
    fetch(cur, 2, fp[0], fq[0]);
#pragma unroll
    for (int i = Q1; i < Q2; ++i) load(nxt, i);
    mma(fp[1], fq[1]);
    __builtin_amdgcn_sched_barrier(0);
    fetch(cur, 3, fp[1], fq[1]);
#pragma unroll
    for (int i = Q2; i < I; ++i) load(nxt, i);
    mma(fp[0], fq[0]);
    advance();
    __builtin_amdgcn_sched_barrier(0);
    // this wave's reads of the stage are complete and its part of the next one
    // has landed: publish it, and free this stage
    __builtin_amdgcn_s_waitcnt(WAIT);
    nt_barrier();
    rd = rd + 1 == S ? 0 : rd + 1;
    wr = wr + 1 == S ? 0 : wr + 1;
    fetch(lds + rd * C::STAGE, 0, fp[0], fq[0]);
    mma(fp[1], fq[1]);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();  // every load has landed and every read is done: LDS is free
}

// A wave's 32 x 32 tile as the products leave it has rows p = 8 (e/4) + 4 (l/32)
// + e%4 of column q = l % 32 in lane l; afterwards v[8h + i] is row 16h + 8 (l/32)
// + i of that column: runs of 8.
template <class Acc>
__device__ __forceinline__ void nt_rows(const Acc& acc, unsigned (&v)[16]) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const auto x = acc[e];  // (a bit cast of a vector's element itself takes element 0)
    v[e] = __builtin_bit_cast(unsigned, x);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto r = __builtin_amdgcn_permlane32_swap(v[8 * h + i], v[8 * h + 4 + i], false, false);
      v[8 * h + i] = (unsigned)r[0];
      v[8 * h + 4 + i] = (unsigned)r[1];
    }
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

typedef NtCfg<2, 2, 4, 4, 2, 1> Nt256;  // 256 x 256
typedef NtCfg<2, 2, 2, 2, 2, 2> Nt128;  // 128 x 128
typedef NtCfg<2, 2, 1, 1, 3, 3> Nt64;   // 64 x 64

}  // namespace fp16k
