// The product of two row-major operands over their rows' common length,
//   D[p][q] = sum_k P[p][k] * Q[q][k],
// for binary16 rows (float32 sums) and 8-bit integer rows (32-bit sums), as the
// inner part of a workgroup's tile.  Both element types take the same bytes the
// same way: a lane's fragment is 16 bytes of one row (8 halves or 16 integers),
// a slice of the reduction is 128 bytes of every row.
//
// A workgroup owns BP x BQ outputs, WP x WQ waves TP x TQ tiles of 32 x 32 each; KG
// such groups split the reduction where few tiles have a long one, and add up in
// LDS.  The slices go through S stages of LDS, loaded past the registers
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

template <int WP_, int WQ_, int TP_, int TQ_, int S_, int KG_, int OCC_>
struct NtCfg {
  static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, S = S_, KG = KG_, OCC = OCC_;
  static constexpr int WAVES = WP * WQ;            // of one group
  static constexpr int THREADS = 64 * WAVES * KG;
  static constexpr int BP = 32 * TP * WP, BQ = 32 * TQ * WQ;
  static constexpr int IP = BP / (8 * WAVES), IQ = BQ / (8 * WAVES);  // loads a wave and slice
  static constexpr int STAGE = (BP + BQ) * 128, RING = S * STAGE;
  static constexpr int LDS = KG * RING;
  static constexpr int SUM = 1024 * TP * TQ * 4 * WAVES;  // one group's sums
  static_assert(IP % 2 == 0 && IQ % 2 == 0, "the chunk order goes by pairs of loads");
  static_assert(LDS * OCC <= 160 * 1024 && (KG - 1) * SUM <= LDS, "LDS");
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
__device__ __forceinline__ void nt_product(const NtTile<NSEG>& t, char* lds0,
                                           typename T::Acc (&acc)[C::TP][C::TQ]) {
  typedef typename T::Frag Frag;
  constexpr int TP = C::TP, TQ = C::TQ, S = C::S, IP = C::IP, IQ = C::IQ, I = IP + IQ;
  constexpr uint32_t OOB = 0x80000000u;
  const int lane = threadIdx.x & 63;
  const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = all % C::WAVES, grp = all / C::WAVES;
  const int wp = wave / C::WQ, wq = wave % C::WQ;
  const int lrow = lane & 31, lhi = lane >> 5;
  char* const lds = lds0 + grp * C::RING;

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
  // the slices of all pairs in order, a range of them for each group
  const int per1 = (t.kbytes + 127) / 128;  // of one pair
  const int KT = (NSEG * per1 + C::KG - 1) / C::KG;
  int k0 = 0, seg = 0;  // the slice loaded next
  int left = KT;        // and how many there are from it
  if (C::KG > 1) {
    const int s0 = grp * KT;
    seg = s0 / per1;
    k0 = (s0 - seg * per1) * 128;
    left = NSEG * per1 - s0 < KT ? NSEG * per1 - s0 : KT;
  }
  const void *pp = t.p[0], *qp = t.q[0];
  auto pair = [&]() {
#pragma unroll
    for (int s = 1; s < NSEG; ++s)
      if (seg == s) {
        pp = t.p[s];
        qp = t.q[s];
      }
  };
  if (C::KG > 1) pair();
  bool in[2];
  auto begin = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) in[h] = k0 + ck[h] < t.kbytes && (C::KG == 1 || left > 0);
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
    --left;
    if (NSEG > 1 && k0 >= t.kbytes && seg + 1 < NSEG) {
      k0 = 0;
      ++seg;
      pair();
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
  // One sub-step: the products of one set of fragments, between them the reads of
  // the next set (sub-step ks of `from`) and loads L0 .. L1 - 1 into `to`, an
  // instruction or two after each product (kept there by the scheduling barriers;
  // left to itself the compiler issues them in bursts that hold the products up).
  auto substep = [&](const Frag (&p)[TP], const Frag (&q)[TQ], const char* from, int ks,
                     Frag (&np)[TP], Frag (&nq)[TQ], char* to, auto l0, auto l1) {
    constexpr int M = TP * TQ, R = TP + TQ, L0 = decltype(l0)::value, V = decltype(l1)::value - L0;
    const int pos = ((ks * 2 + lhi) ^ swz) * 16;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int a = i / TQ, b = i % TQ;
      acc[a][b] = T::mma(p[a], q[b], acc[a][b]);
#pragma unroll
      for (int r = R * i / M; r < R * (i + 1) / M; ++r) {
        if (r < TQ)
          nq[r < TQ ? r : 0] = *reinterpret_cast<const Frag*>(
              from + C::BP * 128 + ((wq * TQ + r) * 32 + lrow) * 128 + pos);
        else
          np[r < TQ ? 0 : r - TQ] = *reinterpret_cast<const Frag*>(
              from + ((wp * TP + r - TQ) * 32 + lrow) * 128 + pos);
      }
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
  fetch(lds, 0, fp[0], fq[0]);
  int rd = 0, wr = S - 1;
  for (int kt = 0; kt < KT; ++kt) {
    const char* cur = lds + rd * C::STAGE;
    char* nxt = lds + wr * C::STAGE;
    constexpr std::integral_constant<int, 0> L0{};
    constexpr std::integral_constant<int, (I + 1) / 2> L1{};
    constexpr std::integral_constant<int, I> L2{};
    begin();
    substep(fp[0], fq[0], cur, 1, fp[1], fq[1], nxt, L0, L1);
    substep(fp[1], fq[1], cur, 2, fp[0], fq[0], nxt, L1, L2);
    advance();
    substep(fp[0], fq[0], cur, 3, fp[1], fq[1], nxt, L2, L2);
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
  if (C::KG > 1) {
    // the groups' sums into the first one's, in order
    typedef typename T::Acc Acc;
    Acc* sums = reinterpret_cast<Acc*>(lds0);
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
      for (int b = 0; b < TQ; ++b)
        if (grp > 0) sums[(((grp - 1) * C::WAVES + wave) * TP * TQ + a * TQ + b) * 64 + lane] = acc[a][b];
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int g = 1; g < C::KG; ++g)
#pragma unroll
        for (int a = 0; a < TP; ++a)
#pragma unroll
          for (int b = 0; b < TQ; ++b)
            acc[a][b] += sums[(((g - 1) * C::WAVES + wave) * TP * TQ + a * TQ + b) * 64 + lane];
    }
    __syncthreads();
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

// A wave's outputs to memory, 32 columns q of its 32 TP rows p at a time.  The
// products leave rows p = 8 (e/4) + 4 (l/32) + e%4 of column q = l%32 in lane l, so
// that memory would see runs of 32 bytes; through LDS each lane gets 8 consecutive
// p of one q and 4 TP lanes a whole run of 32 TP:
//   epi.apply(b, i, p, q, v, out)  v[8] the sums of block b, pass i = 0 .. 2 TP - 1;
//                                  stores there what goes out[q][p ..], and sets
//                                  out[PARTS] for `mirror`
//   epi.load(b, i, p, q)           the same one block ahead: reads what apply needs
// With `mirror`, out is also stored transposed, mir[s][p * ldm + q] (its 16-byte
// chunks in LDS exclusive-ored with the row, since the writes step 8 rows a lane).  Blocks of 32
// rows or columns past plim, qlim are left out (apply and load guard within them).
template <class C, int PARTS>
struct NtEpi {
  static constexpr int TP = C::TP, TQ = C::TQ;
  static constexpr int GB = TQ % 2 == 0 && PARTS == 1 ? 2 : 1;  // blocks a mirrored run
  static constexpr int FLD = 32 * TP + 4, MLD = 32 * GB + 8;    // floats, halves
  static constexpr int WAVE = 32 * FLD * 4 + PARTS * 32 * TP * MLD * 2;
  static constexpr int LDS = WAVE * C::WAVES > C::LDS ? WAVE * C::WAVES : C::LDS;
  static_assert(LDS * C::OCC <= 160 * 1024, "LDS");
};

template <class C, int PARTS, class Acc, class Epi>
__device__ __forceinline__ void nt_store(const Acc (&acc)[C::TP][C::TQ], char* lds, int p0, int q0,
                                         int plim, int qlim, bool mirror, h16* const (&mir)[PARTS],
                                         int ldm, Epi& epi) {
  typedef NtEpi<C, PARTS> E;
  constexpr int TP = E::TP, TQ = E::TQ, GB = E::GB, FLD = E::FLD, MLD = E::MLD;
  constexpr int CPR = 4 * TP, IT = 2 * TP;  // chunks of a run, passes of a block
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lrow = lane & 31, lhi = lane >> 5;
  typedef decltype(acc[0][0][0] + 0) V;
  V* const f = reinterpret_cast<V*>(lds + wave * E::WAVE);
  h16* const m = reinterpret_cast<h16*>(f + 32 * FLD);
  auto load = [&](int b) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int r = (i * 64 + lane) / CPR, c = (i * 64 + lane) % CPR;
      if (b < TQ) epi.load(b, i, p0 + 8 * c, q0 + 32 * b + r);
    }
  };
  load(0);
#pragma unroll
  for (int b = 0; b < TQ; ++b) {
    load(b + 1);
#pragma unroll
    for (int a = 0; a < TP; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        typedef V V4 __attribute__((ext_vector_type(4)));
        const V4 v = {acc[a][b][4 * e], acc[a][b][4 * e + 1], acc[a][b][4 * e + 2],
                      acc[a][b][4 * e + 3]};
        *reinterpret_cast<V4*>(f + lrow * FLD + 32 * a + 8 * e + 4 * lhi) = v;
      }
    nt_wave_sync();
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int r = (i * 64 + lane) / CPR, c = (i * 64 + lane) % CPR;
      V v[8];
      __builtin_memcpy(v, f + r * FLD + 8 * c, 32);
      V8 out[PARTS];
      epi.apply(b, i, p0 + 8 * c, q0 + 32 * b + r, v, out);
      if (mirror) {
#pragma unroll
        for (int s = 0; s < PARTS; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            m[s * 32 * TP * MLD + (8 * c + e) * MLD + (((4 * (b % GB) + r / 8) ^ ((c >> 1) & (4 * GB - 1))) * 8) +
              r % 8] = out[s].h[e];
      }
    }
    nt_wave_sync();
    if (mirror && b % GB == GB - 1) {
      constexpr int MC = 4 * GB;  // chunks of a mirrored run
#pragma unroll
      for (int s = 0; s < PARTS; ++s)
#pragma unroll
        for (int i = 0; i < 32 * TP * MC / 64; ++i) {
          const int r = (i * 64 + lane) / MC, c = (i * 64 + lane) % MC;
          const int q = q0 + 32 * (b - GB + 1) + 8 * c;
          if (p0 + r < plim && q < qlim)
            store16(mir[s] + (int64_t)(p0 + r) * ldm + q,
                    load16(m + s * 32 * TP * MLD + r * MLD + 8 * (c ^ ((r >> 4) & (4 * GB - 1)))));
        }
      nt_wave_sync();
    }
  }
}

//             waves  tile  stages  groups  workgroups a CU
typedef NtCfg<2, 2, 4, 4, 2, 1, 1> Nt256;   // 256 x 256
typedef NtCfg<2, 2, 3, 3, 3, 1, 1> Nt192;   // 192 x 192
typedef NtCfg<2, 2, 2, 2, 2, 1, 2> Nt128;   // 128 x 128
typedef NtCfg<2, 2, 1, 1, 3, 1, 3> Nt64;    // 64 x 64
typedef NtCfg<2, 2, 1, 1, 2, 4, 1> Nt64k;   // 64 x 64, the reduction split in four

}  // namespace fp16k
