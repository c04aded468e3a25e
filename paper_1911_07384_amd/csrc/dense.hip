// Dense layers: y = drop(act(x W^T + bias)) + residual in one product, and the
// gradients of x, W and bias.
//
//   forward   z = x W^T + bias       rows of both operands run along the reduction
//   dx        dz W                   W's columns do
//   dW        dz^T x                 both operands' columns do
//   with dz = drop(dy) act'(z), a pass over the elements that also sums its columns for
//   dbias.
//
// Tile rows p run along the output's rows in memory, tile columns q are its rows.

#include "gemm_dense.hpp"
#include "head.hpp"

#include <stdio.h>

#include <type_traits>

namespace fp16k {
namespace {

// ---- activations -------------------------------------------------------------------

// Phi(-u) exp(u^2 / 2) for u >= 0: a polynomial of t = 1 / (1 + 0.3 u) whose largest
// relative error on [0, 6.2] is 2^-19 (least squares reweighted towards the largest
// error, in 64 bits); past 6.2 u Phi(-u) is below binary16's smallest.
__device__ __forceinline__ float normal_tail(float u) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, u, 1.0f));
  float g = -0.08251488231f;
  g = __builtin_fmaf(g, t, 0.23263196995f);
  g = __builtin_fmaf(g, t, -0.03640279134f);
  g = __builtin_fmaf(g, t, 0.15505104012f);
  g = __builtin_fmaf(g, t, 0.11087362581f);
  g = __builtin_fmaf(g, t, 0.12036026875f);
  return g * t;
}
constexpr float kLog2e = 1.4426950408889634f;

// log2 Phi(-u) for 0 <= u <= 8: a polynomial (least largest difference, its coefficients
// rounded to float32 one after the other) that gives Phi(-u) to 2^-16.7 of itself, float32
// roundings included.  Past 8, u Phi(-u) is nothing to binary16, also times a dropout's
// largest scale.
__device__ __forceinline__ float log2_tail(float u) {
  float g = 7.4281629736e-08f;
  g = __builtin_fmaf(g, u, -3.6551639369e-06f);
  g = __builtin_fmaf(g, u, 7.9570614616e-05f);
  g = __builtin_fmaf(g, u, -1.0219418909e-03f);
  g = __builtin_fmaf(g, u, 8.7619917467e-03f);
  g = __builtin_fmaf(g, u, -5.4336886853e-02f);
  g = __builtin_fmaf(g, u, -4.5819622278e-01f);
  g = __builtin_fmaf(g, u, -1.1513216496e+00f);
  return __builtin_fmaf(g, u, -9.9999230497e-01f);
}

// (maximum and minimum: NaN where an operand is.)  GELU z Phi(z) = max(z, 0) - |z| Phi(-|z|),
// whose terms do not cancel.  An epilogue's activations take the time of their instructions,
// of 8192 x 4096 x 4096 (210 us without) GELU 9 us (14 by normal_tail, which needs a
// reciprocal besides, and erfcf three times that), SiLU 5.
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == kActRelu) return __builtin_elementwise_maximum(z, 0.0f);
  if (ACT == kActGelu) {
    const float u = __builtin_elementwise_minimum(__builtin_fabsf(z), 8.0f);
    return __builtin_fmaf(-u, __builtin_amdgcn_exp2f(log2_tail(u)),
                          __builtin_elementwise_maximum(z, 0.0f));
  }
  if (ACT == kActSilu) {  // (from -110 down the denominator is infinite)
    const float u = __builtin_elementwise_maximum(z, -110.0f);
    return u * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -kLog2e));
  }
  return z;
}
// .. and the slopes, Phi(z) + z phi(z) with 1 - Phi(-z) for positive z, and
// s (1 + z (1 - s)).
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == kActRelu) return z > 0.0f ? 1.0f : __builtin_isnan(z) ? z : 0.0f;
  if (ACT == kActGelu) {
    const float u = __builtin_elementwise_minimum(__builtin_fabsf(z), 15.0f);
    const float e = __builtin_amdgcn_exp2f(u * u * (-0.5f * kLog2e));
    const float h = e * __builtin_fmaf(u, -0.3989422804f, normal_tail(u));
    return z > 0.0f ? 1.0f - h : h;
  }
  if (ACT == kActSilu) {
    const float u = __builtin_elementwise_minimum(
        __builtin_elementwise_maximum(z, -110.0f), 110.0f);
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * -kLog2e));
    return s * __builtin_fmaf(u, 1.0f - s, 1.0f);
  }
  return 1.0f;
}

// Eight elements from element i on (any i) under the dropout's mask.
template <bool XOR3 = false>
__device__ __forceinline__ void drop8(float (&v)[8], int64_t i, const Drop& d) {
  const uint64_t seed = d.state[0], step = d.state[1];
  const uint32_t g = (uint32_t)(i >> 3);
  const int s = (int)(i & 7);
  PhiloxBlock b = philox<XOR3>(g, d.site, step, seed);
  if (s) {  // the words s .. 7 of one block and 0 .. s - 1 of the next
    const PhiloxBlock n = philox<XOR3>(g + 1, d.site, step, seed);
    const uint32_t w[8] = {b.w[0], b.w[1], b.w[2], b.w[3], n.w[0], n.w[1], n.w[2], n.w[3]};
    uint32_t h[5];
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      const uint32_t w0 = w[k], w1 = w[k + 1], w2 = w[k + 2], w3 = w[k + 3 < 8 ? k + 3 : 7];
      const uint32_t x = s & 4 ? w2 : w0, y = s & 4 ? w3 : w1;
      h[k] = s & 2 ? y : x;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      b.w[k] = s & 1 ? __builtin_amdgcn_alignbit(h[k + 1], h[k], 16) : h[k];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = kept(b, e, d.threshold) ? v[e] * d.scale : 0.0f;
}

// ---- what a tile stores (see dense_store) -----------------------------------------------

// Rounded, [q][p].
struct HalfEpi {
  h16* d;
  int np, nq;
  static constexpr int OUTS = 1;
  struct Col {};
  struct Pre {};
  __device__ __forceinline__ Col column(int) const { return {}; }
  __device__ __forceinline__ Pre load(int, int) const { return {}; }
  __device__ __forceinline__ void compute(int, int, const float (&v)[8], Col, Pre,
                                          V8 (&out)[1]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) out[0].h[k] = to_h16(v[k]);
  }
  __device__ __forceinline__ void store(int p, int q, const V8 (&out)[1]) const {
    if (p < np && q < nq) store8_upto(d + (int64_t)q * np + p, out[0], np - p);
  }
};

// The float32 sums of one part of a reduction, [q][p] with rows of whole eights.
struct PartEpi {
  float* d;
  int np, nq, ld;
  static constexpr int OUTS = 2;
  struct Col {};
  struct Pre {};
  __device__ __forceinline__ Col column(int) const { return {}; }
  __device__ __forceinline__ Pre load(int, int) const { return {}; }
  __device__ __forceinline__ void compute(int, int, const float (&v)[8], Col, Pre,
                                          V8 (&out)[2]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) out[k / 4].d[k % 4] = __builtin_bit_cast(uint32_t, v[k]);
  }
  __device__ __forceinline__ void store(int p, int q, const V8 (&out)[2]) const {
    if (p < np && q < nq) {
      float* to = d + (int64_t)q * ld + p;
      store16(to, out[0]);
      store16(to + 4, out[1]);
    }
  }
};

// The layer's outputs.
template <int ACT>
struct LayerEpi {
  const h16 *bias, *residual;
  h16 *y, *z;
  int np, nq;
  Drop drop;
  static constexpr int OUTS = 2;
  struct Col {
    V8 bias;
  };
  struct Pre {
    V8 residual;
  };
  __device__ __forceinline__ Col column(int p) const {
    return {bias && p < np ? load8_upto(bias + p, np - p) : zero8()};
  }
  __device__ __forceinline__ Pre load(int p, int q) const {
    return {residual && p < np && q < nq ? load8_upto(residual + (int64_t)q * np + p, np - p)
                                         : zero8()};
  }
  __device__ __forceinline__ void compute(int p, int q, const float (&sum)[8], const Col& col,
                                          const Pre& pre, V8 (&out)[2]) const {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = sum[k] + to_f32(col.bias.h[k]);
      out[1].h[k] = to_h16(v[k]);
      v[k] = act_value<ACT>(v[k]);
    }
    if (drop.threshold) drop8(v, (int64_t)q * np + p, drop);
#pragma unroll
    for (int k = 0; k < 8; ++k) out[0].h[k] = to_h16(v[k] + to_f32(pre.residual.h[k]));
  }
  __device__ __forceinline__ void store(int p, int q, const V8 (&out)[2]) const {
    if (p < np && q < nq) {
      const int64_t i = (int64_t)q * np + p;
      store8_upto(y + i, out[0], np - p);
      if (z) store8_upto(z + i, out[1], np - p);
    }
  }
};

// ---- the product -----------------------------------------------------------------------

// D[q][p] = sum_k P(p, k) Q(q, k), the operands' rows ldp and ldq elements apart,
// multiples of 8: P[p * ldp + k], or P[k * ldp + p] along its rows; likewise Q.
struct Product {
  const h16 *p, *q;
  int64_t ldp, ldq;
  int np, nq, nk;
  int parts;
};

// Tiles in groups of 8 tile columns, within a group column by column: the 32 tiles that
// an XCD holds at a time share 8 + 4 tiles' rows in its L2.
// Measured (256 x 256 tiles): 8192 x 4096 x 4096 without an epilogue 210 us (1310 TFLOP/s; a
// library product 200), 4096 x 4096 x 4096 forward 104, dx 111, dW 116 (96-100, 120 and
// 139).  Bound by the matrix cores' power, and by an epilogue that nothing overlaps at one
// workgroup a CU: a residual or a kept z of 8192 x 4096 adds 15 us, its bytes' time.
template <class C, class Epi>
__global__ __launch_bounds__(C::BOUND, 2) void dense_product(const Product a, Epi epi) {
  __shared__ __attribute__((aligned(1024))) char lds[C::G * C::LDS];
  const int tp = (a.np + C::BP - 1) / C::BP, tq = (a.nq + C::BQ - 1) / C::BQ;
  const int all = tp * tq * a.parts;
  int t = dense_xcd(blockIdx.x, all);
  if (t >= all) return;
  const int part = t / (tp * tq);
  t -= part * tp * tq;
  const int g = t / (8 * tp), w = t - g * 8 * tp;
  const int gw = tq - 8 * g < 8 ? tq - 8 * g : 8;
  const int p0 = (w / gw) * C::BP, q0 = (8 * g + w % gw) * C::BQ;
  DenseTile d;
  d.ldp = (uint32_t)(a.ldp * 2);
  d.ldq = (uint32_t)(a.ldq * 2);
  d.p = a.p + (C::PS ? (int64_t)p0 : p0 * a.ldp);
  d.q = a.q + (C::QS ? (int64_t)q0 : q0 * a.ldq);
  d.prows = a.np - p0;
  d.qrows = a.nq - q0;
  d.nk = a.nk;
  int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = C::G > 1 ? wave / C::WAVES : 0;
  wave -= group * C::WAVES;
  d.part = part * C::G + group;
  d.parts = a.parts * C::G;
  floatx4 acc[C::TP][C::TQ];
  dense_loop<C>(d, lds + group * C::LDS, wave, acc);
  if constexpr (C::G > 1) {
    dense_groups<C>(lds, group, wave, acc);
    if (group > 0) return;
  }
  if constexpr (std::is_same<Epi, PartEpi>::value) epi.d += (int64_t)part * epi.nq * epi.ld;
  dense_store<C>(acc, p0 + (wave / C::WQ) * 16 * C::TP, q0 + (wave % C::WQ) * 16 * C::TQ, epi);
}

// The parts' sums added in their order, and the product's epilogue: bound by the launch
// and one trip to memory (2.7 us for 8 parts of 128 x 1000, 4.1 for 2 of 24 x 4096).
template <class Epi>
__global__ __launch_bounds__(256) void dense_join(const float* from, int parts, int np, int nq,
                                                  int ld, const Epi epi) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per = ld / 8, q = (int)(i / per), p = (int)(i - (int64_t)q * per) * 8;
  if (q >= nq) return;
  const typename Epi::Col col = epi.column(p);
  const typename Epi::Pre pre = epi.load(p, q);
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const float* f = from + (int64_t)q * ld + p;
#pragma unroll 4
  for (int s = 0; s < parts; ++s, f += (int64_t)nq * ld) {
    const floatx4 x = reinterpret_cast<const floatx4*>(f)[0];
    const floatx4 y = reinterpret_cast<const floatx4*>(f)[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] += x[k];
      v[4 + k] += y[k];
    }
  }
  V8 out[Epi::OUTS];
  epi.compute(p, q, v, col, pre, out);
  epi.store(p, q, out);
}

enum Layout { kForward, kDx, kDw };  // which operands lie along their rows: none, P, both

template <Layout L, int WP, int WQ, int TQ, int S, int OCC, int G = 1>
using Cfg = DenseCfg<WP, WQ, 8, TQ, S, OCC, L != kForward, L == kDw, G>;

//                                 waves  tiles  stages  workgroups a CU (groups)
template <Layout L> using Cfg256 = Cfg<L, 2, 4, 4, 2, 1>;  // 256 x 256
template <Layout L> using Cfg128 = Cfg<L, 1, 4, 2, 2, 2>;  // 128 x 128
template <Layout L> using Cfg128d = Cfg<L, 1, 4, 2, 4, 1>;  // .. loads further ahead
template <Layout L> using Cfg64 = Cfg<L, 1, 4, 1, 3, 2>;   // 128 x 64
template <Layout L> using Cfg32 = Cfg<L, 1, 2, 1, 2, 1, 4>;  // 128 x 32, four groups

template <class Epi>
hipError_t launch_join(const Product& a, const float* sums, int ld, const Epi& epi,
                       hipStream_t st) {
  dense_join<<<(unsigned)ceil_div64((int64_t)a.nq * (ld / 8), 256), 256, 0, st>>>(
      sums, a.parts, a.np, a.nq, ld, epi);
  return hipGetLastError();
}

template <class C, class Epi>
hipError_t run(const Product& a, const Epi& epi, float* sums, hipStream_t st) {
  const int64_t all = ceil_div64(a.np, C::BP) * ceil_div64(a.nq, C::BQ) * a.parts;
  const unsigned grid = (unsigned)(8 * ceil_div64(all, 8));
  if (a.parts == 1) {
    dense_product<C><<<grid, C::THREADS, 0, st>>>(a, epi);
    return hipGetLastError();
  }
  const int ld = (a.np + 7) & ~7;
  dense_product<C><<<grid, C::THREADS, 0, st>>>(a, PartEpi{sums, a.np, a.nq, ld});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_join(a, sums, ld, epi, st);
}

// The tile a product runs on, and the parts its reduction is split into: the least of
// the times below, in microseconds: of a slice with one workgroup a CU and with two, and
// of a workgroup's start and end, for each layout, fitted to 14 products of 32 to 8192
// tokens and 512 to 4096 inputs and outputs in three layouts, each on every tile and
// with up to 32 parts.  What it chooses for them takes 1.4 % longer than the best choice
// (geometric mean; 13 % at most).  For the largest the 256 x 256 tile's slices cost 1.5
// us for four times the outputs that the others do in 0.49 (128 x 128) or 0.62 us.
// One workgroup a CU of 128 x 128 is held up by its loads with two stages: with four a
// forward's slice takes 0.50 us (2048 x 2048 x 2048 26.0 -> 22.7 us; the other layouts
// gain nothing).
// A slice of dx with few workgroups is held up by its fragments' way from LDS through the
// permutes: four groups of two waves, each with a quarter of the reduction, take turns at it
// and join in LDS (dx of 128 x 2048 x 1000 10.5 -> 7.8 us, 256 x 1024 x 1024 10.5 -> 7.7;
// two groups of 128 x 64: 9.0 and 9.0); in parts besides they gain nothing, and where W's
// bytes count they lose (8 x 4096 x 16384 29.2 -> 34.2).  The forward's is held up by its
// loads and gains nothing (64 x 1024 x 4096: 7.9 us, 8.4 so).
struct Choice {
  int side, stages, parts;
};
struct Tile {
  int side, stages, occ;
  double one, two, ends;
  int groups = 1;  // a slice's times are of so many
};
Choice choose(Layout l, int64_t np, int64_t nq, int64_t nk) {
  static const Tile tiles[3][4] = {
      {{256, 2, 1, 1.48, 0, 12}, {128, 2, 2, 0.58, 0.97, 5.5}, {64, 3, 2, 0.30, 0.62, 4.7},
       {128, 4, 1, 0.50, 0, 5.5}},
      {{256, 2, 1, 1.55, 0, 12}, {128, 2, 2, 0.70, 1.12, 5.5}, {64, 3, 2, 0.42, 0.79, 4.7},
       {32, 2, 1, 1.10, 0, 4.6, 4}},
      {{256, 2, 1, 1.60, 0, 12}, {128, 2, 2, 0.78, 1.20, 5.5}}};
  const double launch = 4.0, join = 2.5, bytes = 4.5e6;  // (bytes a microsecond)
  const int64_t slices = ceil_div64(nk, 64);
  Choice best = {128, 2, 1};
  double least = 1e300;
  for (const Tile& t : tiles[l]) {
    if (!t.side) continue;
    const int64_t n1 = ceil_div64(np, t.side < 128 ? 128 : t.side) * ceil_div64(nq, t.side);
    for (int64_t want = 1; want <= 32 && want <= slices; want += 1 + want / 4) {
      const int64_t sl = ceil_div64(slices, want * t.groups);
      const int64_t parts = ceil_div64(slices, sl * t.groups);
      if (parts > 1 && (sl < 2 || t.groups > 1)) break;
      // rounds of workgroups on the busiest CU
      const int64_t n = n1 * parts, cu = ceil_div64(n, 256);
      const double full = (double)(cu / t.occ), rest = (double)(cu % t.occ);
      const double end = t.ends - launch;
      double us = launch + full * ((double)sl * (t.occ == 2 ? t.two : t.one) + t.occ * end) +
                  rest * ((double)sl * t.one + end);
      // (a device that is not full runs at a higher clock)
      if (n < 256) us -= 0.2 * (1.0 - (double)n / 256.0) * (double)sl * t.one;
      if (parts > 1) us += join + (double)(parts * np * nq * 8) / bytes;
      if (us < least) {
        least = us;
        best = {t.side, t.stages, (int)parts};
      }
    }
  }
  return best;
}

size_t sums_bytes(const Choice& c, int64_t np, int64_t nq) {
  return c.parts == 1 ? 0 : (size_t)c.parts * nq * ((np + 7) & ~(int64_t)7) * sizeof(float);
}

template <Layout L, class Epi>
hipError_t launch_product(Product a, const Epi& epi, void* sums, hipStream_t st) {
  const Choice c = choose(L, a.np, a.nq, a.nk);
  a.parts = c.parts;
  float* f = static_cast<float*>(sums);
  if constexpr (L != kDw)
    if (c.side == 64) return run<Cfg64<L>>(a, epi, f, st);
  if constexpr (L == kDx)
    if (c.side == 32) return run<Cfg32<L>>(a, epi, f, st);
  if constexpr (L == kForward)
    if (c.side == 128 && c.stages == 4) return run<Cfg128d<L>>(a, epi, f, st);
  if (c.side == 256) return run<Cfg256<L>>(a, epi, f, st);
  return run<Cfg128<L>>(a, epi, f, st);
}

// ---- few tokens ------------------------------------------------------------------------------

// The forward of at most 32 tokens, bound by reading W once: a workgroup takes 16 RF rows
// of W, its sixteen waves (eight with more registers for 64 rows) the reduction in turns
// of 64, each lane 16 bytes of a row straight into the operand (the next turn's before
// this one's products), with no regard to a row's alignment; the waves' sums are added in
// LDS in their order.  Neighbouring workgroups of an XCD start at different turns: at the
// same one, rows of 8 or 32 KB have all of them ask the same memory channels (one token,
// 4096 x 16384 from memory: 31.2 us, 27.4 so; 16 tokens, 16384 x 4096: 33.9 and 29.4).
// One token, 4096 x 16384: 22.4 us, 6.0 TB/s; 24 tokens, 16384 x 4096: 24.0 and 4.1 for joining
// four parts.  Rows that are not aligned: one token, four matrices W in turn (from memory),
// 4096 x 16000 27.1 us, 4098 x 16000 29.2, 4097 x 16000 36.4; one W again and again (in part
// from the caches) 23.9, 22.7 and 29.8.
constexpr int kFewTokens = 32, kFewSteps = 2, kFewTurn = 32 * kFewSteps;
constexpr int few_waves(int rf) { return rf == 4 ? 8 : 16; }

// Eight elements of a row.  Loads of 16 bytes at odd elements take twice the time of those
// at even ones (one token, 4097 x 16000 from memory: 56 us, 36.4 so), so rows of odd length (ODD) are
// read from the even element at or before the first, the eighth by itself, and put in place
// when they are used.
template <bool ODD>
struct FewVec {
  V8 v;
  __device__ __forceinline__ void load(const h16* p, const h16*) { v = load16u(p); }
  __device__ __forceinline__ half8 get(int) const { return v.h; }
};
template <>
struct FewVec<true> {
  V8 v;
  uint32_t last;
  // (p: the even element, eighth: p's, or the next one, as the row starts)
  __device__ __forceinline__ void load(const h16* p, const h16* eighth) {
    typedef u32x4 even __attribute__((aligned(4)));
    v.u = *reinterpret_cast<const even*>(p);
    last = *reinterpret_cast<const uint16_t*>(eighth);
  }
  __device__ __forceinline__ half8 get(int odd) const {  // (odd: the row starts at an odd one)
    V8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r.d[i] = __builtin_amdgcn_alignbit(i < 3 ? v.d[i + 1] : last, v.d[i], 16 * odd);
    return r.h;
  }
};

template <int RF, int NT, bool ODD, class Epi>
__global__ __launch_bounds__(64 * few_waves(RF)) void dense_few(const Product a, Epi epi) {
  constexpr int U = kFewSteps, TURN = kFewTurn, WAVES = few_waves(RF);
  __shared__ floatx4 sums[WAVES][RF * NT * 64];
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int groups = (a.np + 16 * RF - 1) / (16 * RF);
  const int part = blockIdx.x / groups, p0 = (blockIdx.x - part * groups) * 16 * RF;
  // this part's range of the reduction, in whole turns of all waves
  const int per = ((a.nk + a.parts - 1) / a.parts + 7) & ~7;
  const int kbeg = part * per, kend = a.nk < kbeg + per ? a.nk : kbeg + per;
  const h16* pr[RF];  // (rows and tokens that are not there read the last one)
  const h16* qr[NT];
  int po[RF], qo[NT];  // whether a row starts at an odd element
#pragma unroll
  for (int f = 0; f < RF; ++f) {
    const int r = p0 + 16 * f + m, row = r < a.np ? r : a.np - 1;
    po[f] = ODD ? row & 1 : 0;
    pr[f] = a.p + row * a.ldp + 8 * g - po[f];
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 16 * n + m, row = r < a.nq ? r : a.nq - 1;
    qo[n] = ODD ? row & 1 : 0;
    qr[n] = a.q + row * a.ldq + 8 * g - qo[n];
  }
  typedef FewVec<ODD> Vec;
  Vec w[2][U][RF], x[2][U][NT];
  auto load = [&](int k, Vec (&wv)[U][RF], Vec (&xv)[U][NT]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int f = 0; f < RF; ++f)
        wv[u][f].load(pr[f] + k + 32 * u, pr[f] + po[f] + (k + 32 * u + 7));
#pragma unroll
      for (int n = 0; n < NT; ++n)
        xv[u][n].load(qr[n] + k + 32 * u, qr[n] + qo[n] + (k + 32 * u + 7));
    }
  };
  floatx4 acc[RF][NT];
#pragma unroll
  for (int f = 0; f < RF; ++f)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[f][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  auto mma = [&](const Vec (&wv)[U][RF], const Vec (&xv)[U][NT]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      half8 xh[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) xh[n] = xv[u][n].get(qo[n]);
#pragma unroll
      for (int f = 0; f < RF; ++f) {
        const half8 wh = wv[u][f].get(po[f]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, xh[n], acc[f][n], 0, 0, 0);
      }
    }
  };
  constexpr int STEP = TURN * WAVES;
  // this wave's whole turns, and the one that the range ends in
  const int whole = (kend - kbeg) / TURN, turns = (whole - wave + WAVES - 1) / WAVES;
  if (turns > 0) {
    const int first = kbeg + wave * TURN, end = first + turns * STEP;
    int k = first + (int)((blockIdx.x >> 3) % (unsigned)turns) * STEP;
    auto next = [&]() { k = k + STEP < end ? k + STEP : first; };
    load(k, w[0], x[0]);
    int i = turns;
    for (; i > 2; i -= 2) {
      next();
      load(k, w[1], x[1]);
      mma(w[0], x[0]);
      next();
      load(k, w[0], x[0]);
      mma(w[1], x[1]);
    }
    if (i == 2) {
      next();
      load(k, w[1], x[1]);
    }
    mma(w[0], x[0]);
    if (i == 2) mma(w[1], x[1]);
  }
  if (wave == whole % WAVES) {
#pragma unroll 1
    for (int at = kbeg + whole * TURN; at < kend; at += 32) {
      const int left = kend - at - 8 * g;
      V8 wt[RF], xt[NT];
#pragma unroll
      for (int f = 0; f < RF; ++f)
        wt[f] = left > 0 ? load8_upto(pr[f] + po[f] + at, left) : zero8();
#pragma unroll
      for (int n = 0; n < NT; ++n)
        xt[n] = left > 0 ? load8_upto(qr[n] + qo[n] + at, left) : zero8();
#pragma unroll
      for (int f = 0; f < RF; ++f)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[f][n] =
              __builtin_amdgcn_mfma_f32_16x16x32_f16(wt[f].h, xt[n].h, acc[f][n], 0, 0, 0);
    }
  }
#pragma unroll
  for (int f = 0; f < RF; ++f)
#pragma unroll
    for (int n = 0; n < NT; ++n) sums[wave][(f * NT + n) * 64 + lane] = acc[f][n];
  __syncthreads();
  // 8 rows c of one token t a thread; a sum's rows are 4 (lane / 16) + 0 .. 3
  if constexpr (std::is_same<Epi, PartEpi>::value) epi.d += (int64_t)part * epi.nq * epi.ld;
  const int c = threadIdx.x % (2 * RF), t = threadIdx.x / (2 * RF);
  if (t >= a.nq || p0 + 8 * c >= a.np) return;
  const typename Epi::Col col = epi.column(p0 + 8 * c);
  const typename Epi::Pre pre = epi.load(p0 + 8 * c, t);
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int at = ((c / 2) * NT + t / 16) * 64 + (c % 2) * 32 + t % 16;
#pragma unroll
  for (int s = 0; s < WAVES; ++s) {
    const floatx4 lo = sums[s][at], hi = sums[s][at + 16];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] += lo[e];
      v[4 + e] += hi[e];
    }
  }
  V8 out[Epi::OUTS];
  epi.compute(p0 + 8 * c, t, v, col, pre, out);
  epi.store(p0 + 8 * c, t, out);
}

// The rows of W a workgroup takes, over 16, and the parts of the reduction: the least of
// the times below, in microseconds.  Every workgroup reads the tokens again from L2, which
// adds to the time that W takes from memory (0.5 us a token of 128 workgroups and 32 KB); more
// rows read them less often, but a workgroup alone on its CU takes longer, and joining parts
// takes a launch.  24 tokens: 16384 x 4096 45.5, 36.6 and 32.4 us with 16, 32 and 64 rows, 4096 x
// 16384 46.4, 36.4 and 30.1.
struct Few {
  int rows, parts;
};
Few few_choice(int64_t np, int64_t nq, int64_t nk) {
  Few best = {1, 1};
  double least = 1e300;
  for (int rf = 1; rf <= 4; rf *= 2) {
    const int64_t groups = ceil_div64(np, 16 * rf);
    const double alone = (double)nk / 1024.0 * (0.95 * rf + 0.045 * (double)nq + 0.2);
    const double bytes = (double)(np * nk) / 2.8e6 + (double)(groups * nq * nk) / 4.2e6;
    for (int p = 1; p == 1 || (p * groups <= 256 && nk / p >= 1024); ++p) {
      const double rounds = p * groups > 256 ? (double)groups / 256.0 : 1.0;
      double us = 4.0 + alone / p * rounds;
      if (us < bytes) us = bytes;
      us += rf;  // (a longer start and end)
      if (p > 1) us += 3.4 + (double)(p * np * nq * 8) / 4.5e6;
      if (us < least) {
        least = us;
        best = {rf, p};
      }
    }
  }
  return best;
}
// Past 16 tokens of wide layers the tiles read each token less often (24 tokens of 4096 x
// 4096: 12.8 us, 13.4 here; of 4096 x 2048: 10.2 and 8.0), unless rows have to be laid out
// anew for them (4097 x 4000: 26.1 us, 18.2 here).
bool few_ok(int64_t np, int64_t nq, int64_t nk) {
  return nq <= 16 || (nq <= kFewTokens && (np >= 8192 || nk >= 8192 || np * nk <= 1 << 23 ||
                                           (nk & 7)));
}

template <class Epi>
hipError_t launch_few(Product a, const Epi& epi, void* sums, hipStream_t st) {
  const Few c = few_choice(a.np, a.nq, a.nk);
  const int rf = c.rows;
  a.parts = c.parts;
  const unsigned grid = (unsigned)(ceil_div(a.np, 16 * rf) * a.parts);
  auto go = [&](auto e) {
    typedef decltype(e) E;
    const int threads = 64 * few_waves(rf);
    const auto run = [&](auto kernel) { kernel<<<grid, threads, 0, st>>>(a, e); };
    const auto pick = [&](auto tiles, auto odd) {
      constexpr int NT = decltype(tiles)::value;
      constexpr bool ODD = decltype(odd)::value;
      run(rf == 4   ? dense_few<4, NT, ODD, E>
          : rf == 2 ? dense_few<2, NT, ODD, E>
                    : dense_few<1, NT, ODD, E>);
    };
    const auto of = [&](auto tiles) {
      if (a.ldp & 1)
        pick(tiles, std::true_type{});
      else
        pick(tiles, std::false_type{});
    };
    if (a.nq <= 16)
      of(std::integral_constant<int, 1>{});
    else
      of(std::integral_constant<int, 2>{});
    return hipGetLastError();
  };
  if (a.parts == 1) return go(epi);
  const int ld = (a.np + 7) & ~7;
  float* f = static_cast<float*>(sums);
  const hipError_t e = go(PartEpi{f, a.np, a.nq, ld});
  if (e != hipSuccess) return e;
  return launch_join(a, f, ld, epi, st);
}

// ---- rows laid out anew ------------------------------------------------------------------

// Rows whose length is no multiple of 8, to rows that are, zeros behind them; of up to two
// matrices with rows of one length in a launch (a second one took 3 us).  1111 and 2501 rows
// of 1337: 5.8 us, 19 MB at 3.3 TB/s.
struct Repack {
  int rows;
  const h16* from;
  h16* to;
};
__global__ __launch_bounds__(256) void repack_kernel(int cols, int ld, const Repack one,
                                                     const Repack two) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per = ld / 8;
  int64_t r = i / per;
  const int c = (int)(i - r * per) * 8;
  const bool second = r >= one.rows;
  const Repack m = second ? two : one;
  if (second) r -= one.rows;
  if (r < m.rows) store16(m.to + r * ld + c, load8_row(m.from + r * cols, c, cols, true));
}
hipError_t launch_repack(int cols, const Repack& one, const Repack& two, hipStream_t st) {
  const int ld = (cols + 7) & ~7;
  const int64_t n = ((int64_t)one.rows + two.rows) * (ld / 8);
  if (n == 0) return hipSuccess;
  repack_kernel<<<(unsigned)ceil_div64(n, 256), 256, 0, st>>>(cols, ld, one, two);
  return hipGetLastError();
}

// ---- dz and dbias --------------------------------------------------------------------------

constexpr int kRows = 32;  // of a workgroup's partial sums

// One vector of dz: from a row's dy and z, columns c .. c + 7.  dz is rounded to binary16, to be
// an operand of the matrix cores in both products that follow: two parts of it would take
// the products' time twice.  dx and dW are then off by 2.9e-4 (relative 2-norm, 4096 x 4096 x
// 4096) where a float32 dz leaves their own rounding's 2.1e-4, and a dz past 65504 is
// infinite.  dbias is summed before the rounding.
template <int ACT>
__device__ __forceinline__ V8 dz8(const V8& y, const V8& z, int64_t i, const Drop& drop,
                                  float (&s)[8]) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = to_f32(y.h[e]);
  if (drop.threshold) drop8<true>(v, i, drop);
  V8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (ACT != kActNone) v[e] *= act_slope<ACT>(to_f32(z.h[e]));
    s[e] += v[e];
    o.h[e] = to_h16(v[e]);
  }
  return o;
}

// All of dz and dbias for few tokens in one launch: 64 columns a workgroup, a lane 8 of
// them in every 32nd row.  128 x 1000: 3.1 us, most of it a launch's; at 512 tokens with an
// activation its few workgroups take longer than the two launches of more.
constexpr int kDzFew = 128;
template <int ACT>
__global__ __launch_bounds__(256) void dz_few(int tokens, int outputs, int ld, Drop drop,
                                              const h16* z, const h16* dy, h16* dz, h16* dbias) {
  __shared__ float sums[32][64];
  const int cg = threadIdx.x & 7, rg = threadIdx.x >> 3, c = blockIdx.x * 64 + cg * 8;
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  constexpr int U = 4;
  for (int r0 = rg; r0 < tokens; r0 += 32 * U) {
    V8 vy[U], vz[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + 32 * u;
      const int64_t row = (int64_t)(r < tokens ? r : 0) * outputs;
      vy[u] = load8_row(dy + row, c, outputs, r < tokens);
      if (ACT != kActNone) vz[u] = load8_row(z + row, c, outputs, r < tokens);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + 32 * u;
      const V8 o = dz8<ACT>(vy[u], vz[u], (int64_t)r * outputs + c, drop, s);
      if (dz && r < tokens && c < ld) store16(dz + (int64_t)r * ld + c, o);
    }
  }
  if (!dbias) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[rg][cg * 8 + e] = s[e];
  __syncthreads();
  const int cc = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x >= 64 || cc >= outputs) return;
  double t = 0.0;
#pragma unroll
  for (int i = 0; i < 32; ++i) t += (double)sums[i][threadIdx.x];
  dbias[cc] = dbl_to_h16(t);
}

// dz [tokens][ld] (unless null) with zeros past its columns, and its columns' sums over
// kRows rows (unless null): 256 columns a workgroup, a lane 8 of them in every eighth
// row, all of its loads before the first sum.  4096 x 4096, GELU and dropout: 29.5 us, 101 MB
// at 3.4 TB/s; a dropout's block and 8 slopes are about 1,300 cycles of a SIMD, 19 us in all,
// and its bytes take as long, hidden behind them in part.  The three-word difference saves 5 %
// here, and the clamps in place of comparisons as much.
template <int ACT>
__global__ __launch_bounds__(256) void dz_kernel(int tokens, int outputs, int ld, Drop drop,
                                                 const h16* z, const h16* dy, h16* dz,
                                                 float* part) {
  __shared__ float sums[8][256];
  const int cg = threadIdx.x & 31, rg = threadIdx.x >> 5;
  const int c = blockIdx.x * 256 + cg * 8, r0 = blockIdx.y * kRows;
  constexpr int U = kRows / 8;
  V8 vy[U], vz[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + rg + 8 * u;
    const int64_t row = (int64_t)(r < tokens ? r : 0) * outputs;
    vy[u] = load8_row(dy + row, c, outputs, r < tokens);
    if (ACT != kActNone) vz[u] = load8_row(z + row, c, outputs, r < tokens);
  }
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int r = r0 + rg + 8 * u;
    const V8 o = dz8<ACT>(vy[u], vz[u], (int64_t)r * outputs + c, drop, s);
    if (dz && r < tokens && c < ld) store16(dz + (int64_t)r * ld + c, o);
  }
  if (!part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[rg][cg * 8 + e] = s[e];
  __syncthreads();
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) t += sums[i][threadIdx.x];
  const int cc = blockIdx.x * 256 + threadIdx.x;
  if (cc < outputs) part[(int64_t)blockIdx.y * outputs + cc] = t;
}

// 64 columns a workgroup, the parts dealt to its four waves: 4.5 us for 128 parts of 4096
// columns, 2 MB read by 64 workgroups, 32 loads in turn by eights.
__global__ __launch_bounds__(256) void dbias_kernel(int outputs, int parts, const float* part,
                                                    h16* dbias) {
  __shared__ double sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  double s = 0.0;
  if (c < outputs) {
#pragma unroll 8
    for (int i = wave; i < parts; i += 4) s += (double)part[(int64_t)i * outputs + c];
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < outputs)
    dbias[c] = dbl_to_h16((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
}

template <int ACT>
hipError_t launch_dz(const DenseArgs& a, int ld, h16* dz, float* part, hipStream_t st) {
  if (a.tokens <= kDzFew) {
    dz_few<ACT><<<(unsigned)ceil_div(ld, 64), 256, 0, st>>>(a.tokens, a.outputs, ld, a.drop,
                                                            a.kept, a.dy, dz, a.dbias);
    return hipGetLastError();
  }
  const int parts = ceil_div(a.tokens, kRows);
  dz_kernel<ACT><<<dim3((unsigned)ceil_div(ld, 256), (unsigned)parts), 256, 0, st>>>(
      a.tokens, a.outputs, ld, a.drop, a.kept, a.dy, dz, a.dbias ? part : nullptr);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dbias) return e;
  dbias_kernel<<<(unsigned)ceil_div(a.outputs, 64), 256, 0, st>>>(a.outputs, parts, part, a.dbias);
  return hipGetLastError();
}

// ---- workspace -------------------------------------------------------------------------------

int whole8(int n) { return (n + 7) & ~7; }
size_t rows_bytes(int rows, int cols) {
  return ((size_t)rows * whole8(cols) * 2 + 255) & ~(size_t)255;
}

// Places: x and W with rows of whole vectors (where theirs are not), dz, the parts' sums
// (of one product at a time) and dbias's.
struct Places {
  size_t x = 0, w = 0, dz = 0, part = 0, sums = 0, total = 0;
};
size_t take(Places& p, size_t bytes) {
  const size_t at = p.total;
  p.total += (bytes + 255) & ~(size_t)255;
  return at;
}
Places places(int T, int I, int O, bool backward, bool makes) {
  Places p;
  if (!backward && few_ok(O, T, I)) {  // (takes rows as they are)
    const Choice c = {0, 0, few_choice(O, T, I).parts};
    p.sums = take(p, sums_bytes(c, O, T));
    return p;
  }
  if (I & 7) {
    p.x = take(p, rows_bytes(T, I));
    p.w = take(p, rows_bytes(O, I));
  }
  if (!backward) {
    p.sums = take(p, sums_bytes(choose(kForward, O, T, I), O, T));
    return p;
  }
  if (makes || (O & 7)) p.dz = take(p, rows_bytes(T, O));
  if (T > kDzFew) p.part = take(p, (size_t)ceil_div(T, kRows) * O * sizeof(float));
  const size_t dx = sums_bytes(choose(kDx, I, T, O), I, T);
  const size_t dw = sums_bytes(choose(kDw, I, O, T), I, O);
  p.sums = take(p, dx > dw ? dx : dw);
  return p;
}

template <class T>
T* at(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

}  // namespace

size_t dense_fwd_ws_bytes(int tokens, int inputs, int outputs) {
  return places(tokens, inputs, outputs, false, false).total;
}

size_t dense_bwd_ws_bytes(int tokens, int inputs, int outputs, bool dz) {
  return places(tokens, inputs, outputs, true, dz).total;
}

void dense_name(int tokens, int inputs, int outputs, int product, char* name, size_t size) {
  const int64_t T = tokens, I = inputs, O = outputs;
  char in[16] = "";
  if (product == kForward && few_ok(O, T, I)) {
    const Few c = few_choice(O, T, I);
    if (c.parts > 1) snprintf(in, sizeof(in), " in %d", c.parts);
    snprintf(name, size, "few tokens, %d rows%s", 16 * c.rows, in);
    return;
  }
  const Choice c = product == kForward ? choose(kForward, O, T, I)
                   : product == kDx    ? choose(kDx, I, T, O)
                                       : choose(kDw, I, O, T);
  if (c.parts > 1) snprintf(in, sizeof(in), " in %d", c.parts);
  snprintf(name, size, "%d x %d%s%s", c.side < 128 ? 128 : c.side, c.side,
           c.stages == 4 ? " deep" : "", in);
}

#define RUN(expr)                     \
  do {                                \
    const hipError_t e_ = (expr);     \
    if (e_ != hipSuccess) return e_;  \
  } while (0)

hipError_t launch_dense_fwd(const DenseArgs& a, hipStream_t st) {
  const int T = a.tokens, I = a.inputs, O = a.outputs;
  const bool few = few_ok(O, T, I);
  const int ld = few ? I : whole8(I);
  const Places at_ = places(T, I, O, false, false);
  const h16 *x = a.x, *w = a.w;
  if (ld != I) {
    h16 *xs = at<h16>(a.ws, at_.x), *ws = at<h16>(a.ws, at_.w);
    RUN(launch_repack(I, {T, a.x, xs}, {O, a.w, ws}, st));
    x = xs;
    w = ws;
  }
  const Product p = {w, x, ld, ld, O, T, I, 1};
  void* sums = at<void>(a.ws, at_.sums);
  const auto go = [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    const LayerEpi<ACT> epi = {a.bias, a.residual, a.y, a.z, O, T, a.drop};
    return few ? launch_few(p, epi, sums, st) : launch_product<kForward>(p, epi, sums, st);
  };
  switch (a.act) {
    case kActRelu: return go(std::integral_constant<int, kActRelu>{});
    case kActGelu: return go(std::integral_constant<int, kActGelu>{});
    case kActSilu: return go(std::integral_constant<int, kActSilu>{});
    default: return go(std::integral_constant<int, kActNone>{});
  }
}

hipError_t launch_dense_bwd(const DenseArgs& a, hipStream_t st) {
  const int T = a.tokens, I = a.inputs, O = a.outputs, ldi = whole8(I), ldo = whole8(O);
  const bool makes = a.act != kActNone || a.drop.threshold;
  const Places at_ = places(T, I, O, true, makes);
  const h16 *x = a.x, *w = a.w, *dz = a.dy;
  h16* made = nullptr;
  if (makes || ldo != O) dz = made = at<h16>(a.ws, at_.dz);
  if (!a.dx && !a.dw) made = nullptr;
  if (made || a.dbias) {
    float* part = at<float>(a.ws, at_.part);
    switch (a.act) {
      case kActRelu: RUN(launch_dz<kActRelu>(a, ldo, made, part, st)); break;
      case kActGelu: RUN(launch_dz<kActGelu>(a, ldo, made, part, st)); break;
      case kActSilu: RUN(launch_dz<kActSilu>(a, ldo, made, part, st)); break;
      default: RUN(launch_dz<kActNone>(a, ldo, made, part, st));
    }
  }
  void* sums = at<void>(a.ws, at_.sums);
  if (ldi != I) {
    h16 *xs = at<h16>(a.ws, at_.x), *ws = at<h16>(a.ws, at_.w);
    RUN(launch_repack(I, {a.dw ? T : 0, a.x, xs}, {a.dx ? O : 0, a.w, ws}, st));
    x = xs;
    w = ws;
  }
  if (a.dx) {
    const Product p = {w, dz, ldi, ldo, I, T, O, 1};
    RUN(launch_product<kDx>(p, HalfEpi{a.dx, I, T}, sums, st));
  }
  if (a.dw) {
    const Product p = {x, dz, ldi, ldo, I, O, T, 1};
    RUN(launch_product<kDw>(p, HalfEpi{a.dw, I, O}, sums, st));
  }
  return hipSuccess;
}

}  // namespace fp16k
