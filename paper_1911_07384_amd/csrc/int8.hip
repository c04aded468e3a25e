// Dense layers in 8-bit integers: rows or columns of a binary16 matrix quantised
// with a scale each, and the product of two quantised operands.
//
//   s = max |x| / 127,  q = 127 x / max |x| to the nearest, ties to even;
//   y[i][j] = rne16(fl(sa[i] sb[j]) * (sum_k qa[i][k] qb[j][k]) + bias[j]).
//
// 127 x of a binary16 x is exact in float32 and the quotient is one float32
// division, within 2^-24 of the exact one.  Exact quotients differ from a halfway
// value by at least 2^-20 of it or not at all (254 x and (2k+1) max are integers
// below 2^20 on a common scale), so q is the exact quotient's rounding.  A zero row
// has s = 0 and q = 0; a row with an infinity or NaN has s = NaN, so every product
// with it is NaN.  The sums are exact: 32-bit integers, k <= 131071.

#include "gemm_nt.hpp"
#include "products.hpp"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace fp16k {
namespace {

// ---- quantising ------------------------------------------------------------------

// Magnitudes as bit patterns, which order as integers: an infinity is 0x7c00, a
// NaN above it, so that the maximum finds both.
__device__ __forceinline__ uint32_t i8_mag(uint32_t bits) { return bits & 0x7fffu; }
__device__ __forceinline__ uint32_t i8_mag8(const V8& v, uint32_t top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t m = i8_mag(v.s[e]);
    top = m > top ? m : top;
  }
  return top;
}
__device__ __forceinline__ float i8_top(uint32_t mag) {
  return to_f32(__builtin_bit_cast(h16, (uint16_t)mag));
}
__device__ __forceinline__ float i8_scale(uint32_t mag) {
  return mag >= 0x7c00u ? __builtin_nanf("") : i8_top(mag) / 127.0f;
}
// A row's (or column's) quantiser: the quotient t = 127 x / top as x * 127 * inv and
// one correction by its exact remainder, which leaves a halfway quotient exact and
// any other within 2^-24 of it (a division costs three times as many instructions);
// then t + 1.5 * 2^23, whose last byte is t to the nearest, ties to even.  inv = 0
// for a zero row and for one that is not finite, which makes every byte 0 (a NaN's
// last byte is 0 too).
struct I8Quant {
  float top, inv;
};
__device__ __forceinline__ I8Quant i8_quant(uint32_t mag) {
  const bool live = mag != 0 && mag < 0x7c00u;
  const float top = live ? i8_top(mag) : 0.0f;
  return I8Quant{top, live ? 1.0f / top : 0.0f};
}
// (x127: 127 x, exact)
__device__ __forceinline__ uint32_t i8_byte(float x127, const I8Quant& k) {
  const float t = x127 * k.inv;
  const float u = __builtin_fmaf(__builtin_fmaf(-t, k.top, x127), k.inv, t) + 12582912.0f;
  return __builtin_bit_cast(uint32_t, u);
}
__device__ __forceinline__ float i8_x127(h16 x) { return 127.0f * to_f32(x); }
// the last bytes of four words
__device__ __forceinline__ uint32_t i8_pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
  return lo | hi;
}

__device__ __forceinline__ uint32_t i8_wave_max(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, off, 64);
    v = o > v ? o : v;
  }
  return v;
}

// The maximum over the 32 lanes of a half wave, in every one of them, by register
// permutes alone (quads, eights, sixteens, then the two rows of 16).
template <int CTRL>
__device__ __forceinline__ uint32_t i8_max_dpp(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
  return o > v ? o : v;
}
__device__ __forceinline__ uint32_t i8_half_max(uint32_t v) {
  v = i8_max_dpp<0xB1>(v);   // lanes 1 0 3 2 of each quad
  v = i8_max_dpp<0x4E>(v);   // 2 3 0 1
  v = i8_max_dpp<0x141>(v);  // 7 .. 0 of each eight
  v = i8_max_dpp<0x140>(v);  // 15 .. 0 of each sixteen
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return r[0] > r[1] ? r[0] : r[1];
}

__device__ __forceinline__ uint2 i8_pack(const V8& v, const I8Quant& k) {
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = i8_byte(i8_x127(v.h[e]), k);
  return make_uint2(i8_pack4(b[0], b[1], b[2], b[3]), i8_pack4(b[4], b[5], b[6], b[7]));
}

// One workgroup a row; up to 8192 elements stay in registers between the maximum
// and the quantising, further ones are read again.  Bandwidth-bound: 3 bytes an
// element, 5.7 TB/s at 8192 x 4096 (17.6 us).
constexpr int kRowKeep = 4;
__global__ __launch_bounds__(256) void i8_rows(int cols, int ld, const h16* __restrict__ x,
                                               int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  const int tid = threadIdx.x;
  const h16* xr = x + (int64_t)blockIdx.x * cols;
  int8_t* qr = q + (int64_t)blockIdx.x * ld;
  V8 keep[kRowKeep];
  uint32_t mag = 0;
#pragma unroll
  for (int i = 0; i < kRowKeep; ++i) {
    const int c = (i * 256 + tid) * 8;
    keep[i] = load8_upto(xr + (c < cols ? c : 0), cols - c);
  }
#pragma unroll
  for (int i = 0; i < kRowKeep; ++i) mag = i8_mag8(keep[i], mag);
  for (int c = (kRowKeep * 256 + tid) * 8; c < cols; c += 2048)
    mag = i8_mag8(load8_upto(xr + c, cols - c), mag);
  mag = i8_wave_max(mag);
  if ((tid & 63) == 0) red[tid >> 6] = mag;
  __syncthreads();
  mag = std::max(std::max(red[0], red[1]), std::max(red[2], red[3]));
  if (tid == 0) scale[blockIdx.x] = i8_scale(mag);
  const I8Quant k = i8_quant(mag);
#pragma unroll
  for (int i = 0; i < kRowKeep; ++i) {
    const int c = (i * 256 + tid) * 8;
    if (c < ld) *reinterpret_cast<uint2*>(qr + c) = i8_pack(keep[i], k);
  }
  for (int c = (kRowKeep * 256 + tid) * 8; c < ld; c += 2048)
    *reinterpret_cast<uint2*>(qr + c) = i8_pack(load8_upto(xr + (c < cols ? c : 0), cols - c), k);
}

// Columns, or rows and columns, of up to two matrices (blockIdx.z) in two passes.
//
// First pass: 256 columns of a range of rows a workgroup, a thread 8 columns of
// every eighth row: the largest magnitude (and the sum) of each column over the
// range and, for the rows, of each row over the 256 columns.  Bandwidth-bound: two
// matrices of 4096 x 4096 at 4.8 TB/s (13.9 us).
constexpr int kColChunks = 32, kColRows = 32;  // ranges of rows at most, rows of one at least
__global__ __launch_bounds__(256) void i8_cols_max(const I8Both both) {
  const I8Cols& j = both.job[blockIdx.z];
  if ((int)blockIdx.x * 256 >= j.cols || (int)blockIdx.y >= j.chunks) return;
  __shared__ uint32_t rm[8][256];
  __shared__ float rs[8][256];
  const int tid = threadIdx.x, cg = tid & 31, rg = tid >> 5;
  const int c = blockIdx.x * 256 + cg * 8;
  const int r0 = blockIdx.y * j.per, r1 = std::min(j.rows, r0 + j.per);
  const bool want_rows = j.rmag != nullptr, want_sum = j.psum != nullptr;
  uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  constexpr int U = 4;
  // (whole: rows of whole vectors; one loop for both took 1 us more at 4096 x 4096)
  auto rows = [&](auto whole) {
    for (int r = r0 + rg; r < r1; r += 8 * U) {
      V8 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int ru = r + 8 * u;
        const h16* const row = j.x + (int64_t)(ru < r1 ? ru : r) * j.cols;
        if constexpr (decltype(whole)::value)
          v[u] = c < j.cols && ru < r1 ? load16u(row + c) : zero8();
        else
          v[u] = load8_row(row, c, j.cols, ru < r1);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t b = i8_mag(v[u].s[e]);
          m[e] = b > m[e] ? b : m[e];
          if (want_sum) s[e] += to_f32(v[u].h[e]);
        }
        if (want_rows) {
          const uint32_t top = i8_half_max(i8_mag8(v[u], 0));
          if (cg == 0 && r + 8 * u < r1) j.rmag[(int64_t)blockIdx.x * j.rows + r + 8 * u] = top;
        }
      }
    }
  };
  if (j.cols & 7)
    rows(std::false_type{});
  else
    rows(std::true_type{});
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    rm[rg][cg * 8 + e] = m[e];
    rs[rg][cg * 8 + e] = s[e];
  }
  __syncthreads();
  const int cc = blockIdx.x * 256 + tid;
  if (cc >= j.cols) return;
  uint32_t a = 0;
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a = rm[i][tid] > a ? rm[i][tid] : a;
    t += rs[i][tid];
  }
  j.cmag[(int64_t)blockIdx.y * j.cols + cc] = a;
  if (want_sum) j.psum[(int64_t)blockIdx.y * j.cols + cc] = t;
}

// Second pass: T rows x T columns quantised and written transposed, a run of T bytes
// of each column through LDS, and as laid out, a run of each row.  T = 128 writes
// whole lines (two matrices of 4096 x 4096, one by rows too: 117 MB in 22 us, 5.3
// TB/s); T = 64 has four times the workgroups for small matrices (128 x 1000 and
// 128 x 2048: 6.3 us, 9.0 on T = 128).
template <int T>
__global__ __launch_bounds__(256) void i8_cols_write(const I8Both both) {
  const I8Cols& j = both.job[blockIdx.z];
  const int c0 = blockIdx.x * T, r0 = blockIdx.y * T;
  if (c0 >= j.ldr || r0 >= j.ldc) return;
  constexpr int LD = T + 16;             // bytes from column to column of the tile
  constexpr int CG = T / 8, R = T * T / 2048;  // groups of 8 columns; rows a thread
  __shared__ I8Quant cq[T], rq[T];
  __shared__ __attribute__((aligned(16))) int8_t tile[T * LD];
  const int tid = threadIdx.x;
  const bool want_rows = j.rmag != nullptr;
  const int cg = tid % CG, rg = tid / CG;  // columns 8 cg .. + 7, rows R rg .. + R - 1
  const int c = c0 + cg * 8;
  V8 v[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = r0 + rg * R + i;
    v[i] = load8_row(j.x + (int64_t)(r < j.rows ? r : 0) * j.cols, c, j.cols, r < j.rows);
  }
  if (tid < T) {
    const int k = c0 + tid;
    uint32_t a = 0;
    double s = 0.0;
    if (k < j.cols) {
#pragma unroll 16
      for (int i = 0; i < j.chunks; ++i) {
        const uint32_t b = j.cmag[(int64_t)i * j.cols + k];
        a = b > a ? b : a;
      }
      if (blockIdx.y == 0) {
        j.scale_c[k] = i8_scale(a);
        if (j.psum) {
          for (int i = 0; i < j.chunks; ++i) s += (double)j.psum[(int64_t)i * j.cols + k];
          j.sum[k] = dbl_to_h16(s);
        }
      }
    }
    cq[tid] = i8_quant(a);
  } else if (want_rows && tid < 2 * T) {
    const int k = r0 + tid - T;
    uint32_t a = 0;
    if (k < j.rows) {
      const int n = (j.cols + 255) / 256;
#pragma unroll 16
      for (int i = 0; i < n; ++i) {
        const uint32_t b = j.rmag[(int64_t)i * j.rows + k];
        a = b > a ? b : a;
      }
      if (blockIdx.x == 0) j.scale_r[k] = i8_scale(a);
    }
    rq[tid - T] = i8_quant(a);
  }
  __syncthreads();
  if (want_rows) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = r0 + rg * R + i;
      if (r < j.rows && c < j.ldr)
        *reinterpret_cast<uint2*>(j.qr + (int64_t)r * j.ldr + c) = i8_pack(v[i], rq[rg * R + i]);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const I8Quant k = cq[cg * 8 + e];
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = i < R ? i8_byte(i8_x127(v[i < R ? i : 0].h[e]), k) : 0u;
    // (16-byte chunks exclusive-ored with the columns' group: a lane's columns lie 8
    // lines from its neighbour's)
    const int at = rg * R;
    int8_t* to = tile + (cg * 8 + e) * LD + ((at / 16) ^ (cg % (T / 16))) * 16 + at % 16;
    const uint32_t w = i8_pack4(b[0], b[1], b[2], b[3]);
    if (R == 8)
      *reinterpret_cast<uint2*>(to) = make_uint2(w, i8_pack4(b[4], b[5], b[6], b[7]));
    else
      *reinterpret_cast<uint16_t*>(to) = (uint16_t)w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < T * T / 4096; ++i) {
    const int cc = (i * 256 + tid) / (T / 16), k = (i * 256 + tid) % (T / 16) * 16;
    if (c0 + cc < j.cols && r0 + k < j.ldc)
      *reinterpret_cast<u32x4*>(j.qc + (int64_t)(c0 + cc) * j.ldc + r0 + k) =
          *reinterpret_cast<const u32x4*>(tile + cc * LD + ((k / 16) ^ (cc / 8 % (T / 16))) * 16);
  }
}

// ---- the product --------------------------------------------------------------------

// fl(sa sb) * sum + bias, the sum rounded to float32 first
__device__ __forceinline__ h16 i8_out(int acc, float sa, float sb, bool has_bias, float bias) {
  const float v = (sa * sb) * (float)acc;
  return to_h16(has_bias ? v + bias : v);
}

// What a tile stores, see nt_store: p along a row of y.
struct I8Epi {
  const I8Product& g;
  bool has_bias;
  static constexpr int OUTS = 1;
  static constexpr bool DIAGONAL = false;
  struct Pre {
    float sq, sp[8];
    V8 bp;
  };

  __device__ __forceinline__ Pre load(int p, int q) const {
    Pre r;
    r.sq = g.sa[q < g.m ? q : 0];
    p = p < g.n ? p : 0;
    if (p + 8 <= g.n) {
      const floatx4* sv = reinterpret_cast<const floatx4*>(g.sb + p);
      const floatx4 x = sv[0], y = sv[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        r.sp[k] = x[k];
        r.sp[4 + k] = y[k];
      }
      if (has_bias) r.bp = load16(g.bias + p);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = p + k < g.n ? p + k : 0;
        r.sp[k] = g.sb[i];
        if (has_bias) r.bp.h[k] = g.bias[i];
      }
    }
    return r;
  }
  __device__ __forceinline__ void compute(int, int, const int (&v)[8], const Pre& pre,
                                          V8 (&out)[1]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      out[0].h[k] = i8_out(v[k], pre.sq, pre.sp[k], has_bias, to_f32(pre.bp.h[k]));
  }
  __device__ __forceinline__ void store(int p, int q, const V8 (&out)[1]) const {
    if (p >= g.n || q >= g.m) return;
    store8_upto(g.y + (int64_t)q * g.n + p, out[0], g.n - p);
  }
};

// Tile rows p are rows of b (outputs), q rows of a (tokens).
template <class C>
__global__ __launch_bounds__(C::THREADS, C::OCC) void i8_product(const I8Product g, int tp, int tq) {
  __shared__ __attribute__((aligned(1024))) char lds[NtEpi<C, 1>::LDS];
  const int t = nt_xcd(blockIdx.x, tp * tq);
  if (t >= tp * tq) return;
  const int gr = t / (4 * tq), w = t - gr * 4 * tq;
  const int gw = tp - 4 * gr < 4 ? tp - 4 * gr : 4;
  const int pt = (4 * gr + w % gw) * C::BP, qt = (w / gw) * C::BQ;
  NtTile nt;
  nt.ldp = nt.ldq = (uint32_t)((g.k + 15) & ~15);
  nt.p[0] = nt.p[1] = g.b + (int64_t)pt * nt.ldp;
  nt.q[0] = nt.q[1] = g.a + (int64_t)qt * nt.ldq;
  nt.prows = g.n - pt;
  nt.qrows = g.m - qt;
  nt.kbytes = g.k;
  nt.part = 0;
  nt.parts = 1;
  intx16 acc[C::TP][C::TQ];
  nt_product<NtByte, C>(nt, lds, acc);
  const int wave = threadIdx.x >> 6;
  const I8Epi epi{g, g.bias != nullptr};
  h16* none[1] = {nullptr};
  nt_store<C, 1>(acc, lds, pt + (wave / C::WQ) * 32 * C::TP, qt + (wave % C::WQ) * 32 * C::TQ, g.n,
                 g.m, false, none, 0, epi);
}

// Few rows (at most 16 tokens): bound by reading b once.  A workgroup takes 16
// outputs; its eight waves split the reduction, each lane loading 16 bytes of one
// row of b straight into the operand (the first kFewAhead of them before anything
// else), and add their 32-bit sums in LDS.  One token, 4096 x 4096: 5.0 us, 3.4 TB/s.
// Up to two workgroups a CU: past them every one reads a again, and the 64 x 64 tiles
// are faster.  Product alone, few rows / tiles of 64, in us, of 1 and of 16 tokens:
//     n x k       1000 x 2048   4096 x 4096   8192 x 4096   16384 x 1024   16384 x 4096
//     1             3.3/5.9       5.0/9.0       7.1/9.4        4.7/4.5       14.5/12.2
//     16            3.8/6.0       5.8/9.0       9.6/9.6        5.7/4.6       18.4/12.4
//
// FUSED: the rows of x are quantised by every workgroup for itself into LDS (they are
// small and come from the L2), which saves a launch; that pays for up to 4 tokens of
// 16384 elements together.  One launch / two, in us:
//     n x k         1000 x 2048   2048 x 8192   4096 x 4096   8192 x 4096
//     1 token         4.2/6.1       8.2/10.8      5.7/7.8       7.7/9.9
//     2               4.6/6.1       9.5/10.9      6.4/8.1       8.7/10.1
//     4               4.8/6.1      11.7/11.1      7.5/8.2      10.3/10.4
//     12              7.8/6.4         -          13.7/8.4         -
constexpr int kFewRows = 16, kFewOut = 16, kFewWaves = 8, kFewAhead = 8, kFewGroups = 512;
constexpr int kFusedRows = 4, kFusedElems = 16384;
template <bool FUSED>
__global__ __launch_bounds__(64 * kFewWaves) void i8_few(const I8Product g, const h16* __restrict__ x) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];  // FUSED: [m][ld + 16]
  __shared__ int part[kFewWaves][16][17];
  __shared__ uint32_t top[kFusedRows][kFewWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ld = (g.k + 15) & ~15, lq = ld + 16;
  const int n0 = blockIdx.x * kFewOut;
  const int row = lane & 15, kc = (lane >> 4) * 16;
  const bool ain = row < g.m;
  const int8_t* bp = g.b + (int64_t)(n0 + row < g.n ? n0 + row : 0) * ld;
  const intx4 zero = {0, 0, 0, 0};
  const int steps = (ld + 63) / 64, per = (steps + kFewWaves - 1) / kFewWaves;
  const int s0 = wave * per, s1 = std::min(steps, s0 + per);
  intx4 fb[kFewAhead];
  auto load = [&](int s) {
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int k = (s + u) * 64 + kc;
      fb[u] = s + u < s1 && k < ld ? *reinterpret_cast<const intx4*>(bp + k) : zero;
    }
  };
  load(s0);
  const int wpr = kFewWaves / (g.m >= 3 ? 4 : g.m);  // waves to a row of x
  if (FUSED) {
    const int w = wave % wpr, r = wave / wpr;
    const h16* xr = x + (int64_t)r * g.k;
    if (r < g.m) {
      uint32_t mag = 0;
      for (int c = (w * 64 + lane) * 8; c < g.k; c += 512 * wpr)
        mag = i8_mag8(load8_upto(xr + c, g.k - c), mag);
      mag = i8_wave_max(mag);
      if (lane == 0) top[r][w] = mag;
    }
    __syncthreads();
    if (r < g.m) {
      uint32_t mag = 0;
      for (int i = 0; i < wpr; ++i) mag = std::max(mag, top[r][i]);
      const I8Quant k = i8_quant(mag);
      for (int c = (w * 64 + lane) * 8; c < ld; c += 512 * wpr)
        *reinterpret_cast<uint2*>(dyn + r * lq + c) =
            i8_pack(load8_upto(xr + (c < g.k ? c : 0), g.k - c), k);
    }
    __syncthreads();
  }
  intx4 acc = zero;
  for (int s = s0; s < s1; s += kFewAhead) {
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u) {
      const int k = (s + u) * 64 + kc;
      const bool in = s + u < s1 && ain && k < ld;
      const char* from = FUSED ? dyn + row * lq + k
                               : reinterpret_cast<const char*>(g.a) + (int64_t)row * ld + k;
      const intx4 fa = in ? *reinterpret_cast<const intx4*>(from) : zero;
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u], fa, acc, 0, 0, 0);
    }
    if (s + kFewAhead < s1) load(s + kFewAhead);
  }
  // lane: outputs 4 (lane / 16) + i of token lane % 16
#pragma unroll
  for (int i = 0; i < 4; ++i) part[wave][row][4 * (lane >> 4) + i] = acc[i];
  __syncthreads();
  if (tid < 256) {
    const int q = tid >> 4, p = tid & 15;
    if (q < g.m && n0 + p < g.n) {
      int s = 0;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) s += part[w][q][p];
      float sq;
      if (FUSED) {
        uint32_t mag = 0;
        for (int i = 0; i < wpr; ++i) mag = std::max(mag, top[q][i]);
        sq = i8_scale(mag);
      } else {
        sq = g.sa[q];
      }
      const bool has_bias = g.bias != nullptr;
      g.y[(int64_t)q * g.n + n0 + p] =
          i8_out(s, sq, g.sb[n0 + p], has_bias, has_bias ? to_f32(g.bias[n0 + p]) : 0.0f);
    }
  }
}

template <class C>
hipError_t i8_launch(const I8Product& a, hipStream_t st) {
  const int tp = ceil_div(a.n, C::BP), tq = ceil_div(a.m, C::BQ);
  const int64_t n = (int64_t)tp * tq;
  hipLaunchKernelGGL((i8_product<C>), dim3((unsigned)(8 * ((n + 7) / 8))), dim3(C::THREADS), 0, st,
                     a, tp, tq);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_rows(int rows, int cols, const h16* x, int8_t* q, float* scale,
                          hipStream_t st) {
  hipLaunchKernelGGL(i8_rows, dim3((unsigned)rows), dim3(256), 0, st, cols, (int)i8_row(cols), x, q,
                     scale);
  return hipGetLastError();
}

void i8_cols_plan(I8Cols* j) {
  j->per = std::max(kColRows, ceil_div(ceil_div(j->rows, kColChunks), 32) * 32);
  j->chunks = ceil_div(j->rows, j->per);
  j->ldc = (int)i8_row(j->rows);
  j->ldr = (int)i8_row(j->cols);
}

size_t i8_cols_ws_bytes(int rows, int cols, bool by_rows, bool sum) {
  I8Cols j{};
  j.rows = rows;
  j.cols = cols;
  i8_cols_plan(&j);
  return (size_t)j.chunks * cols * (sum ? 8 : 4) +
         (by_rows ? (size_t)ceil_div(cols, 256) * rows * 4 : 0);
}

I8Cols i8_cols_job(int rows, int cols, const h16* x, int8_t* qc, float* scale_c, int8_t* qr,
                   float* scale_r, h16* sum, void* ws) {
  I8Cols j{};
  j.rows = rows;
  j.cols = cols;
  j.x = x;
  i8_cols_plan(&j);
  j.qc = qc;
  j.scale_c = scale_c;
  j.qr = qr;
  j.scale_r = scale_r;
  j.sum = sum;
  j.cmag = static_cast<uint32_t*>(ws);
  uint32_t* next = j.cmag + (size_t)j.chunks * cols;
  if (sum) {
    j.psum = reinterpret_cast<float*>(next);
    next += (size_t)j.chunks * cols;
  }
  if (qr) j.rmag = next;
  return j;
}

hipError_t launch_i8_cols(const I8Cols* jobs, int count, hipStream_t st) {
  I8Both b{};
  int cols = 0, chunks = 0, rows = 0;
  for (int i = 0; i < count; ++i) {
    b.job[i] = jobs[i];
    cols = std::max(cols, jobs[i].ldr);
    rows = std::max(rows, jobs[i].ldc);
    chunks = std::max(chunks, jobs[i].chunks);
  }
  hipLaunchKernelGGL(i8_cols_max, dim3((unsigned)ceil_div(cols, 256), (unsigned)chunks, (unsigned)count),
                     dim3(256), 0, st, b);
  const bool small = (int64_t)ceil_div(cols, 128) * ceil_div(rows, 128) * count < 512;
  const int t = small ? 64 : 128;
  const dim3 grid((unsigned)ceil_div(cols, t), (unsigned)ceil_div(rows, t), (unsigned)count);
  if (small)
    hipLaunchKernelGGL(i8_cols_write<64>, grid, dim3(256), 0, st, b);
  else
    hipLaunchKernelGGL(i8_cols_write<128>, grid, dim3(256), 0, st, b);
  return hipGetLastError();
}

bool i8_fused_ok(int m, int n, int k) {
  return m <= kFusedRows && (int64_t)m * k <= kFusedElems &&
         ceil_div(n, kFewOut) <= kFewGroups;
}

hipError_t launch_i8_fused(const I8Product& a, const h16* x, hipStream_t st) {
  const size_t lds = (size_t)a.m * (i8_row(a.k) + 16);
  hipLaunchKernelGGL((i8_few<true>), dim3((unsigned)ceil_div(a.n, kFewOut)), dim3(64 * kFewWaves), lds,
                     st, a, x);
  return hipGetLastError();
}

namespace {
// The square tiles of a product: workgroups a CU holds; microseconds that a
// 128-byte slice of the reduction takes one workgroup alone, and a CU for each
// workgroup it holds, that a launch takes besides, and every round of workgroups.
// Fitted to 22 sizes; the times below (in us) are met within 8 % but for 2048 x 4096 x
// 4096 on 256 (15 % low), 2048^3 on 128 (14 % low) and 128 x 1000 x 2048 on 128 (11 %
// high), none of which the choice takes:
//   m x n x k               256    128  128 deep     64
//   8192 x 4096 x 4096      129    147       168    229
//   2048 x 2048 x 2048       30     18        15     22
//   2048 x 4096 x 4096       53     38        45     60
//   128 x 1000 x 2048        27     14        12      8
//   8192 x 8192 x 300        67     72       113    113
struct I8Tile {
  int side, occ;
  double alone, cu, launch, round;
  const char* name;
};
constexpr int kI8Kinds = 4;
constexpr I8Tile kI8Tiles[kI8Kinds + 1] = {{256, 1, 1.02, 1.72, 1.5, 11.1, "tile 256"},
                                           {128, 2, 0.56, 0.50, 0.0, 6.6, "tile 128"},
                                           {128, 1, 0.33, 0.51, 1.7, 5.3, "tile 128 deep"},
                                           {64, 2, 0.18, 0.20, 2.7, 2.4, "tile 64"},
                                           {0, 0, 0.0, 0.0, 0.0, 0.0, "few rows"}};

// The one that finishes soonest by that estimate, or few rows (see i8_few).
int i8_tile(int m, int n, int k) {
  if (m <= kFewRows && ceil_div(n, kFewOut) <= kFewGroups) return kI8Kinds;
  int best = 0;
  double bt = 0;
  for (int i = 0; i < kI8Kinds; ++i) {
    const I8Tile& c = kI8Tiles[i];
    const double tiles = (double)ceil_div(n, c.side) * ceil_div(m, c.side), full = 256.0 * c.occ;
    const double rounds = ceil(tiles / full), rest = (tiles - (rounds - 1) * full) / 256.0;
    const double t = c.launch + rounds * c.round +
                     ceil_div(k, 128) * ((rounds - 1) * c.cu * c.occ + std::max(c.alone, c.cu * rest));
    if (i == 0 || t < bt) {
      bt = t;
      best = i;
    }
  }
  return best;
}
}  // namespace

const char* i8_product_name(int m, int n, int k) { return kI8Tiles[i8_tile(m, n, k)].name; }

hipError_t launch_i8_product(const I8Product& a, hipStream_t st) {
  switch (i8_tile(a.m, a.n, a.k)) {
    case 0: return i8_launch<Nt256>(a, st);
    case 1: return i8_launch<Nt128>(a, st);
    case 2: return i8_launch<Nt128d>(a, st);
    case 3: return i8_launch<Nt64>(a, st);
  }
  hipLaunchKernelGGL((i8_few<false>), dim3((unsigned)ceil_div(a.n, kFewOut)), dim3(64 * kFewWaves), 0, st,
                     a, (const h16*)nullptr);
  return hipGetLastError();
}

}  // namespace fp16k
