// Orthogonalised momentum (the Muon update) on binary16 weights, gradients and
// momentum, and the orthogonalisation alone, for a set of matrices at once.
//
// With u = mu m' + g (or m'), m' = rne16(mu m + g), X = u / ||u||_F taken over its
// shorter side m (n the longer), each step is
//   A = X X^T,  B = bA + cA^2,  X <- aX + BX,
// three products of 2 m^2 n, 2 m^3 and 2 m^2 n operations, the first two symmetric:
// only tiles on and below the diagonal are computed and each is stored twice.
//
// Numbers.  The matrix cores multiply binary16, so A, B and X are rounded to
// binary16 as operands; everything else stays in float32:
//  - X is kept as a sum of two binary16 values, X = Xh + Xl (22 bits): early steps
//    multiply what the last rounding lost in the directions of small singular
//    values by a (3.4 each step) along with X itself;
//  - the diagonals of A and B are kept in float32 and the operands hold 0 there:
//    X' = (a + E) X + B'X with B = diag(E) + B'.  For rows that are nearly
//    orthogonal all diagonal entries are nearly equal and round the same way, an
//    error of one sign in every singular value;
//  - products = 1 takes the high parts as operands.  E multiplies Xh only, as the
//    rest of B does: with E (Xh + Xl) the small directions would get E Xl without
//    the -E Xl that B'Xl takes away from them.  Relative error of the result (2-norm,
//    against float64, five steps): 3e-4 to 2e-3 for matrices whose entries round
//    independently; entries of one magnitude round alike, and off the diagonal that
//    error of one sign remains: 1e-2 for a constant matrix of 1000 x 2048 (89 x 92:
//    9e-3, equal rows of 8 x 8: 4e-3);
//  - products = 3 takes every operand as high + low part, three products for one
//    (the product of the low parts is below 2^-22): 5e-7 to 4e-6 for independent
//    entries, 5e-5 for the constant matrix.  Directions of zero singular values take a
//    times the last step's errors each step, and at 22 bits the float32 sums': 2.5e-4
//    for a matrix of rank one, 2500 x 4096.
// Operands carry powers of two (X 2^12, A 2^12, B 2^11) that keep binary16 normal:
// entries of X are near 1/sqrt(mn) at first.  They leave room for |X| < 16 and
// |B| < 32 (the default coefficients reach 1.3 and 8).
//
// Split: one grid covers the tiles of every matrix of the set, one kernel each for
// A, B and X', so a step is three launches however many matrices there are; which
// matrix a tile belongs to is looked up in a map that the first launch writes.  X is
// kept as laid out and transposed, since A reduces over its columns and X' over its
// rows, both as operands with the reduction contiguous; a tile is written one way
// from registers and the other through LDS.  The last X' updates the weights itself.

#include "gemm_nt.hpp"
#include "products.hpp"

#include <math.h>

#include <algorithm>

namespace fp16k {
namespace {

// The tiles by the number of products: with three, the parts of both operands lie
// in LDS together, so slices are half as long.
template <int PROD>
struct NsTiles {
  typedef Nt256 T256;
  typedef Nt192 T192;
  typedef Nt128 T128;
  typedef Nt128d T128d;
  typedef Nt64 T64;
  typedef NtCfg<2, 2, 1, 1, 128, 8, 1> T64d;
};
template <>
struct NsTiles<3> {
  typedef NtCfg<2, 2, 4, 4, 64, 2, 1, 2> T256;
  typedef NtCfg<2, 2, 3, 3, 64, 3, 1, 2> T192;
  typedef NtCfg<2, 2, 2, 2, 64, 2, 2, 2> T128;
  typedef NtCfg<2, 2, 2, 2, 64, 4, 1, 2> T128d;
  typedef NtCfg<2, 2, 1, 1, 128, 2, 2, 2> T64;
  typedef NtCfg<2, 2, 1, 1, 128, 4, 1, 2> T64d;
};

constexpr float kSx = 4096.0f, kSa = 4096.0f, kSb = 2048.0f;

struct NsDev {
  char* ws;
  uint32_t table, map, sums;  // in units of 256 bytes
  int tiles;
  int single;  // one matrix only
};

template <class T>
__device__ __forceinline__ T* at(char* ws, uint32_t place) {
  return reinterpret_cast<T*>(ws + (size_t)place * 256);
}

// Tiles of one matrix in a launch for A (stage 0), B (1) or X' (2).
__host__ __device__ inline int ns_tiles(const NsJob& j, int stage, int side) {
  const int tr = (j.rp + side - 1) / side, tc = (j.cp + side - 1) / side;
  const int tm = j.tall ? tc : tr;
  return stage == 2 ? tr * tc : tm * (tm + 1) / 2;
}

// ---- pass 1: momentum, squares, and the table ---------------------------------

constexpr int kJobsPerLaunch = 24;
struct NsChunk {
  NsJob job[kJobsPerLaunch];
};
static_assert(sizeof(NsChunk) <= 3584, "kernel arguments");

struct NsPlaces {
  uint32_t table, map[3], map_pre;
  int side[3];
};

__device__ __forceinline__ double ns_block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((red[0] + red[1]) + red[2]) + red[3];
}

// The factor of X from the sum of squares: 0 for a zero matrix (no epsilon, since
// gradients trained without loss scaling are small), not a number where an element
// is not finite.
__device__ __forceinline__ float ns_rsqrt(double s) {
  if (s > 0.0 && s < __builtin_inf()) return (float)((double)kSx / sqrt(s));
  return s == 0.0 ? 0.0f : __builtin_nanf("");
}

// the float32 update direction before normalisation
__device__ __forceinline__ float ns_dir(h16 g, h16 m, float mu, bool has_m, bool nesterov) {
  if (!has_m) return to_f32(g);
  return nesterov ? __builtin_fmaf(mu, to_f32(m), to_f32(g)) : to_f32(m);
}

// Reads g and m, writes m' and this block's sum of squares of u (float64); block 0
// of a matrix also writes its entry of the table and its part of the maps.
// Bandwidth-bound: 6 bytes an element, 3.6 TB/s at 4096 x 4096 (28 us).
__global__ __launch_bounds__(256) void ns_first(const NsChunk c, char* ws, NsPlaces pl, int first,
                                                float mu, int nesterov) {
  __shared__ double red[4];
  const NsJob& j = c.job[blockIdx.y];
  if ((int)blockIdx.x >= j.nparts) return;
  const int tid = threadIdx.x;
  if (blockIdx.x == 0) {
    const int idx = first + blockIdx.y;
    if (tid == 0) at<NsJob>(ws, pl.table)[idx] = j;
    for (int stage = 0; stage < 3; ++stage) {
      const int n = ns_tiles(j, stage, pl.side[stage]);
      uint16_t* const map = at<uint16_t>(ws, pl.map[stage]) + j.t[stage];
      for (int i = tid; i < n; i += 256) map[i] = (uint16_t)idx;
    }
    const int npre = (j.rp / 64) * (j.cp / 64);
    for (int i = tid; i < npre; i += 256) at<uint16_t>(ws, pl.map_pre)[j.t_pre + i] = (uint16_t)idx;
  }
  const bool has_m = j.m != nullptr;
  const int64_t n = (int64_t)j.rows * j.cols, nvec = n / 8;
  double s = 0.0;
  constexpr int U = 4;
  const int64_t step = (int64_t)j.nparts * 256;
  for (int64_t i0 = (int64_t)blockIdx.x * 256 + tid; i0 < nvec; i0 += U * step) {
    V8 g[U], m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * step;
      g[u] = i < nvec ? load16u(j.g + i * 8) : zero8();
      m[u] = has_m && i < nvec ? load16u(j.m + i * 8) : zero8();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * step;
      if (has_m) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          m[u].h[e] = to_h16(__builtin_fmaf(mu, to_f32(m[u].h[e]), to_f32(g[u].h[e])));
        if (i < nvec) store16u(j.m + i * 8, m[u]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double x = (double)ns_dir(g[u].h[e], m[u].h[e], mu, has_m, nesterov);
        s = __builtin_fma(x, x, s);
      }
    }
  }
  if (blockIdx.x == 0 && tid < n - nvec * 8) {  // the last elements
    const int64_t i = nvec * 8 + tid;
    h16 m = 0;
    if (has_m) {
      m = to_h16(__builtin_fmaf(mu, to_f32(j.m[i]), to_f32(j.g[i])));
      j.m[i] = m;
    }
    const double u = (double)ns_dir(j.g[i], m, mu, has_m, nesterov);
    s = __builtin_fma(u, u, s);
  }
  s = ns_block_sum(s, red);
  if (tid == 0) at<double>(ws, j.part)[blockIdx.x] = s;
}

// The matrix that tile t of the launch belongs to (without a look at the map, a
// dependent read, where there is only one).
__device__ __forceinline__ const NsJob& ns_job(const NsDev& dv, int t) {
  return at<NsJob>(dv.ws, dv.table)[dv.single ? 0 : at<uint16_t>(dv.ws, dv.map)[t]];
}

// ---- pass 2: X = u / ||u|| split in two binary16 parts, both ways round --------
//
// Bandwidth-bound: 10 bytes an element (12 with three products), 5.5 TB/s at
// 4096 x 4096 (30 us).
template <int PROD>
__global__ __launch_bounds__(256) void ns_split(const NsDev dv, float mu, int nesterov) {
  constexpr int LD = 64;
  __shared__ double red[4];
  __shared__ __attribute__((aligned(16))) h16 tile[PROD == 3 ? 2 : 1][64 * LD];
  const NsJob& j = ns_job(dv, blockIdx.x);
  const int tid = threadIdx.x;
  double s = 0.0;
  for (int i = tid; i < j.nparts; i += 256) s += at<double>(dv.ws, j.part)[i];
  s = ns_block_sum(s, red);
  const float rs = ns_rsqrt(s);
  const int local = blockIdx.x - j.t_pre, tc = j.cp / 64;
  const int r0 = (local / tc) * 64, c0 = (local % tc) * 64;
  const bool has_m = j.m != nullptr;
  // thread: 8 columns of rows tid / 8 and tid / 8 + 32; 8 threads a row's 128 bytes.
  // Transposed through LDS, the 8-row chunks of a column exclusive-ored with the
  // column's chunk.
  const int cg = tid & 7, col = c0 + cg * 8;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int rl = tid / 8 + 32 * v, row = r0 + rl;
    V8 g = zero8(), m = zero8(), hi, lo;
    const int64_t o = (int64_t)row * j.cols + col;
    if (row < j.rows && col < j.cols) {
      g = load8_upto(j.g + o, j.cols - col);
      if (has_m) m = load8_upto(j.m + o, j.cols - col);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = ns_dir(g.h[e], m.h[e], mu, has_m, nesterov);
      const float x = row < j.rows && col + e < j.cols ? u * rs : 0.0f;
      hi.h[e] = to_h16(x);
      lo.h[e] = to_h16(x - to_f32(hi.h[e]));
      const int to = (cg * 8 + e) * LD + ((rl / 8) ^ cg) * 8 + rl % 8;
      tile[0][to] = hi.h[e];
      if (PROD == 3) tile[PROD == 3][to] = lo.h[e];
    }
    store16(at<h16>(dv.ws, j.nat[0]) + (int64_t)row * j.cp + col, hi);
    store16(at<h16>(dv.ws, j.natl[0]) + (int64_t)row * j.cp + col, lo);
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int cl = tid / 8 + 32 * v, k = tid & 7;
    const int from = cl * LD + (k ^ (cl / 8)) * 8;
    const int64_t mo = (int64_t)(c0 + cl) * j.rp + r0 + k * 8;
    store16(at<h16>(dv.ws, j.mir[0]) + mo, load16(&tile[0][from]));
    if (PROD == 3) store16(at<h16>(dv.ws, j.mirl[0]) + mo, load16(&tile[PROD == 3][from]));
  }
}

// ---- the three products of a step -----------------------------------------------


// tile t of a lower triangle, rows in order
__device__ __forceinline__ void ns_triangle(int t, int* i, int* j) {
  int r = (int)((__builtin_sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while (r * (r + 1) / 2 > t) --r;
  while ((r + 1) * (r + 2) / 2 <= t) ++r;
  *i = r;
  *j = t - r * (r + 1) / 2;
}

// What a tile of A (STEP 0) or B (STEP 1) stores, see nt_store.
template <int STEP, int PARTS>
struct NsSymEpi {
  int m;
  const h16 *ah, *al;  // A, for B
  h16 *oh, *ol;
  float *d, *e;
  float cb, cc;
  static constexpr int OUTS = PARTS;
  static constexpr bool DIAGONAL = true;
  struct Pre {
    V8 a[STEP == 1 ? PARTS : 1];
    float dp[8], dq;
  };

  __device__ __forceinline__ Pre load(int p, int q) const {
    Pre r;
    if (STEP == 1) {
      p = p < m ? p : 0;
      q = q < m ? q : 0;
      const int64_t o = (int64_t)q * m + p;
      r.a[0] = load16(ah + o);
      if (PARTS == 2) r.a[PARTS - 1] = load16(al + o);
      r.dq = d[q];
      const floatx4* dv = reinterpret_cast<const floatx4*>(d + p);
      const floatx4 x = dv[0], y = dv[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        r.dp[k] = x[k];
        r.dp[4 + k] = y[k];
      }
    }
    return r;
  }
  __device__ __forceinline__ void compute(int p, int q, const float (&f)[8], const Pre& pre,
                                          V8 (&out)[PARTS]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float r;
      if (STEP == 0) {
        r = f[k] * (kSa / (kSx * kSx));
      } else {
        float a = to_f32(pre.a[0].h[k]);
        if (PARTS == 2) a += to_f32(pre.a[PARTS - 1].h[k]);
        a *= 1.0f / kSa;
        const float a2 = f[k] * (1.0f / (kSa * kSa));
        r = kSb * __builtin_fmaf(cc, __builtin_fmaf(pre.dq + pre.dp[k], a, a2), cb * a);
      }
      if (p + k == q) r = 0.0f;
      out[0].h[k] = to_h16(r);
      if (PARTS == 2) out[PARTS - 1].h[k] = to_h16(r - to_f32(out[0].h[k]));
    }
  }
  __device__ __forceinline__ void store(int p, int q, const V8 (&out)[PARTS]) const {
    if (p >= m || q >= m) return;
    const int64_t o = (int64_t)q * m + p;
    store16(oh + o, out[0]);
    if (PARTS == 2) store16(ol + o, out[PARTS - 1]);
  }
  __device__ __forceinline__ void diagonal(int q, float v) const {
    if (q >= m) return;
    if (STEP == 0) {
      d[q] = v * (1.0f / (kSx * kSx));
    } else {
      const float dq = d[q];
      e[q] = __builtin_fmaf(cc, __builtin_fmaf(dq, dq, v * (1.0f / (kSa * kSa))), cb * dq);
    }
  }
};

// The operands of one tile of A or B.
template <int STEP>
__device__ __forceinline__ void ns_sym_tile(const NsDev& dv, const NsJob& j, int pt, int qt,
                                            NtTile* nt) {
  const int m = j.tall ? j.cp : j.rp, n = j.tall ? j.rp : j.cp;
  // X as [m][n]: laid out so, or the transpose of a tall matrix
  const h16* hi = at<h16>(dv.ws, STEP == 1 ? j.a : j.tall ? j.mir[0] : j.nat[0]);
  const h16* lo = at<h16>(dv.ws, STEP == 1 ? j.al : j.tall ? j.mirl[0] : j.natl[0]);
  const int k = STEP == 0 ? n : m;
  const int64_t po = (int64_t)pt * k, qo = (int64_t)qt * k;
  nt->p[0] = hi + po;
  nt->q[0] = hi + qo;
  nt->p[1] = lo + po;
  nt->q[1] = lo + qo;
  nt->ldp = nt->ldq = (uint32_t)k * 2u;
  nt->prows = m - pt;
  nt->qrows = m - qt;
  nt->kbytes = k * 2;
}

// Stores a tile of A or B at rows p0, q0 (those of this wave).
template <class C, int STEP, int PROD>
__device__ __forceinline__ void ns_sym_out(const NsDev& dv, const NsJob& j, float cb, float cc,
                                           const floatx16 (&acc)[C::TP][C::TQ], char* lds, int p0,
                                           int q0, bool mirror) {
  constexpr int PARTS = PROD == 3 ? 2 : 1;
  const int m = j.tall ? j.cp : j.rp;
  NsSymEpi<STEP, PARTS> epi;
  epi.m = m;
  epi.ah = at<h16>(dv.ws, j.a);
  epi.al = at<h16>(dv.ws, j.al);
  epi.oh = at<h16>(dv.ws, STEP == 0 ? j.a : j.b);
  epi.ol = at<h16>(dv.ws, STEP == 0 ? j.al : j.bl);
  epi.d = at<float>(dv.ws, j.d);
  epi.e = at<float>(dv.ws, j.e);
  epi.cb = cb;
  epi.cc = cc;
  h16* mir[PARTS];
  mir[0] = epi.oh;
  mir[PARTS - 1] = PARTS == 2 ? epi.ol : epi.oh;
  nt_store<C, PARTS>(acc, lds, p0, q0, m, m, mirror, mir, m, epi);
}

// A = X X^T (STEP 0) or B = bA + cA^2 (STEP 1), off the diagonal, and the diagonal.
// One product, 4096 x 4096, tiles of 192: 88 and 91 us for the 69 GFLOP of a triangle
// (253 tiles, one a CU: 63 us of products and an epilogue that nothing hides).
template <class C, int STEP, int PROD>
__global__ __launch_bounds__(C::THREADS, C::OCC) void ns_sym(const NsDev dv, float cb, float cc) {
  __shared__ __attribute__((aligned(1024))) char lds[NtEpi<C, PROD == 3 ? 2 : 1>::LDS];
  const int t = nt_xcd(blockIdx.x, dv.tiles);
  if (t >= dv.tiles) return;
  const NsJob& j = ns_job(dv, t);
  int ti, tj;
  ns_triangle(t - j.t[STEP], &ti, &tj);
  NtTile nt;
  ns_sym_tile<STEP>(dv, j, ti * C::BP, tj * C::BQ, &nt);
  nt.part = 0;
  nt.parts = 1;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C>(nt, lds, acc);
  const int wave = threadIdx.x >> 6;
  ns_sym_out<C, STEP, PROD>(dv, j, cb, cc, acc, lds, ti * C::BP + (wave / C::WQ) * 32 * C::TP,
                            tj * C::BQ + (wave % C::WQ) * 32 * C::TQ, ti != tj);
}

// What a tile of X' stores: X' as laid out in two parts (its transpose through
// nt_store), or with LAST the weights' update or the result.
template <int PARTS, bool LAST>
struct NsXEpi {
  int rows, cols, rp, cp, tall;
  const h16 *nh, *nl;
  h16 *nho, *nlo, *w;
  const float* e;
  float ca, keep, alpha;
  bool update;
  static constexpr int OUTS = 2;  // X' in two parts, or the weights in the first
  static constexpr bool DIAGONAL = false;
  struct Pre {
    V8 h, l, w;
    float e[8];
  };

  __device__ __forceinline__ Pre load(int p, int q) const {
    Pre r;
    if (LAST && update) {
      const int pw = p < cols ? p : 0, qw = q < rows ? q : 0;
      const h16* wp = w + (int64_t)qw * cols + pw;
      if (pw + 8 <= cols) {
        r.w = load16u(wp);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) r.w.h[k] = wp[pw + k < cols ? k : 0];
      }
    }
    p = p < cp ? p : 0;
    q = q < rp ? q : 0;
    const int64_t o = (int64_t)q * cp + p;
    r.h = load16(nh + o);
    r.l = load16(nl + o);
    // (a tall matrix's diagonal runs along p)
    const floatx4* ev = reinterpret_cast<const floatx4*>(e + (tall ? p : q & ~7));
    const floatx4 x = ev[0], y = ev[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r.e[k] = x[k];
      r.e[4 + k] = y[k];
    }
    if (!tall) {
      float eq = r.e[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) eq = (q & 7) == k ? r.e[k] : eq;
#pragma unroll
      for (int k = 0; k < 8; ++k) r.e[k] = eq;
    }
    return r;
  }
  __device__ __forceinline__ void compute(int p, int q, const float (&f)[8], const Pre& pre,
                                          V8 (&out)[2]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float h = to_f32(pre.h.h[k]), l = to_f32(pre.l.h[k]), E = pre.e[k];
      // (products = 1: the low part takes part in aX only, as in B'X)
      const float y = __builtin_fmaf(PARTS == 2 ? ca + E : ca, l, f[k] * (1.0f / kSb));
      const float x = __builtin_fmaf(ca + E, h, y);
      if (!LAST) {
        out[0].h[k] = to_h16(x);
        out[1].h[k] = to_h16(x - to_f32(out[0].h[k]));
      } else {
        const float ox = x * (1.0f / kSx);
        out[0].h[k] =
            to_h16(update ? __builtin_fmaf(-alpha, ox, keep * to_f32(pre.w.h[k])) : alpha * ox);
      }
    }
  }
  __device__ __forceinline__ void store(int p, int q, const V8 (&out)[2]) const {
    if (!LAST) {
      // (X' is zero in the padding, which is part of the next operands)
      if (p >= cp || q >= rp) return;
      const int64_t o = (int64_t)q * cp + p;
      store16(nho + o, out[0]);
      store16(nlo + o, out[1]);
      return;
    }
    if (p >= cols || q >= rows) return;
    store8_upto(w + (int64_t)q * cols + p, out[0], cols - p);
  }
};

// The operands of one tile of X'; rows p run along the columns of the matrix as
// laid out, q along its rows.
__device__ __forceinline__ void ns_x_tile(const NsDev& dv, const NsJob& j, int cur, int pt, int qt,
                                          NtTile* nt) {
  const int tall = j.tall, m = tall ? j.cp : j.rp;
  const h16* bh = at<h16>(dv.ws, j.b);
  const h16* bl = at<h16>(dv.ws, j.bl);
  // X^T as [n][m]: the transpose, or a tall matrix as laid out
  const h16* xh = at<h16>(dv.ws, tall ? j.nat[cur] : j.mir[cur]);
  const h16* xl = at<h16>(dv.ws, tall ? j.natl[cur] : j.mirl[cur]);
  const int64_t po = (int64_t)pt * m, qo = (int64_t)qt * m;
  nt->p[0] = (tall ? bh : xh) + po;
  nt->q[0] = (tall ? xh : bh) + qo;
  nt->p[1] = (tall ? bl : xl) + po;
  nt->q[1] = (tall ? xl : bl) + qo;
  nt->ldp = nt->ldq = (uint32_t)m * 2u;
  nt->prows = j.cp - pt;
  nt->qrows = j.rp - qt;
  nt->kbytes = m * 2;
}

// Tile t of X' of a matrix: four tiles of rows p at a time, their rows q in turn.
template <class C>
__device__ __forceinline__ void ns_x_place(const NsJob& j, int t, int* pt, int* qt) {
  const int tp = (j.cp + C::BP - 1) / C::BP, tq = (j.rp + C::BQ - 1) / C::BQ;
  const int g = t / (4 * tq), w = t - g * 4 * tq;
  const int gw = tp - 4 * g < 4 ? tp - 4 * g : 4;
  *pt = (4 * g + w % gw) * C::BP;
  *qt = (w / gw) * C::BQ;
}

template <class C, int PROD, bool LAST>
__device__ __forceinline__ void ns_x_out(const NsDev& dv, const NsJob& j, int cur, float ca,
                                         float keep, const floatx16 (&acc)[C::TP][C::TQ], char* lds,
                                         int p0, int q0) {
  constexpr int PARTS = PROD == 3 ? 2 : 1;
  const int tall = j.tall;
  // X as laid out, now and next; its low part is an operand (and alternates) only
  // with three products
  const int nc = tall ? cur : 0, nn = tall ? cur ^ 1 : 0, mn = tall ? 0 : cur ^ 1;
  NsXEpi<PARTS, LAST> epi;
  epi.rows = j.rows;
  epi.cols = j.cols;
  epi.rp = j.rp;
  epi.cp = j.cp;
  epi.tall = tall;
  epi.nh = at<h16>(dv.ws, j.nat[nc]);
  epi.nl = at<h16>(dv.ws, j.natl[PARTS == 2 ? nc : 0]);
  epi.nho = at<h16>(dv.ws, j.nat[nn]);
  epi.nlo = at<h16>(dv.ws, j.natl[PARTS == 2 ? nn : 0]);
  epi.w = j.w;
  epi.e = at<float>(dv.ws, j.e);
  epi.ca = ca;
  epi.keep = keep;
  epi.alpha = j.alpha;
  epi.update = j.m != nullptr;
  h16* mir[PARTS];
  mir[0] = at<h16>(dv.ws, j.mir[mn]);
  mir[PARTS - 1] = at<h16>(dv.ws, PARTS == 2 ? j.mirl[mn] : j.mir[mn]);
  nt_store<C, PARTS>(acc, lds, p0, q0, j.cp, j.rp, !LAST, mir, j.rp, epi);
}

// The XCDs take the tiles of X' of a set of matrices in groups of 32 in turn: with an
// eighth of the list each, which is sorted, the first has the longest reductions
// (ResNet-50's 54 matrices 95 us, 81 so; groups of 8 81, of 16 82).
constexpr int kNsGroup = 32;
__host__ __device__ inline int ns_group(int n, bool single) {
  const int e = (n + 7) >> 3;
  return single || e < kNsGroup ? e : kNsGroup;
}
__device__ __forceinline__ int ns_xcd(const NsDev& dv) {
  const int g = ns_group(dv.tiles, dv.single), i = blockIdx.x >> 3;
  return (i / g * 8 + (blockIdx.x & 7)) * g + i % g;
}

// X' = (a + E) X + B'X.  Bound by the products where m is long (4096 x 4096: 153 us,
// 137 GFLOP; about 90 us of them the products) and by the epilogue's 10 bytes an element
// where it is short (ResNet-50's 54 matrices, 25.5 million elements: 79 us, 358 MB
// moved, the matrix cores 18 % busy).  A low part in 8 bits, 8 bytes an element,
// measured the same.
template <class C, int PROD, bool LAST>
__global__ __launch_bounds__(C::THREADS, C::OCC) void ns_x(const NsDev dv, int cur, float ca,
                                                           float keep) {
  __shared__ __attribute__((aligned(1024))) char lds[NtEpi<C, PROD == 3 ? 2 : 1>::LDS];
  const int t = ns_xcd(dv);
  if (t >= dv.tiles) return;
  const NsJob& j = ns_job(dv, t);
  int pt, qt;
  ns_x_place<C>(j, t - j.t[2], &pt, &qt);
  NtTile nt;
  ns_x_tile(dv, j, cur, pt, qt, &nt);
  nt.part = 0;
  nt.parts = 1;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C>(nt, lds, acc);
  const int wave = threadIdx.x >> 6;
  ns_x_out<C, PROD, LAST>(dv, j, cur, ca, keep, acc, lds, pt + (wave / C::WQ) * 32 * C::TP,
                          qt + (wave % C::WQ) * 32 * C::TQ);
}

// A of few tiles with a long reduction: each reduction in `parts` workgroups, whose
// sums a second launch adds in order (64 x 64 of a tile a workgroup) and stores.  The
// workgroups of one part are neighbours: they share operands in the L2.
// (3 of 512 x 4608, three products: 24 us, 75 on whole 128 x 128 tiles, 29 on 64.)
template <int PROD>
__global__ __launch_bounds__(256, 1) void ns_part(const NsDev dv, int parts) {
  typedef typename NsTiles<PROD>::T128d C;
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  const int x = nt_xcd(blockIdx.x, dv.tiles * parts);
  if (x >= dv.tiles * parts) return;
  const int part = x / dv.tiles, t = x - part * dv.tiles;
  const NsJob& j = ns_job(dv, t);
  int ti, tj;
  ns_triangle(t - j.t[0], &ti, &tj);
  NtTile nt;
  ns_sym_tile<0>(dv, j, ti * C::BP, tj * C::BQ, &nt);
  nt.part = part;
  nt.parts = parts;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C>(nt, lds, acc);
  nt_put<C>(acc, at<floatx4>(dv.ws, dv.sums) + ((size_t)t * parts + part) * (C::BP * C::BQ / 4));
}

template <int PROD>
__global__ __launch_bounds__(256) void ns_sum(const NsDev dv, int parts) {
  typedef typename NsTiles<PROD>::T128d C;
  typedef NtCfg<2, 2, 1, 1, 128, 1, 1> O;  // 64 x 64, 32 x 32 a wave
  __shared__ __attribute__((aligned(1024))) char lds[NtEpi<O, PROD == 3 ? 2 : 1>::LDS];
  const int t = blockIdx.x / C::WAVES, w = blockIdx.x % C::WAVES;  // tile and wave of it
  const NsJob& j = ns_job(dv, t);
  const int wave = threadIdx.x >> 6;
  const floatx4* from = at<floatx4>(dv.ws, dv.sums) + (size_t)t * parts * (C::BP * C::BQ / 4);
  floatx16 acc[1][1] = {{nt_get<C>(from, parts, w, wave / 2, wave % 2)}};
  int ti, tj;
  ns_triangle(t - j.t[0], &ti, &tj);
  ns_sym_out<O, 0, PROD>(dv, j, 0.0f, 0.0f, acc, lds,
                         ti * C::BP + (w / C::WQ) * 64 + (wave / 2) * 32,
                         tj * C::BQ + (w % C::WQ) * 64 + (wave % 2) * 32, ti != tj);
}

// ---- few small matrices: one workgroup each, one launch --------------------------
//
// With a short side of at most 64 and a long one of at most 1024, X stays in registers,
// high and low part of an element in one, from the first read to the last store: a wave holds tiles of 32 n x 64 m
// (n along the longer side), lane l column m = l % 32 of each half and 16 values of n.
// For A, which reduces over n, that is an operand's layout already (any order of n
// serves if both operands share it); for B'X each wave turns its own tiles around
// through LDS.  Only the waves' shares of A are exchanged.  Bound by latency, the
// barriers and the one CU's products and LDS.  Against the same as launches over all
// CUs, five steps, in us (1 to 24 matrices take the same time here):
//                       products 1     products 3
//     64 x 64             20 / 57        26 / 63
//     64 x 576            37 / 69        52 / 81
//     64 x 1024           53 / 77        78 / 91
//     24 of 64 x 1024     54 / 94        79 / 111
// (25 of them, which the arguments do not hold, take 108 and 131 over all CUs.)
constexpr int kSmallWaves = 8, kSmallTiles = 4;           // tiles of a wave at most
constexpr int kSmallShort = 64, kSmallLong = 32 * kSmallWaves * kSmallTiles;

struct NsSmall {
  float coef[3 * kNsMaxSteps];
  int steps, nesterov;
  float mu, keep;
};
static_assert(sizeof(NsChunk) + sizeof(NsSmall) <= 4096, "kernel arguments");

// half of (row, k) of an operand of rows of 64 halves, in the order of nt_product
__device__ __forceinline__ int ns_at(int row, int k) {
  return row * 64 + (((k >> 3) ^ ((row >> 1) & 7)) * 8) + (k & 7);
}

template <int PROD>
__global__ __launch_bounds__(64 * kSmallWaves) void ns_small(const NsChunk c, const NsSmall a) {
  constexpr int H = PROD == 3 ? 2 : 1, W = kSmallWaves, T = kSmallTiles;
  constexpr int WAVE = 12288;                 // bytes of a wave's own region
  constexpr int GLD = 36, TLD = 72, FLD = 36, ULD = 68;  // strides: 64 m x 32 n, 32 n x 64 m
  static_assert(2 * 64 * GLD * 2 <= WAVE && 2 * 32 * TLD * 2 <= WAVE, "inputs");
  static_assert(64 * FLD * 4 <= WAVE && 32 * ULD * 4 <= WAVE, "outputs");
  static_assert(H * 32 * 64 * 2 <= WAVE && 3 * 4096 <= WAVE, "operands, sums");
  __shared__ __attribute__((aligned(1024))) char region[W][WAVE];
  __shared__ __attribute__((aligned(1024))) h16 la[H][64 * 64], lb[H][64 * 64];
  __shared__ __attribute__((aligned(16))) float ld[64], le[64];
  __shared__ double red[W];
  const NsJob& j = c.job[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lrow = lane & 31, lhi = lane >> 5;
  const bool tall = j.tall, has_m = j.m != nullptr;
  const int nlen = tall ? j.rows : j.cols;
  char* const own = region[wave];
  h16* const oh = reinterpret_cast<h16*>(own);
  float* const of = reinterpret_cast<float*>(own);

  // an element of X, v * f: its high and low part
  auto pack = [](float v, float f) {
    const h16 h = (h16)(v * f);
    return half2{h, (h16)__builtin_fmaf(v, f, -to_f32(h))};
  };
  // chunk i of this lane of a tile from n0: its offset in the matrix, the elements of
  // it that are there, and its place in a tile laid out by rows of ld elements
  auto chunk = [&](int n0, int i, int ld, int64_t* off, int* left, int* at) {
    const int r = tall ? 8 * i + (lane >> 3) : 16 * i + (lane >> 2);
    const int k = tall ? 8 * (lane & 7) : 8 * (lane & 3);
    const int row = tall ? n0 + r : r, col = tall ? k : n0 + k;
    *off = (int64_t)row * j.cols + col;
    *left = row < j.rows ? j.cols - col : 0;
    *at = r * ld + k;
  };

  // momentum, and X in registers.  u = cm m' + cg g is any of ns_dir's, exactly.
  const float cm = !has_m ? 0.0f : a.nesterov ? a.mu : 1.0f;
  const float cg = has_m && !a.nesterov ? 0.0f : 1.0f;
  half2 x[T][2][16];
  double s = 0.0;
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][b][e] = half2{0, 0};
  constexpr int IN = 64 * GLD;  // halves of one staged input
  static_assert(32 * TLD <= IN, "staging");
  V8 g[4], m[4];
  // (one copy of the code for all tiles: fetching it is what a launch waits for)
#pragma unroll 1
  for (int t = -1; t < T; ++t) {
    const int n0 = 32 * (wave + W * t);
    if (n0 >= nlen) break;
    if (t >= 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int64_t off;
        int left, at;
        chunk(n0, i, tall ? TLD : GLD, &off, &left, &at);
        if (has_m) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            m[i].h[e] = to_h16(__builtin_fmaf(a.mu, to_f32(m[i].h[e]), to_f32(g[i].h[e])));
          if (left > 0) store8_upto(j.m + off, m[i], left);
        }
        uint2* pg = reinterpret_cast<uint2*>(oh + at);
        uint2* pm = reinterpret_cast<uint2*>(oh + IN + at);
        pg[0] = make_uint2(g[i].u[0], g[i].u[1]);
        pg[1] = make_uint2(g[i].u[2], g[i].u[3]);
        pm[0] = make_uint2(m[i].u[0], m[i].u[1]);
        pm[1] = make_uint2(m[i].u[2], m[i].u[3]);
      }
      nt_wave_sync();
    }
    // the next tile's loads
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int64_t off;
      int left, at;
      chunk(n0 + 32 * W, i, 0, &off, &left, &at);
      g[i] = m[i] = zero8();
      if (t + 1 < T && left > 0) {
        g[i] = load8_upto(j.g + off, left);
        if (has_m) m[i] = load8_upto(j.m + off, left);
      }
    }
    if (t >= 0) {
      const h16* const from = oh + (tall ? 4 * lhi * TLD + lrow : lrow * GLD + 4 * lhi);
      // (squares in float64: those of a finite float32 need not be finite in float32)
      float u[2][16];
      double sq[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int n = 8 * (e / 4) + e % 4, at = tall ? n * TLD + 32 * b : 32 * b * GLD + n;
          // (elements past the matrix were read as zeros)
          u[b][e] = __builtin_fmaf(cm, to_f32(from[IN + at]), cg * to_f32(from[at]));
          sq[e / 4] = __builtin_fma((double)u[b][e], (double)u[b][e], sq[e / 4]);
        }
      s += (sq[0] + sq[1]) + (sq[2] + sq[3]);
#pragma unroll
      for (int k = 0; k < T; ++k) {
        if (k != t) continue;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[k][b][e] = __builtin_bit_cast(half2, u[b][e]);
      }
      nt_wave_sync();
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  if (lane == 0) red[wave] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int i = 0; i < W; ++i) s += red[i];
  const float rs = ns_rsqrt(s);
#pragma unroll
  for (int t = 0; t < T; ++t) {
    if (32 * (wave + W * t) >= nlen) continue;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][b][e] = pack(__builtin_bit_cast(float, x[t][b][e]), rs);
  }

  auto frag = [&](const h16* rows, int row, int ks) {
    return *reinterpret_cast<const half8*>(rows + ns_at(row, ks * 16 + lhi * 8));
  };
  // four elements k .. k + 3 of a row of A or B, and their mirror images
  auto put = [&](h16* hi, h16* lo, int q, int p, const float (&v)[4], bool mirror) {
    h16 th[4], tl[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      th[r] = to_h16(v[r]);
      tl[r] = to_h16(v[r] - to_f32(th[r]));
    }
    __builtin_memcpy(__builtin_assume_aligned(hi + ns_at(q, p), 8), th, 8);
    if (H == 2) __builtin_memcpy(__builtin_assume_aligned(lo + ns_at(q, p), 8), tl, 8);
    if (mirror) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        hi[ns_at(p + r, q)] = th[r];
        if (H == 2) lo[ns_at(p + r, q)] = tl[r];
      }
    }
  };

  for (int step = 0; step < a.steps; ++step) {
    const float ca = a.coef[3 * step], cb = a.coef[3 * step + 1], cc = a.coef[3 * step + 2];
    // A = X X^T of the wave's tiles: its 32 x 32 tiles (0, 0), (1, 0) and (1, 1)
    floatx16 acc[3];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][e] = 0.0f;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (32 * (wave + W * t) >= nlen) continue;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        half8 f[H][2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            f[0][b][e] = x[t][b][8 * k + e][0];
            if (H == 2) f[H - 1][b][e] = x[t][b][8 * k + e][1];
          }
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int p = i > 0, q = i > 1;
          if (H == 2) {
            acc[i] = NtHalf::mma(f[H - 1][p], f[0][q], acc[i]);
            acc[i] = NtHalf::mma(f[0][p], f[H - 1][q], acc[i]);
          }
          acc[i] = NtHalf::mma(f[0][p], f[0][q], acc[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const floatx4 v = {acc[i][4 * e], acc[i][4 * e + 1], acc[i][4 * e + 2], acc[i][4 * e + 3]};
        reinterpret_cast<floatx4*>(own)[(i * 4 + e) * 64 + lane] = v;
      }
    __syncthreads();
    for (int o = tid; o < 768; o += 64 * W) {
      floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < W; ++w) v += reinterpret_cast<const floatx4*>(region[w])[o];
      const int i = o / 256, e = o / 64 % 4, l = o % 64;
      const int p = 32 * (i > 0) + 8 * e + 4 * (l / 32), q = 32 * (i > 1) + l % 32;
      float r[4], dq = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        dq = p + k == q ? v[k] * (1.0f / (kSx * kSx)) : dq;
        r[k] = p + k == q ? 0.0f : v[k] * (kSa / (kSx * kSx));
      }
      if ((unsigned)(q - p) < 4u) ld[q] = dq;
      put(la[0], la[H - 1], q, p, r, i == 1);
    }
    __syncthreads();
    // B = bA + cA^2, a tile each of the first four waves
    if (wave < 4) {
      const int p0 = 32 * (wave / 2), q0 = 32 * (wave % 2);
      floatx16 b;
#pragma unroll
      for (int e = 0; e < 16; ++e) b[e] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const half8 ph = frag(la[0], p0 + lrow, ks), qh = frag(la[0], q0 + lrow, ks);
        if (H == 2) {
          b = NtHalf::mma(frag(la[H - 1], p0 + lrow, ks), qh, b);
          b = NtHalf::mma(ph, frag(la[H - 1], q0 + lrow, ks), b);
        }
        b = NtHalf::mma(ph, qh, b);
      }
      const int q = q0 + lrow;
      const float dq = ld[q];
      float b2 = 0.0f;  // of the diagonal
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int p = p0 + 8 * e + 4 * lhi;
        h16 ah[4], al[4] = {0, 0, 0, 0};
        __builtin_memcpy(ah, __builtin_assume_aligned(la[0] + ns_at(q, p), 8), 8);
        if (H == 2) __builtin_memcpy(al, __builtin_assume_aligned(la[H - 1] + ns_at(q, p), 8), 8);
        const floatx4 dp = *reinterpret_cast<const floatx4*>(ld + p);
        float r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float av = (to_f32(ah[k]) + to_f32(al[k])) * (1.0f / kSa);
          const float a2 = b[4 * e + k] * (1.0f / (kSa * kSa));
          b2 = p + k == q ? a2 : b2;
          r[k] = kSb * __builtin_fmaf(cc, __builtin_fmaf(dq + dp[k], av, a2), cb * av);
          r[k] = p + k == q ? 0.0f : r[k];
        }
        put(lb[0], lb[H - 1], q, p, r, false);
      }
      if (p0 == q0 && lhi == (lrow >> 2 & 1))
        le[q] = __builtin_fmaf(cc, __builtin_fmaf(dq, dq, b2), cb * dq);
    }
    __syncthreads();
    // X = (a + E) X + B'X, tile by tile
    const float kE[2] = {kSb * (ca + le[lrow]), kSb * (ca + le[32 + lrow])};
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (32 * (wave + W * t) >= nlen) continue;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          // ns_at(8 (e / 4) + 4 lhi + e % 4, 32 b + lrow), lanes and constants apart
          const int lanes = lhi * 256 + (((lrow >> 3) ^ (2 * lhi) ^ (e % 4 / 2)) * 8) + (lrow & 7);
          h16* const to = oh + lanes + (8 * (e / 4) + e % 4) * 64 + 32 * (b ^ (e / 4 & 1));
          to[0] = x[t][b][e][0];
          if (H == 2) to[2048] = x[t][b][e][1];
        }
      nt_wave_sync();
      floatx16 y[2];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) y[b][e] = 0.0f;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const half8 ph = frag(oh, lrow, ks);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const half8 qh = frag(lb[0], 32 * b + lrow, ks);
          if (H == 2) {
            y[b] = NtHalf::mma(frag(oh + 2048, lrow, ks), qh, y[b]);
            y[b] = NtHalf::mma(ph, frag(lb[H - 1], 32 * b + lrow, ks), y[b]);
          }
          y[b] = NtHalf::mma(ph, qh, y[b]);
        }
      }
      nt_wave_sync();
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          // (see NsXEpi)
          const float h = to_f32(x[t][b][e][0]), l = to_f32(x[t][b][e][1]);
          const float f = __builtin_fmaf(H == 2 ? kE[b] : kSb * ca, l, y[b][e]);
          x[t][b][e] = pack(__builtin_fmaf(kE[b], h, f), 1.0f / kSb);
        }
    }
  }

  // the weights' update or the result, rows whole
#pragma unroll 1
  for (int t = 0; t < T; ++t) {
    const int n0 = 32 * (wave + W * t);
    if (n0 >= nlen) break;
    float* const to = of + (tall ? 4 * lhi * ULD + lrow : lrow * FLD + 4 * lhi);
#pragma unroll
    for (int k = 0; k < T; ++k) {
      if (k != t) continue;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int n = 8 * (e / 4) + e % 4;
          to[tall ? n * ULD + 32 * b : 32 * b * FLD + n] =
              (to_f32(x[k][b][e][0]) + to_f32(x[k][b][e][1])) * (1.0f / kSx);
        }
    }
    nt_wave_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int64_t off;
      int left, at;
      chunk(n0, i, tall ? ULD : FLD, &off, &left, &at);
      if (left <= 0) continue;
      const floatx4 lo = *reinterpret_cast<const floatx4*>(of + at);
      const floatx4 hi = *reinterpret_cast<const floatx4*>(of + at + 4);
      const V8 w = has_m ? load8_upto(j.w + off, left) : zero8();
      V8 out;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float o = e < 4 ? lo[e & 3] : hi[e & 3];
        out.h[e] = to_h16(has_m ? __builtin_fmaf(-j.alpha, o, a.keep * to_f32(w.h[e])) : j.alpha * o);
      }
      store8_upto(j.w + off, out, left);
    }
    nt_wave_sync();
  }
}

// ---- the plan ------------------------------------------------------------------

int up(int v, int t) { return (v + t - 1) / t * t; }

// The tiles a product may run on, with one product and with three.  Times of a
// 128-byte slice of the reduction in microseconds, for one workgroup alone (alone)
// and for a CU whatever it holds (cu); of a launch besides, for A or B and for X',
// whose outputs read more; and of the sums of a workgroup to memory and back.  Fitted
// to what each tile took on ten sets of 256 to 8192 rows and columns.  Of the times
// below (A / X' in us) four in five are met within 13 %; X' of the three matrices is
// estimated 15 to 34 % low on 64, 64 deep and 128 deep (what a tile stores counts for
// the launch only), X' of 4096 x 4096 up to 20 % high on tiles below 192, A in parts up
// to 28 % high.  The choice costs 7 us at most there (X' of the three matrices, one
// product: 128 deep):
//                          256       192       128  128 deep        64   64 deep  128 in parts
//  1: 4096 x 4096      101/136    79/171   114/150   110/177   166/275   184/346       -
//     1024 x 4096        80/40     49/34     46/25     30/23     18/26     17/33   18/-
//     3 of 512 x 4608    88/33     53/30     49/22     30/29     18/30     18/41   16/-
//  3: 4096 x 4096      280/398   193/433   294/430   272/463   319/511   338/544       -
//     1024 x 4096       227/92    117/54    100/47     67/39     45/40     27/46   26/-
//     3 of 512 x 4608   258/67    128/43    109/37     75/46     49/45     29/53   24/-
// a_only: rows that are offered to A alone.  The last cuts reductions, which only A's
// are long enough for.  64 deep wins by its shorter `alone` time where one reduction
// bounds the launch; with one product that takes more than 16 slices (12 for X'), and
// B and X' of a side that long have tiles enough to bound it by `cu`.
constexpr int kNsKinds = 7;
constexpr NsTile kNsTiles[2][kNsKinds] = {
    {{"256", 256, 1, 1, 1.23, 1.87, {11.1, 19.3}, 0.0, false},
     {"192", 192, 1, 1, 0.68, 1.09, {11.8, 21.0}, 0.0, false},
     {"128", 128, 1, 2, 0.68, 0.57, {6.4, 13.0}, 0.0, false},
     {"128 deep", 128, 1, 1, 0.31, 0.74, {7.7, 8.5}, 0.0, false},
     {"64", 64, 1, 2, 0.19, 0.29, {4.7, 6.3}, 0.0, false},
     {"64 deep", 64, 1, 1, 0.165, 0.37, {5.1, 0.0}, 0.0, true},
     {"128", 128, 2, 1, 0.31, 0.30, {9.0, 0.0}, 0.036, true}},
    {{"256", 256, 1, 1, 3.80, 5.50, {15.7, 31.8}, 0.0, false},
     {"192", 192, 1, 1, 1.71, 2.82, {14.6, 23.1}, 0.0, false},
     {"128", 128, 1, 2, 1.53, 1.76, {7.8, 12.9}, 0.0, false},
     {"128 deep", 128, 1, 1, 1.04, 1.72, {8.1, 11.6}, 0.0, false},
     {"64", 64, 1, 2, 0.62, 0.53, {5.0, 6.9}, 0.0, false},
     {"64 deep", 64, 1, 1, 0.30, 0.60, {5.5, 7.0}, 0.0, false},
     {"128", 128, 2, 1, 0.44, 0.59, {11.0, 0.0}, 0.033, true}}};

// The tile that a product of the set finishes soonest on, by that estimate: the
// work spread over the CUs (and half of the longest reduction for the last round),
// or the longest reduction if that takes longer.  The last kind, for A only, splits
// reductions in as many parts as give every CU one; its sums go to memory and back.
// stage 0: A, 1: B, 2: X'.
int ns_choose(int stage, int count, const int32_t* rows, const int32_t* cols, int products,
              NsTile* tile) {
  constexpr double cus = 256.0;
  int best = -1;
  double bt = 0;
  for (int i = 0; i < kNsKinds; ++i) {
    NsTile c = kNsTiles[products == 3][i];
    if (c.a_only && stage != 0) continue;
    double tiles = 0, work = 0, longest = 0;
    for (int n = 0; n < count; ++n) {
      const int r = up(rows[n], 64), l = up(cols[n], 64), m = std::min(r, l);
      const double k = (stage == 0 ? std::max(r, l) : m) / 64, tm = ceil_div(m, c.side);
      const double t =
          stage == 2 ? (double)ceil_div(l, c.side) * ceil_div(r, c.side) : tm * (tm + 1) / 2;
      tiles += t;
      work += t * k;
      longest = std::max(longest, k);
    }
    double t = c.fixed[stage == 2];
    if (c.parts > 1) {
      c.parts = (int)std::min(std::min(cus / tiles, longest / 2), 16.0);
      if (c.parts < 2) continue;
      longest = ceil(longest / c.parts);
      t += tiles * c.parts * c.sums;
    }
    const double tail = tiles > cus * c.occ ? 0.5 * longest * c.alone : 0.0;
    t += std::max(work / cus * c.cu + tail, longest * c.alone);
    if (best < 0 || t < bt) {
      bt = t;
      best = i;
      *tile = c;
    }
  }
  return best;
}

struct NsStep {
  int stage, cur;
  bool last;
  float ca, cb, cc, keep;
};

// (A_ONLY: a tile of A alone, see kNsTiles)
template <class C, int PROD, bool A_ONLY = false>
void ns_launch(const NsStep& s, const NsDev& d, hipStream_t st) {
  // (a multiple of the XCDs' groups, see ns_xcd and nt_xcd)
  const int gr = 8 * ns_group(d.tiles, s.stage < 2 || d.single);
  const dim3 grid((unsigned)ceil_div(d.tiles, gr) * gr), block(C::THREADS);
  if constexpr (A_ONLY) {
    hipLaunchKernelGGL((ns_sym<C, 0, PROD>), grid, block, 0, st, d, s.cb, s.cc);
  } else {
    if (s.stage == 0)
      hipLaunchKernelGGL((ns_sym<C, 0, PROD>), grid, block, 0, st, d, s.cb, s.cc);
    else if (s.stage == 1)
      hipLaunchKernelGGL((ns_sym<C, 1, PROD>), grid, block, 0, st, d, s.cb, s.cc);
    else if (!s.last)
      hipLaunchKernelGGL((ns_x<C, PROD, false>), grid, block, 0, st, d, s.cur, s.ca, s.keep);
    else
      hipLaunchKernelGGL((ns_x<C, PROD, true>), grid, block, 0, st, d, s.cur, s.ca, s.keep);
  }
}

template <int PROD>
hipError_t ns_run(const NsPlan& p, const NsArgs& a, char* ws, hipStream_t st) {
  const NsDev pre{ws, p.table, p.map_pre, 0, p.n_pre, p.count == 1};
  hipLaunchKernelGGL((ns_split<PROD>), dim3((unsigned)p.n_pre), dim3(256), 0, st, pre, a.momentum,
                     a.nesterov);
  for (int i = 0; i < a.steps; ++i) {
    for (int stage = 0; stage < 3; ++stage) {
      const NsStep s{stage, i & 1, i + 1 == a.steps, a.coef[3 * i], a.coef[3 * i + 1],
                     a.coef[3 * i + 2], a.keep};
      const NsDev d{ws, p.table, p.map[stage], p.sums, p.tiles[stage], p.count == 1};
      const int parts = p.kind[stage].parts;
      switch (p.variant[stage]) {
        case 0: ns_launch<typename NsTiles<PROD>::T256, PROD>(s, d, st); break;
        case 1: ns_launch<typename NsTiles<PROD>::T192, PROD>(s, d, st); break;
        case 2: ns_launch<typename NsTiles<PROD>::T128, PROD>(s, d, st); break;
        case 3: ns_launch<typename NsTiles<PROD>::T128d, PROD>(s, d, st); break;
        case 4: ns_launch<typename NsTiles<PROD>::T64, PROD>(s, d, st); break;
        case 5: ns_launch<typename NsTiles<PROD>::T64d, PROD, PROD == 1>(s, d, st); break;
        default:
          hipLaunchKernelGGL((ns_part<PROD>), dim3((unsigned)(8 * ((d.tiles * parts + 7) / 8))),
                             dim3(256), 0, st, d, parts);
          hipLaunchKernelGGL((ns_sum<PROD>), dim3((unsigned)(d.tiles * 4)), dim3(256), 0, st, d,
                             parts);
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

}  // namespace

void ns_plan(int count, const int32_t* rows, const int32_t* cols, int products, NsPlan* plan) {
  NsPlan& P = *plan;
  P.count = count;
  P.small = count <= kJobsPerLaunch;
  for (int i = 0; i < count; ++i)
    P.small = P.small && std::min(rows[i], cols[i]) <= kSmallShort &&
              std::max(rows[i], cols[i]) <= kSmallLong;
  for (int stage = 0; stage < 3; ++stage)
    P.variant[stage] = ns_choose(stage, count, rows, cols, products, &P.kind[stage]);
  // the longest products first
  for (int i = 0; i < count; ++i) P.order[i] = i;
  std::sort(P.order, P.order + count, [&](int x, int y) {
    const int64_t a = (int64_t)rows[x] + cols[x], b = (int64_t)rows[y] + cols[y];
    return a != b ? a > b : x < y;
  });
  uint64_t off = 0;  // units of 256 bytes
  auto take = [&](uint64_t bytes) {
    const uint64_t o = off;
    off += (bytes + 255) / 256;
    return (uint32_t)o;
  };
  P.table = take((uint64_t)count * sizeof(NsJob));
  P.tiles[0] = P.tiles[1] = P.tiles[2] = P.n_pre = 0;
  for (int i = 0; i < count; ++i) {
    NsJob& j = P.jobs[i];
    const int o = P.order[i];
    j = NsJob{};
    j.rows = rows[o];
    j.cols = cols[o];
    j.tall = j.rows > j.cols;
    j.rp = up(j.rows, 64);
    j.cp = up(j.cols, 64);
    const int m = j.tall ? j.cp : j.rp;
    for (int stage = 0; stage < 3; ++stage) {
      j.t[stage] = P.tiles[stage];
      P.tiles[stage] += ns_tiles(j, stage, P.kind[stage].side);
    }
    j.t_pre = P.n_pre;
    P.n_pre += (j.rp / 64) * (j.cp / 64);
    const int64_t n = (int64_t)j.rows * j.cols;
    j.nparts = (int)std::min<int64_t>(kNsParts, (n + 8191) / 8192);
    const uint64_t xb = (uint64_t)j.rp * j.cp * 2, ab = (uint64_t)m * m * 2;
    const bool split = products == 3;
    j.nat[0] = take(xb);
    j.mir[0] = take(xb);
    j.nat[1] = j.tall ? take(xb) : j.nat[0];
    j.mir[1] = j.tall ? j.mir[0] : take(xb);
    j.natl[0] = take(xb);
    j.mirl[0] = split ? take(xb) : 0;
    j.natl[1] = split && j.tall ? take(xb) : j.natl[0];
    j.mirl[1] = split && !j.tall ? take(xb) : j.mirl[0];
    j.a = take(ab);
    j.b = take(ab);
    j.al = split ? take(ab) : 0;
    j.bl = split ? take(ab) : 0;
    j.d = take((uint64_t)m * 4);
    j.e = take((uint64_t)m * 4);
    j.part = take((uint64_t)j.nparts * 8);
  }
  for (int stage = 0; stage < 3; ++stage) P.map[stage] = take((uint64_t)P.tiles[stage] * 2);
  P.map_pre = take((uint64_t)P.n_pre * 2);
  P.sums = take(P.kind[0].parts > 1 ? (uint64_t)P.tiles[0] * P.kind[0].parts * 65536 : 0);
  P.bytes = P.small ? 256 : (size_t)off * 256;  // (not used; 0 would mean a bad list)
}

hipError_t launch_ns(const NsPlan& p, const NsArgs& a, void* ws, hipStream_t st) {
  char* w = static_cast<char*>(ws);
  if (p.small) {
    NsChunk c{};
    std::copy(p.jobs, p.jobs + p.count, c.job);
    NsSmall s{};
    std::copy(a.coef, a.coef + 3 * a.steps, s.coef);
    s.steps = a.steps;
    s.nesterov = a.nesterov;
    s.mu = a.momentum;
    s.keep = a.keep;
    const dim3 grid((unsigned)p.count), block(64 * kSmallWaves);
    if (a.products == 3)
      hipLaunchKernelGGL(ns_small<3>, grid, block, 0, st, c, s);
    else
      hipLaunchKernelGGL(ns_small<1>, grid, block, 0, st, c, s);
    return hipGetLastError();
  }
  const NsPlaces pl{p.table, {p.map[0], p.map[1], p.map[2]}, p.map_pre,
                    {p.kind[0].side, p.kind[1].side, p.kind[2].side}};
  for (int first = 0; first < p.count; first += kJobsPerLaunch) {
    NsChunk c{};
    const int n = std::min(kJobsPerLaunch, p.count - first);
    int parts = 1;
    for (int i = 0; i < n; ++i) {
      c.job[i] = p.jobs[first + i];
      parts = std::max(parts, c.job[i].nparts);
    }
    hipLaunchKernelGGL(ns_first, dim3((unsigned)parts, (unsigned)n), dim3(256), 0, st, c, w, pl,
                       first, a.momentum, a.nesterov);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return a.products == 3 ? ns_run<3>(p, a, w, st) : ns_run<1>(p, a, w, st);
}

}  // namespace fp16k
