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
//    against float64): 2e-4 to 2e-3;
//  - products = 3 takes every operand as high + low part, three products for one
//    (the product of the low parts is below 2^-22): 1e-6 to 3e-5, so that the
//    result is rounded once, to binary16.
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

#include <algorithm>

namespace fp16k {
namespace {

constexpr float kSx = 4096.0f, kSa = 4096.0f, kSb = 2048.0f;

struct NsDev {
  char* ws;
  uint32_t table, map;  // in units of 256 bytes
  int tiles;
};

template <class T>
__device__ __forceinline__ T* at(char* ws, uint32_t place) {
  return reinterpret_cast<T*>(ws + (size_t)place * 256);
}

// ---- pass 1: momentum, squares, and the table ---------------------------------

constexpr int kJobsPerLaunch = 24;
struct NsChunk {
  NsJob job[kJobsPerLaunch];
};
static_assert(sizeof(NsChunk) <= 3584, "kernel arguments");

struct NsPlaces {
  uint32_t table, map_sym, map_x, map_pre;
  int tile_sym, tile_x;
};

__device__ __forceinline__ double ns_block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((red[0] + red[1]) + red[2]) + red[3];
}

// eight elements, at once where the matrix is 16-byte aligned
__device__ __forceinline__ V8 ns_load8(const h16* p, bool aligned) {
  if (aligned) return load16(p);
  V8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v.h[e] = p[e];
  return v;
}

// the float32 update direction before normalisation
__device__ __forceinline__ float ns_dir(h16 g, h16 m, float mu, bool has_m, bool nesterov) {
  if (!has_m) return to_f32(g);
  return nesterov ? __builtin_fmaf(mu, to_f32(m), to_f32(g)) : to_f32(m);
}

// Reads g and m, writes m' and this block's sum of squares of u (float64); block 0
// of a matrix also writes its entry of the table and its part of the maps.
// Bandwidth-bound: 6 bytes an element.
__global__ __launch_bounds__(256) void ns_first(const NsChunk c, char* ws, NsPlaces pl, int first,
                                                float mu, int nesterov) {
  __shared__ double red[4];
  const NsJob& j = c.job[blockIdx.y];
  if ((int)blockIdx.x >= j.nparts) return;
  const int tid = threadIdx.x;
  if (blockIdx.x == 0) {
    const int idx = first + blockIdx.y;
    if (tid == 0) at<NsJob>(ws, pl.table)[idx] = j;
    const int m = j.tall ? j.cp : j.rp, tm = (m + pl.tile_sym - 1) / pl.tile_sym;
    const int nsym = tm * (tm + 1) / 2;
    const int nx = ((j.rp + pl.tile_x - 1) / pl.tile_x) * ((j.cp + pl.tile_x - 1) / pl.tile_x);
    const int npre = (j.rp / 64) * (j.cp / 64);
    for (int i = tid; i < nsym; i += 256) at<uint16_t>(ws, pl.map_sym)[j.t_sym + i] = (uint16_t)idx;
    for (int i = tid; i < nx; i += 256) at<uint16_t>(ws, pl.map_x)[j.t_x + i] = (uint16_t)idx;
    for (int i = tid; i < npre; i += 256) at<uint16_t>(ws, pl.map_pre)[j.t_pre + i] = (uint16_t)idx;
  }
  const bool has_m = j.m != nullptr;
  const int64_t n = (int64_t)j.rows * j.cols, nvec = n / 8;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < nvec; i += (int64_t)j.nparts * 256) {
    const V8 g = ns_load8(j.g + i * 8, j.aligned);
    V8 m = zero8();
    if (has_m) {
      m = ns_load8(j.m + i * 8, j.aligned);
#pragma unroll
      for (int e = 0; e < 8; ++e) m.h[e] = to_h16(__builtin_fmaf(mu, to_f32(m.h[e]), to_f32(g.h[e])));
      if (j.aligned) {
        store16(j.m + i * 8, m);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) j.m[i * 8 + e] = m.h[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double u = (double)ns_dir(g.h[e], m.h[e], mu, has_m, nesterov);
      s = __builtin_fma(u, u, s);
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

// ---- pass 2: X = u / ||u|| split in two binary16 parts, both ways round --------

template <int PROD>
__global__ __launch_bounds__(256) void ns_split(const NsDev dv, float mu, int nesterov) {
  constexpr int LD = 72;
  __shared__ double red[4];
  __shared__ __attribute__((aligned(16))) h16 tile[PROD == 3 ? 2 : 1][64 * LD];
  const NsJob& j = at<NsJob>(dv.ws, dv.table)[at<uint16_t>(dv.ws, dv.map)[blockIdx.x]];
  const int tid = threadIdx.x;
  double s = 0.0;
  for (int i = tid; i < j.nparts; i += 256) s += at<double>(dv.ws, j.part)[i];
  s = ns_block_sum(s, red);
  // 0 for a zero matrix; no epsilon, since gradients trained without loss scaling
  // are small.  Not a number where an element is not finite.
  const float rs = s > 0.0 && s < __builtin_inf() ? (float)((double)kSx / sqrt(s))
                                                  : (s == 0.0 ? 0.0f : __builtin_nanf(""));
  const int local = blockIdx.x - j.t_pre, tc = j.cp / 64;
  const int r0 = (local / tc) * 64, c0 = (local % tc) * 64;
  const int row = r0 + tid / 4;
  const bool has_m = j.m != nullptr, whole = j.whole;
  h16* nat = at<h16>(dv.ws, j.nat[0]) + (int64_t)row * j.cp;
  h16* natl = at<h16>(dv.ws, j.natl[0]) + (int64_t)row * j.cp;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int col = c0 + (tid & 3) * 16 + v * 8;
    V8 g = zero8(), m = zero8(), hi, lo;
    const int64_t o = (int64_t)row * j.cols + col;
    if (row < j.rows && col < j.cols) {
      if (whole) {
        g = load16(j.g + o);
        if (has_m) m = load16(j.m + o);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e < j.cols) {
            g.h[e] = j.g[o + e];
            if (has_m) m.h[e] = j.m[o + e];
          }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = ns_dir(g.h[e], m.h[e], mu, has_m, nesterov);
      const float x = row < j.rows && col + e < j.cols ? u * rs : 0.0f;
      hi.h[e] = to_h16(x);
      lo.h[e] = to_h16(x - to_f32(hi.h[e]));
      tile[0][((tid & 3) * 16 + v * 8 + e) * LD + tid / 4] = hi.h[e];
      if (PROD == 3) tile[PROD == 3][((tid & 3) * 16 + v * 8 + e) * LD + tid / 4] = lo.h[e];
    }
    store16(nat + col, hi);
    store16(natl + col, lo);
  }
  __syncthreads();
  const int64_t mo = (int64_t)(c0 + tid / 4) * j.rp + r0;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int k = (tid & 3) * 16 + v * 8;
    store16(at<h16>(dv.ws, j.mir[0]) + mo + k, load16(&tile[0][(tid / 4) * LD + k]));
    if (PROD == 3)
      store16(at<h16>(dv.ws, j.mirl[0]) + mo + k, load16(&tile[PROD == 3][(tid / 4) * LD + k]));
  }
}

// ---- the three products of a step -----------------------------------------------

// This workgroup's matrix and its tile of the launch, or null.
__device__ __forceinline__ const NsJob* ns_job(const NsDev& dv, int* t) {
  *t = nt_xcd(blockIdx.x, dv.tiles);
  if (*t >= dv.tiles) return nullptr;
  return at<NsJob>(dv.ws, dv.table) + at<uint16_t>(dv.ws, dv.map)[*t];
}

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

// A = X X^T (STEP 0) or B = bA + cA^2 (STEP 1), off the diagonal, and the diagonal.
template <class C, int STEP, int PROD>
__global__ __launch_bounds__(C::THREADS, C::OCC) void ns_sym(const NsDev dv, float cb, float cc) {
  constexpr int PARTS = PROD == 3 ? 2 : 1;
  __shared__ __attribute__((aligned(1024))) char lds[NtEpi<C, PARTS>::LDS];
  int t;
  const NsJob* jp = ns_job(dv, &t);
  if (!jp) return;
  const NsJob& j = *jp;
  const int m = j.tall ? j.cp : j.rp, n = j.tall ? j.rp : j.cp;
  int ti, tj;
  ns_triangle(t - j.t_sym, &ti, &tj);
  const int pt = ti * C::BP, qt = tj * C::BQ;
  // X as [m][n]: laid out so, or the transpose of a tall matrix
  const h16* xh = at<h16>(dv.ws, j.tall ? j.mir[0] : j.nat[0]);
  const h16* xl = at<h16>(dv.ws, j.tall ? j.mirl[0] : j.natl[0]);
  const h16* ah = at<h16>(dv.ws, j.a);
  const h16* al = at<h16>(dv.ws, j.al);
  const h16* hi = STEP == 0 ? xh : ah;
  const h16* lo = STEP == 0 ? xl : al;
  const int k = STEP == 0 ? n : m;
  NtTile<PROD> nt;
  if (PROD == 3) {
    nt.p[0] = hi + (int64_t)pt * k;
    nt.q[0] = lo + (int64_t)qt * k;
    nt.p[PROD / 2] = lo + (int64_t)pt * k;
    nt.q[PROD / 2] = hi + (int64_t)qt * k;
  }
  nt.p[PROD - 1] = hi + (int64_t)pt * k;
  nt.q[PROD - 1] = hi + (int64_t)qt * k;
  nt.ldp = nt.ldq = (uint32_t)k * 2u;
  nt.prows = m - pt;
  nt.qrows = m - qt;
  nt.kbytes = k * 2;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C, PROD>(nt, lds, acc);
  const int wave = threadIdx.x >> 6;
  if (wave >= C::WAVES) return;
  NsSymEpi<STEP, PARTS> epi;
  epi.m = m;
  epi.ah = ah;
  epi.al = al;
  epi.oh = at<h16>(dv.ws, STEP == 0 ? j.a : j.b);
  epi.ol = at<h16>(dv.ws, STEP == 0 ? j.al : j.bl);
  epi.d = at<float>(dv.ws, j.d);
  epi.e = at<float>(dv.ws, j.e);
  epi.cb = cb;
  epi.cc = cc;
  h16* mir[PARTS];
  mir[0] = epi.oh;
  mir[PARTS - 1] = PARTS == 2 ? epi.ol : epi.oh;
  nt_store<C, PARTS>(acc, lds, pt + (wave / C::WQ) * 32 * C::TP, qt + (wave % C::WQ) * 32 * C::TQ, m,
                     m, ti != tj, mir, m, epi);
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
  bool update, whole;
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
      if (whole) {
        r.w = load16(wp);
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
    h16* const wp = w + (int64_t)q * cols + p;
    if (whole) {
      store16(wp, out[0]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (p + k < cols) wp[k] = out[0].h[k];
    }
  }
};

// X' = (a + E) X + B'X, tile rows p along the columns of the matrix as laid out and
// q along its rows.
template <class C, int PROD, bool LAST>
__global__ __launch_bounds__(C::THREADS, C::OCC) void ns_x(const NsDev dv, int cur, float ca,
                                                           float keep) {
  constexpr int PARTS = PROD == 3 ? 2 : 1;
  __shared__ __attribute__((aligned(1024))) char lds[NtEpi<C, PARTS>::LDS];
  int t;
  const NsJob* jp = ns_job(dv, &t);
  if (!jp) return;
  const NsJob& j = *jp;
  t -= j.t_x;
  // four tiles of rows p at a time, their rows q in turn
  const int tp = (j.cp + C::BP - 1) / C::BP, tq = (j.rp + C::BQ - 1) / C::BQ;
  const int g = t / (4 * tq), w = t - g * 4 * tq;
  const int gw = tp - 4 * g < 4 ? tp - 4 * g : 4;
  const int pt = (4 * g + w % gw) * C::BP, qt = (w / gw) * C::BQ;
  const int tall = j.tall, m = tall ? j.cp : j.rp;
  const h16* bh = at<h16>(dv.ws, j.b);
  const h16* bl = at<h16>(dv.ws, j.bl);
  // X^T as [n][m]: the transpose, or a tall matrix as laid out
  const h16* xh = at<h16>(dv.ws, tall ? j.nat[cur] : j.mir[cur]);
  const h16* xl = at<h16>(dv.ws, tall ? j.natl[cur] : j.mirl[cur]);
  const int64_t po = (int64_t)pt * m, qo = (int64_t)qt * m;
  NtTile<PROD> nt;
  if (PROD == 3) {
    nt.p[0] = (tall ? bh : xh) + po;
    nt.q[0] = (tall ? xl : bl) + qo;
    nt.p[PROD / 2] = (tall ? bl : xl) + po;
    nt.q[PROD / 2] = (tall ? xh : bh) + qo;
  }
  nt.p[PROD - 1] = (tall ? bh : xh) + po;
  nt.q[PROD - 1] = (tall ? xh : bh) + qo;
  nt.ldp = nt.ldq = (uint32_t)m * 2u;
  nt.prows = j.cp - pt;
  nt.qrows = j.rp - qt;
  nt.kbytes = m * 2;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C, PROD>(nt, lds, acc);
  const int wave = threadIdx.x >> 6;
  if (wave >= C::WAVES) return;
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
  epi.whole = j.whole;
  h16* mir[PARTS];
  mir[0] = at<h16>(dv.ws, j.mir[mn]);
  mir[PARTS - 1] = at<h16>(dv.ws, PARTS == 2 ? j.mirl[mn] : j.mir[mn]);
  nt_store<C, PARTS>(acc, lds, pt + (wave / C::WQ) * 32 * C::TP, qt + (wave % C::WQ) * 32 * C::TQ,
                     j.cp, j.rp, !LAST, mir, j.rp, epi);
}

// ---- the plan ------------------------------------------------------------------

int up(int v, int t) { return (v + t - 1) / t * t; }

// The tiles a product may run on: workgroups the device holds at once, microseconds
// a 128-byte slice of the reduction takes and a launch takes besides.
constexpr NsTile kNsTiles[5] = {{256, 1, 256, 1.15, 12.0},
                                {192, 1, 256, 0.75, 9.0},
                                {128, 1, 512, 0.72, 6.0},
                                {64, 1, 512, 0.40, 4.0},
                                {64, 2, 256, 0.30, 5.0}};

// The tile that a product of the set finishes soonest on, by that estimate: rounds
// of workgroups over the device, or the longest reduction if that takes longer.
// stage 0: A, 1: B, 2: X'.
NsTile ns_choose(int stage, int count, const int32_t* rows, const int32_t* cols, int products) {
  NsTile best = kNsTiles[0];
  double bt = 0;
  for (const NsTile& c : kNsTiles) {
    double work = 0, longest = 0;
    for (int i = 0; i < count; ++i) {
      const int m = up(std::min(rows[i], cols[i]), 64), n = up(std::max(rows[i], cols[i]), 64);
      const double tm = ceil_div(m, c.tile), tn = ceil_div(n, c.tile);
      const double k = ceil_div(products * ((stage == 0 ? n : m) / 64), c.groups);
      work += (stage == 2 ? tm * tn : tm * (tm + 1) / 2) * k;
      longest = std::max(longest, k);
    }
    const double t = c.fixed + c.slice * std::max(work / c.slots, longest);
    if (bt == 0 || t < bt) {
      bt = t;
      best = c;
    }
  }
  return best;
}

template <class C, int PROD>
void ns_launch(int stage, bool last, const NsDev& d, int cur, float ca, float cb, float cc,
               float keep, hipStream_t st) {
  const dim3 grid((unsigned)(8 * ((d.tiles + 7) / 8))), block(C::THREADS);
  if (stage == 0)
    hipLaunchKernelGGL((ns_sym<C, 0, PROD>), grid, block, 0, st, d, cb, cc);
  else if (stage == 1)
    hipLaunchKernelGGL((ns_sym<C, 1, PROD>), grid, block, 0, st, d, cb, cc);
  else if (!last)
    hipLaunchKernelGGL((ns_x<C, PROD, false>), grid, block, 0, st, d, cur, ca, keep);
  else
    hipLaunchKernelGGL((ns_x<C, PROD, true>), grid, block, 0, st, d, cur, ca, keep);
}

template <int PROD>
hipError_t ns_run(const NsPlan& p, const NsArgs& a, char* ws, hipStream_t st) {
  const NsDev pre{ws, p.table, p.map_pre, p.n_pre};
  hipLaunchKernelGGL((ns_split<PROD>), dim3((unsigned)p.n_pre), dim3(256), 0, st, pre, a.momentum,
                     a.nesterov);
  const NsDev sym{ws, p.table, p.map_sym, p.n_sym}, x{ws, p.table, p.map_x, p.n_x};
  for (int s = 0; s < a.steps; ++s) {
    const float ca = a.coef[3 * s], cb = a.coef[3 * s + 1], cc = a.coef[3 * s + 2];
    for (int stage = 0; stage < 3; ++stage) {
      const NsDev& d = stage == 2 ? x : sym;
      const NsTile& k = p.kind[stage];
      const bool last = s + 1 == a.steps;
      if (k.tile == 256)
        ns_launch<Nt256, PROD>(stage, last, d, s & 1, ca, cb, cc, a.keep, st);
      else if (k.tile == 192)
        ns_launch<Nt192, PROD>(stage, last, d, s & 1, ca, cb, cc, a.keep, st);
      else if (k.tile == 128)
        ns_launch<Nt128, PROD>(stage, last, d, s & 1, ca, cb, cc, a.keep, st);
      else if (k.groups == 1)
        ns_launch<Nt64, PROD>(stage, last, d, s & 1, ca, cb, cc, a.keep, st);
      else
        ns_launch<Nt64k, PROD>(stage, last, d, s & 1, ca, cb, cc, a.keep, st);
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
  // (A and B share their tiles' map, so their tile sides are one choice)
  P.kind[0] = ns_choose(0, count, rows, cols, products);
  P.kind[1] = ns_choose(1, count, rows, cols, products);
  if (P.kind[1].tile != P.kind[0].tile) P.kind[1] = P.kind[0];
  P.kind[2] = ns_choose(2, count, rows, cols, products);
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
  P.n_sym = P.n_x = P.n_pre = 0;
  for (int i = 0; i < count; ++i) {
    NsJob& j = P.jobs[i];
    const int o = P.order[i];
    j = NsJob{};
    j.rows = rows[o];
    j.cols = cols[o];
    j.tall = j.rows > j.cols;
    j.rp = up(j.rows, 64);
    j.cp = up(j.cols, 64);
    const int m = j.tall ? j.cp : j.rp, tm = ceil_div(m, P.kind[0].tile);
    j.t_sym = P.n_sym;
    j.t_x = P.n_x;
    j.t_pre = P.n_pre;
    P.n_sym += tm * (tm + 1) / 2;
    P.n_x += ceil_div(j.rp, P.kind[2].tile) * ceil_div(j.cp, P.kind[2].tile);
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
  P.map_sym = take((uint64_t)P.n_sym * 2);
  P.map_x = take((uint64_t)P.n_x * 2);
  P.map_pre = take((uint64_t)P.n_pre * 2);
  P.bytes = (size_t)off * 256;
}

hipError_t launch_ns(const NsPlan& p, const NsArgs& a, void* ws, hipStream_t st) {
  char* w = static_cast<char*>(ws);
  const NsPlaces pl{p.table, p.map_sym, p.map_x, p.map_pre, p.kind[0].tile, p.kind[2].tile};
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
