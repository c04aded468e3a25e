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
  int tile;
};

__device__ __forceinline__ double ns_block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return ((red[0] + red[1]) + red[2]) + red[3];
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
    const int m = j.tall ? j.cp : j.rp, tm = m / pl.tile;
    const int nsym = tm * (tm + 1) / 2, nx = (j.rp / pl.tile) * (j.cp / pl.tile);
    const int npre = (j.rp / 64) * (j.cp / 64);
    for (int i = tid; i < nsym; i += 256) at<uint16_t>(ws, pl.map_sym)[j.t_sym + i] = (uint16_t)idx;
    for (int i = tid; i < nx; i += 256) at<uint16_t>(ws, pl.map_x)[j.t_x + i] = (uint16_t)idx;
    for (int i = tid; i < npre; i += 256) at<uint16_t>(ws, pl.map_pre)[j.t_pre + i] = (uint16_t)idx;
  }
  const bool has_m = j.m != nullptr;
  const int64_t n = (int64_t)j.rows * j.cols, nvec = n / 8;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < nvec; i += (int64_t)j.nparts * 256) {
    const V8 g = load16(j.g + i * 8);
    V8 m = zero8();
    if (has_m) {
      m = load16(j.m + i * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) m.h[e] = to_h16(__builtin_fmaf(mu, to_f32(m.h[e]), to_f32(g.h[e])));
      store16(j.m + i * 8, m);
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
  const bool has_m = j.m != nullptr, whole = j.cols % 8 == 0;
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

// Walks a wave's tiles in runs of 8 rows p of one column q: value(p, q, v[8]) gives
// the run's halves to store there (natural, out[q][p ..]) in n_out parts; with
// `mirror` the same halves go out[p][q ..] as well, through this wave's LDS.
template <class C, int PARTS, class Value>
__device__ __forceinline__ void ns_store(const typename NtHalf::Acc (&acc)[C::TP][C::TQ], char* lds,
                                         int p0, int q0, bool mirror, h16* const (&mir)[PARTS],
                                         int ldm, Value value) {
  constexpr int TP = C::TP, TQ = C::TQ, LD = 32 * TQ + 8;  // halves
  static_assert(PARTS * 32 * LD * 2 * C::WAVES <= C::LDS, "LDS");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lrow = lane & 31, lhi = lane >> 5;
  h16* buf = reinterpret_cast<h16*>(lds) + wave * (PARTS * 32 * LD);
#pragma unroll
  for (int a = 0; a < TP; ++a) {
#pragma unroll
    for (int b = 0; b < TQ; ++b) {
      unsigned v[16];
      nt_rows(acc[a][b], v);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int p = 32 * a + 16 * h + 8 * lhi, q = 32 * b + lrow;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = __builtin_bit_cast(float, v[8 * h + e]);
        V8 out[PARTS];
        value(p0 + p, q0 + q, f, out);
        if (mirror) {
#pragma unroll
          for (int s = 0; s < PARTS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) buf[s * 32 * LD + (16 * h + 8 * lhi + e) * LD + q] = out[s].h[e];
        }
      }
    }
    if (mirror) {
      nt_wave_sync();
#pragma unroll
      for (int s = 0; s < PARTS; ++s)
#pragma unroll
        for (int i = 0; i < 2 * TQ; ++i) {
          const int r = (i * 64 + lane) / (4 * TQ), c = (i * 64 + lane) % (4 * TQ);
          store16(mir[s] + (int64_t)(p0 + 32 * a + r) * ldm + q0 + c * 8,
                  load16(buf + s * 32 * LD + r * LD + c * 8));
        }
      nt_wave_sync();
    }
  }
}

// This workgroup's matrix and its tile of the launch, or -1.
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

// A = X X^T (STEP 0) or B = bA + cA^2 (STEP 1), off the diagonal, and the diagonal.
template <class C, int STEP, int PROD>
__global__ __launch_bounds__(C::THREADS, C::OCC) void ns_sym(const NsDev dv, int cur, float cb,
                                                             float cc) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
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
  nt.prows = nt.qrows = C::BP;
  nt.kbytes = k * 2;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C, PROD>(nt, lds, acc);
  constexpr int PARTS = PROD == 3 ? 2 : 1;
  const int wave = threadIdx.x >> 6;
  const int p0 = pt + (wave / C::WQ) * 32 * C::TP, q0 = qt + (wave % C::WQ) * 32 * C::TQ;
  h16* const oh = at<h16>(dv.ws, STEP == 0 ? j.a : j.b);
  h16* const ol = at<h16>(dv.ws, STEP == 0 ? j.al : j.bl);
  h16* mir[PARTS];
  mir[0] = oh;
  mir[PARTS - 1] = PARTS == 2 ? ol : oh;
  float* const d = at<float>(dv.ws, j.d);
  float* const ev = at<float>(dv.ws, j.e);
  ns_store<C, PARTS>(acc, lds, p0, q0, ti != tj, mir, m, [&](int p, int q, const float (&f)[8],
                                                            V8 (&out)[PARTS]) {
    const int64_t o = (int64_t)q * m + p;
    V8 va, vl;
    float dp[8], dq = 0.0f;
    if (STEP == 1) {
      va = load16(ah + o);
      if (PROD == 3) vl = load16(al + o);
      dq = d[q];
#pragma unroll
      for (int e = 0; e < 8; ++e) dp[e] = d[p + e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float r;
      if (STEP == 0) {
        r = f[e] * (kSa / (kSx * kSx));
        if (p + e == q) {
          d[q] = f[e] * (1.0f / (kSx * kSx));
          r = 0.0f;
        }
      } else {
        float a = to_f32(va.h[e]);
        if (PROD == 3) a += to_f32(vl.h[e]);
        a *= 1.0f / kSa;
        const float a2 = f[e] * (1.0f / (kSa * kSa));
        if (p + e == q) {
          ev[q] = __builtin_fmaf(cc, __builtin_fmaf(dq, dq, a2), cb * dq);
          r = 0.0f;
        } else {
          r = kSb * __builtin_fmaf(cc, __builtin_fmaf(dq + dp[e], a, a2), cb * a);
        }
      }
      out[0].h[e] = to_h16(r);
      if (PARTS == 2) out[PARTS - 1].h[e] = to_h16(r - to_f32(out[0].h[e]));
    }
    store16(oh + o, out[0]);
    if (PARTS == 2) store16(ol + o, out[PARTS - 1]);
  });
}

// X' = (a + E) X + B'X, tile rows p along the columns of the matrix as laid out and
// q along its rows.  LAST: the weights' update (or the result) instead of X'.
template <class C, int PROD, bool LAST>
__global__ __launch_bounds__(C::THREADS, C::OCC) void ns_x(const NsDev dv, int cur, float ca,
                                                           float keep) {
  __shared__ __attribute__((aligned(1024))) char lds[C::LDS];
  int t;
  const NsJob* jp = ns_job(dv, &t);
  if (!jp) return;
  const NsJob& j = *jp;
  t -= j.t_x;
  const int tp = j.cp / C::BP;
  // four tiles of rows p at a time, their rows q in turn
  const int tq = j.rp / C::BQ, g = t / (4 * tq), w = t - g * 4 * tq;
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
  nt.prows = C::BP;
  nt.qrows = C::BQ;
  nt.kbytes = m * 2;
  floatx16 acc[C::TP][C::TQ];
  nt_product<NtHalf, C, PROD>(nt, lds, acc);

  constexpr int PARTS = PROD == 3 ? 2 : 1;
  const int wave = threadIdx.x >> 6;
  const int p0 = pt + (wave / C::WQ) * 32 * C::TP, q0 = qt + (wave % C::WQ) * 32 * C::TQ;
  const int cp = j.cp, rows = j.rows, cols = j.cols;
  const int nc = tall ? cur : 0, nn = tall ? cur ^ 1 : 0;  // X as laid out, now and next
  const int lc = PROD == 3 ? nc : 0, ln = PROD == 3 ? nn : 0;
  const int mn = tall ? 0 : cur ^ 1;
  const h16* nh = at<h16>(dv.ws, j.nat[nc]);
  const h16* nl = at<h16>(dv.ws, j.natl[lc]);
  h16* const nho = at<h16>(dv.ws, j.nat[nn]);
  h16* const nlo = at<h16>(dv.ws, j.natl[ln]);
  const float* ev = at<float>(dv.ws, j.e);
  h16* mir[PARTS];
  mir[0] = at<h16>(dv.ws, j.mir[mn]);
  mir[PARTS - 1] = at<h16>(dv.ws, PARTS == 2 ? j.mirl[mn] : j.mir[mn]);
  h16* const wt = j.w;
  const bool update = j.m != nullptr, whole = cols % 8 == 0;
  const float alpha = j.alpha;
  ns_store<C, PARTS>(acc, lds, p0, q0, !LAST, mir, j.rp, [&](int p, int q, const float (&f)[8],
                                                             V8 (&out)[PARTS]) {
    const int64_t o = (int64_t)q * cp + p;
    if (LAST && (q >= rows || p >= cols)) return;
    const V8 vh = load16(nh + o), vl = load16(nl + o);
    float x[8];
    const float eq = tall ? 0.0f : ev[q];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float E = tall ? ev[p + e] : eq;
      const float h = to_f32(vh.h[e]), l = to_f32(vl.h[e]);
      // (products = 1: the low part takes part in aX only, as in B'X)
      const float y = __builtin_fmaf(PROD == 3 ? ca + E : ca, l, f[e] * (1.0f / kSb));
      x[e] = __builtin_fmaf(ca + E, h, y);
    }
    if (!LAST) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        out[0].h[e] = to_h16(x[e]);
        const h16 lo = to_h16(x[e] - to_f32(out[0].h[e]));
        if (PARTS == 2)
          out[PARTS - 1].h[e] = lo;
        else
          x[e] = to_f32(lo);
      }
      store16(nho + o, out[0]);
      V8 lo;
      if (PARTS == 2) {
        lo = out[PARTS - 1];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) lo.h[e] = (h16)x[e];
      }
      store16(nlo + o, lo);
    } else {
      h16* const wp = wt + (int64_t)q * cols + p;
      V8 v = zero8();
      if (update) {
        if (whole) {
          v = load16(wp);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (p + e < cols) v.h[e] = wp[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ox = x[e] * (1.0f / kSx);
        v.h[e] = to_h16(update ? __builtin_fmaf(-alpha, ox, keep * to_f32(v.h[e])) : alpha * ox);
      }
      if (whole) {
        store16(wp, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (p + e < cols) wp[e] = v.h[e];
      }
    }
  });
}

// ---- the plan ------------------------------------------------------------------

int up(int v, int t) { return (v + t - 1) / t * t; }

// Estimated time of one step with tiles of side T, in microseconds: rounds of
// workgroups over the device at so long a slice each.
struct NsTileCost {
  int tile, slots;
  double slice, fixed;
};
constexpr NsTileCost kNsTiles[3] = {{256, 256, 1.25, 8.0}, {128, 512, 0.70, 4.0}, {64, 768, 0.45, 3.0}};

double ns_cost(const NsTileCost& c, int count, const int32_t* rows, const int32_t* cols) {
  double work[3] = {0, 0, 0}, longest[3] = {0, 0, 0};
  for (int i = 0; i < count; ++i) {
    const int m = up(std::min(rows[i], cols[i]), c.tile), n = up(std::max(rows[i], cols[i]), c.tile);
    const double tm = m / c.tile, tn = n / c.tile, sym = tm * (tm + 1) / 2;
    const double w[3] = {sym * (n / 64), sym * (m / 64), tm * tn * (m / 64)};
    const double k[3] = {n / 64.0, m / 64.0, m / 64.0};
    for (int s = 0; s < 3; ++s) {
      work[s] += w[s];
      longest[s] = std::max(longest[s], k[s]);
    }
  }
  double t = 0;
  for (int s = 0; s < 3; ++s) t += c.fixed + c.slice * std::max(work[s] / c.slots, longest[s]);
  return t;
}

template <class C, int PROD>
hipError_t ns_steps(const NsPlan& p, const NsArgs& a, char* ws, hipStream_t st) {
  const NsDev sym{ws, p.table, p.map_sym, p.n_sym}, x{ws, p.table, p.map_x, p.n_x};
  const dim3 gs((unsigned)(8 * ((p.n_sym + 7) / 8))), gx((unsigned)(8 * ((p.n_x + 7) / 8)));
  for (int s = 0; s < a.steps; ++s) {
    const float ca = a.coef[3 * s], cb = a.coef[3 * s + 1], cc = a.coef[3 * s + 2];
    const int cur = s & 1;
    hipLaunchKernelGGL((ns_sym<C, 0, PROD>), gs, dim3(C::THREADS), 0, st, sym, cur, cb, cc);
    hipLaunchKernelGGL((ns_sym<C, 1, PROD>), gs, dim3(C::THREADS), 0, st, sym, cur, cb, cc);
    if (s + 1 < a.steps)
      hipLaunchKernelGGL((ns_x<C, PROD, false>), gx, dim3(C::THREADS), 0, st, x, cur, ca, a.keep);
    else
      hipLaunchKernelGGL((ns_x<C, PROD, true>), gx, dim3(C::THREADS), 0, st, x, cur, ca, a.keep);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int PROD>
hipError_t ns_run(const NsPlan& p, const NsArgs& a, char* ws, hipStream_t st) {
  const NsDev pre{ws, p.table, p.map_pre, p.n_pre};
  hipLaunchKernelGGL((ns_split<PROD>), dim3((unsigned)p.n_pre), dim3(256), 0, st, pre, a.momentum,
                     a.nesterov);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (p.tile == 256) return ns_steps<Nt256, PROD>(p, a, ws, st);
  if (p.tile == 128) return ns_steps<Nt128, PROD>(p, a, ws, st);
  return ns_steps<Nt64, PROD>(p, a, ws, st);
}

}  // namespace

void ns_plan(int count, const int32_t* rows, const int32_t* cols, int products, NsPlan* plan) {
  NsPlan& P = *plan;
  P.count = count;
  double best = 0;
  P.tile = 0;
  for (const NsTileCost& c : kNsTiles) {
    const double t = ns_cost(c, count, rows, cols);
    if (P.tile == 0 || t < best) {
      best = t;
      P.tile = c.tile;
    }
  }
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
    j.rp = up(j.rows, P.tile);
    j.cp = up(j.cols, P.tile);
    const int m = j.tall ? j.cp : j.rp, tm = m / P.tile;
    j.t_sym = P.n_sym;
    j.t_x = P.n_x;
    j.t_pre = P.n_pre;
    P.n_sym += tm * (tm + 1) / 2;
    P.n_x += (j.rp / P.tile) * (j.cp / P.tile);
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
  const NsPlaces pl{p.table, p.map_sym, p.map_x, p.map_pre, p.tile};
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
