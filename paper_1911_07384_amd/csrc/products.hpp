// Internal launch interface of the matrix-product operators beside the
// convolutions: orthogonalised momentum (muon.hip) and 8-bit integer dense
// layers (int8.hip).  Arguments have already been validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.hpp"

namespace fp16k {

// ---- orthogonalised momentum (muon.hip) --------------------------------------
constexpr int kNsMaxJobs = 1024, kNsMaxSteps = 32, kNsMaxSide = 65536, kNsMaxShort = 16384;
constexpr int kNsParts = 256;  // partial sums of a matrix's squares, at most

// One matrix [rows][cols].  Workspace arrays are given in units of 256 bytes from
// the workspace's start; "nat" holds X as the matrix is laid out, "mir" its
// transpose, each padded with zeros to multiples of 64, [rp][cp] ([cp][rp]); the operand of the
// update that is not also its elementwise argument alternates between two.
struct NsJob {
  const h16* g;  // the gradient, or the matrix itself
  h16* m;        // the momentum, or null
  h16* w;        // the weights, or the result
  float alpha;   // factor of the orthogonalised matrix
  int rows, cols, rp, cp, tall;
  uint32_t nat[2], mir[2], natl[2], mirl[2];  // X (high parts, low parts)
  uint32_t a, al, b, bl;                      // A and B off the diagonal
  uint32_t d, e;                              // their diagonals, float32
  uint32_t part;                              // float64 partial sums
  int nparts;
  int t[3], t_pre;  // its first tile in the launches for A, B, X' and the first pass
};

// A square tile that a product may run on: its side, the parts of the reduction,
// workgroups a CU holds, and times in microseconds (see ns_choose).
struct NsTile {
  const char* name;
  int side, parts, occ;
  double alone, cu, fixed[2], sums;
  bool a_only;
};

struct NsPlan {
  NsTile kind[3];              // of A, B and X'
  int variant[3];              // their places in the list of tiles
  int count;
  bool small;                  // one workgroup a matrix, none of the rest
  int tiles[3], n_pre;         // in all
  uint32_t table, map[3], map_pre, sums;  // in the workspace
  size_t bytes;
  int* order;                  // [count]: jobs[i] is the caller's matrix order[i]
  NsJob* jobs;                 // [count]
};

// Fills the plan's sizes, tiles and workspace places from rows[i], cols[i], and order
// and jobs, which are the caller's (a list may be long, and its stack short).
void ns_plan(int count, const int32_t* rows, const int32_t* cols, int products, NsPlan* plan);

struct NsArgs {
  int steps, products;
  const float* coef;  // [steps][3], host
  float momentum, keep;
  int nesterov;
};
hipError_t launch_ns(const NsPlan& plan, const NsArgs& a, void* ws, hipStream_t st);

// ---- 8-bit integer dense layers (int8.hip) ------------------------------------
constexpr int kI8MaxK = 131071;  // 32-bit sums of products of bytes: k * 2^14 < 2^31
inline int64_t i8_row(int64_t n) { return (n + 15) & ~(int64_t)15; }  // bytes of a row

// x [rows][cols] by rows: q [rows][i8_row(cols)] and scale [rows].
hipError_t launch_i8_rows(int rows, int cols, const h16* x, int8_t* q, float* scale,
                          hipStream_t st);
// x [rows][cols] by columns, qc [cols][i8_row(rows)] and scale_c [cols]; and unless
// qr is null by rows, qr [rows][i8_row(cols)] and scale_r [rows]; sum (nullable): the
// columns' sums, rounded.  ws: i8_cols_ws_bytes.  Up to two of them in a launch.
struct I8Cols {
  int rows, cols, per, chunks, ldc, ldr;
  const h16* x;
  int8_t *qc, *qr;
  float *scale_c, *scale_r;
  h16* sum;
  uint32_t *cmag, *rmag;  // largest magnitudes: [chunks][cols], [cols / 256][rows]
  float* psum;            // sums: [chunks][cols]
};
struct I8Both {
  I8Cols job[2];
};
size_t i8_cols_ws_bytes(int rows, int cols, bool by_rows, bool sum);
I8Cols i8_cols_job(int rows, int cols, const h16* x, int8_t* qc, float* scale_c, int8_t* qr,
                   float* scale_r, h16* sum, void* ws);
hipError_t launch_i8_cols(const I8Cols* jobs, int count, hipStream_t st);
// y [m][n] = rne16(sa sb (a b^T) + bias): a [m][i8_row(k)], b [n][i8_row(k)].
struct I8Product {
  int m, n, k;
  const int8_t *a, *b;
  const float *sa, *sb;
  const h16* bias;
  h16* y;
};
hipError_t launch_i8_product(const I8Product& a, hipStream_t st);
const char* i8_product_name(int m, int n, int k);
// Whether a product of few rows quantises its binary16 rows itself, and that call.
bool i8_fused_ok(int m, int n, int k);
hipError_t launch_i8_fused(const I8Product& a, const h16* x, hipStream_t st);

}  // namespace fp16k
