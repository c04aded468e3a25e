// Internal launch interface of a network's dense head: dense layers with an epilogue
// (dense.hip), dropout (dropout.hip) and log probabilities (logprob.hip).  Arguments
// have already been validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.hpp"
#include "philox.hpp"

namespace fp16k {

// ---- dropout (dropout.hip) ---------------------------------------------------------
hipError_t launch_dropout(int64_t n, const h16* x, const h16* residual, h16* y, const Drop& d,
                          hipStream_t st);
hipError_t launch_rng_advance(uint64_t* state, uint64_t steps, hipStream_t st);

// ---- dense layers (dense.hip) ------------------------------------------------------
enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

struct DenseArgs {
  int tokens, inputs, outputs, act;
  Drop drop;
  const h16 *x, *w, *bias, *residual;
  h16 *y, *z;              // forward
  const h16 *kept, *dy;    // backward: the forward's z, and dy
  h16 *dx, *dw, *dbias;
  void* ws;
};
size_t dense_fwd_ws_bytes(int tokens, int inputs, int outputs);
size_t dense_bwd_ws_bytes(int tokens, int inputs, int outputs, bool dz);
// The kernel of a product (0 forward, 1 dx, 2 dW).
void dense_name(int tokens, int inputs, int outputs, int product, char* name, size_t size);
hipError_t launch_dense_fwd(const DenseArgs& a, hipStream_t st);
hipError_t launch_dense_bwd(const DenseArgs& a, hipStream_t st);

// ---- log probabilities (logprob.hip) -----------------------------------------------
constexpr int kTopMax = 64;

struct LogprobArgs {
  int rows, classes;
  int64_t stride;
  float scale;
  int top;
  const h16* z;
  const int32_t* token;
  float *logp, *stats;
  int32_t* top_id;
  float* top_logp;
  const float *dlogp, *dentropy;  // backward
  h16* dz;
  void* ws;
};
size_t logprob_ws_bytes(int rows, int classes, int top);
hipError_t launch_logprob(const LogprobArgs& a, hipStream_t st);
hipError_t launch_logprob_bwd(const LogprobArgs& a, hipStream_t st);

}  // namespace fp16k
