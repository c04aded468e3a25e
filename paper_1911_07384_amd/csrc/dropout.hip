// Dropout from a counter-based generator (philox.hpp): y = kept ? fl(x * scale) : +0,
// plus the residual if there is one, rounded once.  The gradient is the same call on
// dy.
//
// A lane takes the 8 elements of one block of the generator: 16 bytes in, 16 out, nothing
// kept.  Bound by its bytes: 2^27 elements 81 us (6.6 TB/s; a large copy reaches 5.1), with a
// residual 136 (5.9).  The block's 20 products of 32 bits take 0.4 times as long and hide
// behind the loads; 128 x 2048 elements take 2.0 us, a launch's.

#include "head.hpp"

namespace fp16k {
namespace {

constexpr int kThreads = 256;

template <bool RES>
__global__ __launch_bounds__(kThreads) void dropout_kernel(int64_t n, const h16* x,
                                                           const h16* residual, h16* y, Drop d) {
  const uint64_t seed = d.state[0], step = d.state[1];
  const int64_t g = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t left = n - g * 8;
  if (left <= 0) return;
  const bool whole = left >= 8;
  const V8 v = whole ? load16(x + g * 8) : load8_upto(x + g * 8, (int)left);
  V8 r = zero8();
  if (RES) r = whole ? load16(residual + g * 8) : load8_upto(residual + g * 8, (int)left);
  const PhiloxBlock b = philox((uint32_t)g, d.site, step, seed);
  V8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float f = kept(b, e, d.threshold) ? to_f32(v.h[e]) * d.scale : 0.0f;
    if (RES) f = f + to_f32(r.h[e]);
    o.h[e] = to_h16(f);
  }
  if (whole)
    store16(y + g * 8, o);
  else
    store8_upto(y + g * 8, o, (int)left);
}

__global__ void rng_advance_kernel(uint64_t* state, uint64_t steps) { state[1] += steps; }

}  // namespace

hipError_t launch_dropout(int64_t n, const h16* x, const h16* residual, h16* y, const Drop& d,
                          hipStream_t st) {
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)ceil_div64(ceil_div64(n, 8), kThreads));
  if (residual)
    dropout_kernel<true><<<grid, kThreads, 0, st>>>(n, x, residual, y, d);
  else
    dropout_kernel<false><<<grid, kThreads, 0, st>>>(n, x, residual, y, d);
  return hipGetLastError();
}

hipError_t launch_rng_advance(uint64_t* state, uint64_t steps, hipStream_t st) {
  rng_advance_kernel<<<1, 1, 0, st>>>(state, steps);
  return hipGetLastError();
}

}  // namespace fp16k
