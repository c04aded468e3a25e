// Dense layers: y = drop(act(x W^T + bias)) + residual in one product, and the
// gradients of x, W and bias.
//
//   forward   z = x W^T + bias       rows of both operands run along the reduction
//   dx        dz W                   W's columns do
//   dW        dz^T x                 both operands' columns do
//   with dz = drop(dy) act'(z), a pass over the elements that also sums its columns for
//   dbias.

#include "head.hpp"

namespace fp16k {
namespace {

// ---- activations -------------------------------------------------------------------

// (Past these the values are their limits: -0 and z, slopes 0 and 1; the formulas would
// multiply an infinity by 0.)
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == kActRelu) return relu_keep_nan(z);
  if (act == kActGelu) return z < -15.0f ? -0.0f : 0.5f * z * erfcf(z * -0.70710678f);
  if (act == kActSilu) return z < -110.0f ? -0.0f : z / (1.0f + expf(-z));
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  if (act == kActRelu) return z > 0.0f ? 1.0f : __builtin_isnan(z) ? z : 0.0f;
  if (act == kActGelu) {
    if (__builtin_fabsf(z) > 15.0f) return z > 0.0f ? 1.0f : 0.0f;
    return 0.5f * erfcf(z * -0.70710678f) + z * (0.39894228f * expf(-0.5f * z * z));
  }
  if (act == kActSilu) {
    if (__builtin_fabsf(z) > 110.0f) return z > 0.0f ? 1.0f : 0.0f;
    const float s = 1.0f / (1.0f + expf(-z));
    return s * (1.0f + z * (1.0f - s));
  }
  return 1.0f;
}

// ---- the product -------------------------------------------------------------------

// D[q][p] = sum_k P(p, k) Q(q, k), P(p, k) = P[p * ldp + k], or P[k * ldp + p] with PS
// (likewise Q), D's rows ldd apart.
struct Product {
  const h16 *p, *q;
  int64_t ldp, ldq;
  int np, nq, nk;
};

struct ToHalf {  // rounded and stored
  h16* d;
  int64_t ldd;
  __device__ __forceinline__ void operator()(int p, int q, float v) const {
    d[q * ldd + p] = to_h16(v);
  }
};

struct Forward {
  const h16 *bias, *residual;
  h16 *y, *z;
  int64_t ldd;
  int act;
  Drop drop;
  __device__ __forceinline__ void operator()(int p, int q, float v) const {
    if (bias) v = v + to_f32(bias[p]);
    const int64_t i = q * ldd + p;
    if (z) z[i] = to_h16(v);
    v = act_value(act, v);
    if (drop.threshold) {
      const PhiloxBlock b = philox((uint32_t)(i >> 3), drop.site, drop.state[1], drop.state[0]);
      v = kept(b, (int)(i & 7), drop.threshold) ? v * drop.scale : 0.0f;
    }
    if (residual) v = v + to_f32(residual[i]);
    y[i] = to_h16(v);
  }
};

constexpr int kSide = 64, kDeep = 32, kLd = kDeep + 8;

// A tile's 64 rows x 32 of one operand into LDS, [row][k], zeros past its ends.
template <bool S>
__device__ __forceinline__ void stage(h16* to, const h16* m, int64_t ld, int r0, int rows, int k0,
                                      int nk) {
  const int t = threadIdx.x;
  if (!S) {
    const int r = t >> 2, k = (t & 3) * 8;
    const V8 v = r0 + r < rows && k0 + k < nk ? load8_upto(m + (r0 + r) * ld + k0 + k, nk - k0 - k)
                                              : zero8();
    store16(to + r * kLd + k, v);
  } else {
    const int k = t >> 3, r = (t & 7) * 8;
    const V8 v = k0 + k < nk && r0 + r < rows ? load8_upto(m + (k0 + k) * ld + r0 + r, rows - r0 - r)
                                              : zero8();
#pragma unroll
    for (int e = 0; e < 8; ++e) to[(r + e) * kLd + k] = v.h[e];
  }
}

template <bool PS, bool QS, class Epi>
__global__ __launch_bounds__(256) void product_kernel(const Product a, const Epi epi) {
  __shared__ __attribute__((aligned(16))) h16 lp[kSide * kLd], lq[kSide * kLd];
  const int tp = (a.np + kSide - 1) / kSide;
  const int p0 = (blockIdx.x % tp) * kSide, q0 = (blockIdx.x / tp) * kSide;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lrow = lane & 31, lhi = lane >> 5, wp = (wave & 1) * 32, wq = (wave >> 1) * 32;
  floatx16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
  for (int k0 = 0; k0 < a.nk; k0 += kDeep) {
    stage<PS>(lp, a.p, a.ldp, p0, a.np, k0, a.nk);
    stage<QS>(lq, a.q, a.ldq, q0, a.nq, k0, a.nk);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const V8 fp = load16(lp + (wp + lrow) * kLd + s * 16 + lhi * 8);
      const V8 fq = load16(lq + (wq + lrow) * kLd + s * 16 + lhi * 8);
      acc = mfma32x32x16(fp.h, fq.h, acc);
    }
    __syncthreads();
  }
  const int q = q0 + wq + lrow;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int p = p0 + wp + 8 * (e >> 2) + 4 * lhi + (e & 3);
    if (p < a.np && q < a.nq) epi(p, q, acc[e]);
  }
}

template <bool PS, bool QS, class Epi>
hipError_t launch_product(const Product& a, const Epi& epi, hipStream_t st) {
  const int64_t tiles = ceil_div64(a.np, kSide) * ceil_div64(a.nq, kSide);
  product_kernel<PS, QS><<<(unsigned)tiles, 256, 0, st>>>(a, epi);
  return hipGetLastError();
}

// ---- dz and dbias --------------------------------------------------------------------

constexpr int kRows = 64;  // of a workgroup's partial sums

// dz (unless null) and its columns' sums over kRows rows (unless null), 256 columns a
// workgroup.
__global__ __launch_bounds__(256) void dz_kernel(int tokens, int outputs, int act, Drop drop,
                                                 const h16* z, const h16* dy, h16* dz, float* part) {
  const int c = blockIdx.x * 256 + threadIdx.x, r0 = blockIdx.y * kRows;
  if (c >= outputs) return;
  float sum = 0.0f;
  for (int r = r0; r < r0 + kRows && r < tokens; ++r) {
    const int64_t i = (int64_t)r * outputs + c;
    float v = to_f32(dy[i]);
    if (drop.threshold) {
      const PhiloxBlock b = philox((uint32_t)(i >> 3), drop.site, drop.state[1], drop.state[0]);
      v = kept(b, (int)(i & 7), drop.threshold) ? v * drop.scale : 0.0f;
    }
    if (act != kActNone) v *= act_slope(act, to_f32(z[i]));
    if (dz) dz[i] = to_h16(v);
    sum += v;
  }
  if (part) part[(int64_t)blockIdx.y * outputs + c] = sum;
}

__global__ __launch_bounds__(256) void dbias_kernel(int outputs, int parts, const float* part,
                                                    h16* dbias) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= outputs) return;
  double s = 0.0;
  for (int i = 0; i < parts; ++i) s += (double)part[(int64_t)i * outputs + c];
  dbias[c] = dbl_to_h16(s);
}

size_t dz_bytes(int tokens, int outputs) {
  return ((size_t)tokens * outputs * 2 + 255) & ~(size_t)255;
}

}  // namespace

size_t dense_fwd_ws_bytes(int, int, int) { return 0; }

size_t dense_bwd_ws_bytes(int tokens, int inputs, int outputs, bool dz) {
  return (dz ? dz_bytes(tokens, outputs) : 0) +
         (size_t)ceil_div(tokens, kRows) * outputs * sizeof(float);
}

hipError_t launch_dense_fwd(const DenseArgs& a, hipStream_t st) {
  const Product p = {a.w, a.x, a.inputs, a.inputs, a.outputs, a.tokens, a.inputs};
  return launch_product<false, false>(
      p, Forward{a.bias, a.residual, a.y, a.z, a.outputs, a.act, a.drop}, st);
}

hipError_t launch_dense_bwd(const DenseArgs& a, hipStream_t st) {
  const bool makes = a.act != kActNone || a.drop.threshold;
  const h16* dz = a.dy;
  h16* made = makes ? static_cast<h16*>(a.ws) : nullptr;
  float* part = reinterpret_cast<float*>(static_cast<char*>(a.ws) +
                                         (makes ? dz_bytes(a.tokens, a.outputs) : 0));
  if (makes || a.dbias) {
    const int parts = ceil_div(a.tokens, kRows);
    dz_kernel<<<dim3((unsigned)ceil_div(a.outputs, 256), (unsigned)parts), 256, 0, st>>>(
        a.tokens, a.outputs, a.act, a.drop, a.kept, a.dy, made, a.dbias ? part : nullptr);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.dbias) {
      dbias_kernel<<<(unsigned)ceil_div(a.outputs, 256), 256, 0, st>>>(a.outputs, parts, part,
                                                                       a.dbias);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  if (makes) dz = made;
  if (a.dx) {
    const Product p = {a.w, dz, a.inputs, a.outputs, a.inputs, a.tokens, a.outputs};
    const hipError_t e = launch_product<true, false>(p, ToHalf{a.dx, a.inputs}, st);
    if (e != hipSuccess) return e;
  }
  if (a.dw) {
    const Product p = {a.x, dz, a.inputs, a.outputs, a.inputs, a.outputs, a.tokens};
    return launch_product<true, true>(p, ToHalf{a.dw, a.inputs}, st);
  }
  return hipSuccess;
}

}  // namespace fp16k
