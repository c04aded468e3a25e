// C ABI of a network's dense head: dense layers with an epilogue, dropout, log
// probabilities.  Argument validation, workspace places and dispatch; nothing here
// allocates device memory.

#include "../../include/fp16train.h"
#include "api_util.hpp"
#include "head.hpp"

using namespace fp16k;

namespace {

constexpr int32_t kMaxSide = 1 << 20;          // of a dense layer's sizes
// Elements of a tensor: below 2^32 threads of a launch over its groups of 8, for two
// matrices in one launch (rows laid out anew) too.
constexpr int64_t kMaxElems = (int64_t)1 << 34;

const h16* hp(const fp16_t* p) { return reinterpret_cast<const h16*>(p); }
h16* hp(fp16_t* p) { return reinterpret_cast<h16*>(p); }

// Buffers of one call.  A written one may overlap no other, but one of `same` may be
// the buffer of its own that it is written from.
struct Buf {
  const void* p;
  size_t bytes;
  bool written;
  int same = -1;
};
template <int N>
fp16_status bufs_ok(const Buf (&b)[N]) {
  for (int i = 0; i < N; ++i)
    if (!aligned16(b[i].p)) return FP16_ERR_MISALIGNED;
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N; ++j) {
      if (i == j || !b[i].written || (b[i].same == j && b[i].p == b[j].p)) continue;
      if (overlap(b[i].p, b[i].bytes, b[j].p, b[j].bytes)) return FP16_ERR_ALIASING;
    }
  return FP16_OK;
}

fp16_status ws_ok(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return FP16_OK;
  if (!ws || ws_bytes < need) return FP16_ERR_WORKSPACE;
  return aligned16(ws) ? FP16_OK : FP16_ERR_MISALIGNED;
}

bool probability(float p) { return p >= 0.0f && p <= 1.0f; }
bool rng_aligned(const void* p) { return ((uintptr_t)p & 7u) == 0; }

bool dense_ok(const fp16_dense_desc* d) {
  const int64_t t = d->tokens, i = d->inputs, o = d->outputs;
  return t >= 1 && i >= 1 && o >= 1 && t <= kMaxSide && i <= kMaxSide && o <= kMaxSide &&
         t * i < kMaxElems && t * o < kMaxElems && i * o < kMaxElems && d->act >= FP16_ACT_NONE &&
         d->act <= FP16_ACT_SILU && probability(d->drop);
}

bool makes_dz(const fp16_dense_desc* d) {
  return d->act != FP16_ACT_NONE || make_drop(d->drop, 0, nullptr).threshold != 0;
}

size_t dense_need(const fp16_dense_desc* d, int call) {
  return call == FP16_DENSE_FWD ? dense_fwd_ws_bytes(d->tokens, d->inputs, d->outputs)
                                : dense_bwd_ws_bytes(d->tokens, d->inputs, d->outputs, makes_dz(d));
}

DenseArgs dense_args(const fp16_dense_desc* d, const uint64_t* rng, void* ws) {
  DenseArgs a = {};
  a.tokens = d->tokens;
  a.inputs = d->inputs;
  a.outputs = d->outputs;
  a.act = d->act;
  a.drop = make_drop(d->drop, d->site, rng);
  a.ws = ws;
  return a;
}

bool logprob_ok(const fp16_logprob_desc* d) {
  return d->rows >= 1 && d->rows < (1 << 24) && d->classes >= 1 && d->classes <= kMaxSide &&
         d->stride >= d->classes && d->stride <= 2 * kMaxSide &&
         (int64_t)d->rows * d->stride < kMaxElems && d->scale > 0.0f && d->scale <= 1e30f &&
         d->top >= 0 && d->top <= FP16_LOGPROB_TOP_MAX && d->top <= d->classes;
}

// Bytes of a logits buffer, up to its last row's last class.
size_t logits_bytes(const fp16_logprob_desc* d) {
  return ((size_t)(d->rows - 1) * d->stride + d->classes) * 2;
}

LogprobArgs logprob_args(const fp16_logprob_desc* d, const fp16_t* z, const int32_t* tokens) {
  LogprobArgs a = {};
  a.rows = d->rows;
  a.classes = d->classes;
  a.stride = d->stride;
  a.scale = d->scale;
  a.top = d->top;
  a.z = hp(z);
  a.token = tokens;
  return a;
}

static_assert(FP16_LOGPROB_TOP_MAX == kTopMax, "limits");
static_assert(FP16_ACT_NONE == kActNone && FP16_ACT_RELU == kActRelu &&
                  FP16_ACT_GELU == kActGelu && FP16_ACT_SILU == kActSilu,
              "activations");

}  // namespace

extern "C" {

fp16_status fp16_dropout(size_t n, const fp16_t* x, const fp16_t* residual, fp16_t* y, float p,
                         const uint64_t* rng, uint32_t site, fp16_stream_t stream) {
  if (n >= (size_t)kMaxElems || !probability(p)) return FP16_ERR_SHAPE;
  if (n == 0) return FP16_OK;
  if (!x || !y || !rng) return FP16_ERR_NULL;
  if (!rng_aligned(rng)) return FP16_ERR_MISALIGNED;
  // y may be x or the residual (each element is read before its place is written)
  const Buf b[] = {{x, n * 2, false},
                   {residual, residual ? n * 2 : 0, false},
                   {y, n * 2, true, y == residual ? 1 : 0}};
  const fp16_status s = bufs_ok(b);
  if (s != FP16_OK) return s;
  if (overlap(y, n * 2, rng, 16)) return FP16_ERR_ALIASING;
  return hip_status(launch_dropout((int64_t)n, hp(x), hp(residual), hp(y), make_drop(p, site, rng),
                                   static_cast<hipStream_t>(stream)));
}

fp16_status fp16_rng_advance(uint64_t* rng, uint64_t steps, fp16_stream_t stream) {
  if (!rng) return FP16_ERR_NULL;
  if (!rng_aligned(rng)) return FP16_ERR_MISALIGNED;
  return hip_status(launch_rng_advance(rng, steps, static_cast<hipStream_t>(stream)));
}

size_t fp16_dense_workspace_bytes(const fp16_dense_desc* desc, int32_t call) {
  if (!desc || !dense_ok(desc) || (call != FP16_DENSE_FWD && call != FP16_DENSE_BWD)) return 0;
  return dense_need(desc, call);
}

fp16_status fp16_dense_fwd(const fp16_dense_desc* desc, const fp16_t* x, const fp16_t* w,
                           const fp16_t* bias, const fp16_t* residual, const uint64_t* rng,
                           fp16_t* y, fp16_t* z, void* ws, size_t ws_bytes, fp16_stream_t stream) {
  if (!desc || !x || !w || !y) return FP16_ERR_NULL;
  if (!dense_ok(desc)) return FP16_ERR_SHAPE;
  DenseArgs a = dense_args(desc, rng, ws);
  if (a.drop.threshold && !rng) return FP16_ERR_NULL;
  if (!rng_aligned(rng)) return FP16_ERR_MISALIGNED;
  const size_t T = desc->tokens, I = desc->inputs, O = desc->outputs;
  const size_t need = dense_need(desc, FP16_DENSE_FWD);
  fp16_status s = ws_ok(ws, ws_bytes, need);
  if (s != FP16_OK) return s;
  const Buf b[] = {{x, T * I * 2, false},
                   {w, O * I * 2, false},
                   {bias, bias ? O * 2 : 0, false},
                   {residual, residual ? T * O * 2 : 0, false},
                   {y, T * O * 2, true, 3},
                   {z, z ? T * O * 2 : 0, true},
                   {need ? ws : nullptr, need, true}};
  s = bufs_ok(b);
  if (s != FP16_OK) return s;
  if (a.drop.threshold && (overlap(y, T * O * 2, rng, 16) || overlap(z, T * O * 2, rng, 16) ||
                           overlap(ws, need, rng, 16)))
    return FP16_ERR_ALIASING;
  a.x = hp(x);
  a.w = hp(w);
  a.bias = hp(bias);
  a.residual = hp(residual);
  a.y = hp(y);
  a.z = hp(z);
  return hip_status(launch_dense_fwd(a, static_cast<hipStream_t>(stream)));
}

fp16_status fp16_dense_bwd(const fp16_dense_desc* desc, const fp16_t* x, const fp16_t* w,
                           const fp16_t* z, const fp16_t* dy, const uint64_t* rng, fp16_t* dx,
                           fp16_t* dw, fp16_t* dbias, void* ws, size_t ws_bytes,
                           fp16_stream_t stream) {
  if (!desc || !dy || (dx && !w) || (dw && !x)) return FP16_ERR_NULL;
  if (!dense_ok(desc)) return FP16_ERR_SHAPE;
  DenseArgs a = dense_args(desc, rng, ws);
  const bool act = desc->act != FP16_ACT_NONE;
  if ((act && !z) || (a.drop.threshold && !rng)) return FP16_ERR_NULL;
  if (!rng_aligned(rng)) return FP16_ERR_MISALIGNED;
  if (!dx && !dw && !dbias) return FP16_OK;
  const size_t T = desc->tokens, I = desc->inputs, O = desc->outputs;
  const size_t need = dense_need(desc, FP16_DENSE_BWD);
  fp16_status s = ws_ok(ws, ws_bytes, need);
  if (s != FP16_OK) return s;
  const Buf b[] = {{dw ? x : nullptr, T * I * 2, false},
                   {dx ? w : nullptr, O * I * 2, false},
                   {act ? z : nullptr, T * O * 2, false},
                   {dy, T * O * 2, false},
                   {dx, T * I * 2, true},
                   {dw, O * I * 2, true},
                   {dbias, O * 2, true},
                   {need ? ws : nullptr, need, true}};
  s = bufs_ok(b);
  if (s != FP16_OK) return s;
  if (a.drop.threshold && (overlap(dx, T * I * 2, rng, 16) || overlap(dw, O * I * 2, rng, 16) ||
                           overlap(dbias, O * 2, rng, 16) || overlap(ws, need, rng, 16)))
    return FP16_ERR_ALIASING;
  a.x = hp(x);
  a.w = hp(w);
  a.kept = hp(z);
  a.dy = hp(dy);
  a.dx = hp(dx);
  a.dw = hp(dw);
  a.dbias = hp(dbias);
  return hip_status(launch_dense_bwd(a, static_cast<hipStream_t>(stream)));
}

const char* fp16_dense_kernel(const fp16_dense_desc* desc, int32_t product) {
  thread_local char name[48];
  if (!desc || !dense_ok(desc) || product < 0 || product > 2) return "";
  dense_name(desc->tokens, desc->inputs, desc->outputs, product, name, sizeof(name));
  return name;
}

size_t fp16_logprobs_workspace_bytes(const fp16_logprob_desc* desc) {
  if (!desc || !logprob_ok(desc)) return 0;
  return logprob_ws_bytes(desc->rows, desc->classes, desc->top);
}

fp16_status fp16_logprobs(const fp16_logprob_desc* desc, const fp16_t* z, const int32_t* tokens,
                          float* logp, float* stats, int32_t* top_id, float* top_logp, void* ws,
                          size_t ws_bytes, fp16_stream_t stream) {
  if (!desc || !z || !stats || (logp && !tokens)) return FP16_ERR_NULL;
  if (!logprob_ok(desc)) return FP16_ERR_SHAPE;
  if (desc->top && (!top_id || !top_logp)) return FP16_ERR_NULL;
  const size_t N = desc->rows, top = desc->top;
  const size_t need = logprob_ws_bytes(desc->rows, desc->classes, desc->top);
  fp16_status s = ws_ok(ws, ws_bytes, need);
  if (s != FP16_OK) return s;
  const Buf b[] = {{z, logits_bytes(desc), false},
                   {logp ? tokens : nullptr, N * 4, false},
                   {logp, N * 4, true},
                   {stats, N * 12, true},
                   {top ? top_id : nullptr, N * top * 4, true},
                   {top ? top_logp : nullptr, N * top * 4, true},
                   {need ? ws : nullptr, need, true}};
  s = bufs_ok(b);
  if (s != FP16_OK) return s;
  LogprobArgs a = logprob_args(desc, z, tokens);
  a.logp = logp;
  a.stats = stats;
  a.top_id = top_id;
  a.top_logp = top_logp;
  a.ws = ws;
  return hip_status(launch_logprob(a, static_cast<hipStream_t>(stream)));
}

fp16_status fp16_logprobs_bwd(const fp16_logprob_desc* desc, const fp16_t* z, const int32_t* tokens,
                              const float* stats, const float* dlogp, const float* dentropy,
                              fp16_t* dz, fp16_stream_t stream) {
  if (!desc || !z || !stats || !dz || (!dlogp && !dentropy) || (dlogp && !tokens))
    return FP16_ERR_NULL;
  if (!logprob_ok(desc)) return FP16_ERR_SHAPE;
  const size_t N = desc->rows;
  const Buf b[] = {{z, logits_bytes(desc), false},
                   {dlogp ? tokens : nullptr, N * 4, false},
                   {stats, N * 12, false},
                   {dlogp, N * 4, false},
                   {dentropy, N * 4, false},
                   {dz, logits_bytes(desc), true, 0}};
  const fp16_status s = bufs_ok(b);
  if (s != FP16_OK) return s;
  LogprobArgs a = logprob_args(desc, z, dlogp ? tokens : nullptr);
  a.stats = const_cast<float*>(stats);
  a.dlogp = dlogp;
  a.dentropy = dentropy;
  a.dz = hp(dz);
  return hip_status(launch_logprob_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
