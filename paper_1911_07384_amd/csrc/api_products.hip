// C ABI of the matrix-product operators beside the convolutions: orthogonalised
// momentum and 8-bit integer dense layers.  Argument validation, workspace places
// and dispatch; nothing here allocates device memory.

#include "../../include/fp16train.h"
#include "api_util.hpp"
#include "products.hpp"

#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>

using namespace fp16k;

namespace {

// ---- orthogonalised momentum ------------------------------------------------------

static_assert(FP16_MUON_MAX == kNsMaxJobs && FP16_MUON_MAX_STEPS == kNsMaxSteps, "limits");

bool ns_list_ok(int32_t count, const fp16_muon_desc* d, int32_t products) {
  if (count < 1 || count > kNsMaxJobs || !d || (products != 1 && products != 3)) return false;
  for (int i = 0; i < count; ++i)
    if (d[i].rows < 1 || d[i].cols < 1 || d[i].rows > kNsMaxSide || d[i].cols > kNsMaxSide ||
        std::min(d[i].rows, d[i].cols) > kNsMaxShort ||
        (int64_t)d[i].rows * d[i].cols >= ((int64_t)1 << 30) || !isfinite(d[i].scale))
      return false;
  return true;
}

// Buffers of one call: a written one may overlap no other.
struct Span {
  uintptr_t at;
  size_t bytes;
  bool written;
};

// A list's plan and spans, in one allocation of the list's size: a thread's stack need
// not hold a list of kNsMaxJobs.  false if the host has no memory for it.
struct NsHost {
  NsPlan plan;
  Span* spans = nullptr;  // [3 count + 1]
  void* block = nullptr;
  NsHost() = default;
  NsHost(const NsHost&) = delete;
  NsHost& operator=(const NsHost&) = delete;
  ~NsHost() { free(block); }

  bool make(int32_t count, const fp16_muon_desc* d, int32_t products) {
    static_assert(alignof(NsJob) <= 8 && sizeof(NsJob) % 8 == 0 && alignof(Span) == 8, "places");
    const size_t n = (size_t)count;
    block = malloc(n * (sizeof(NsJob) + 3 * sizeof(Span) + 3 * sizeof(int32_t)) + sizeof(Span));
    if (!block) return false;
    plan.jobs = static_cast<NsJob*>(block);
    spans = reinterpret_cast<Span*>(plan.jobs + n);
    plan.order = reinterpret_cast<int*>(spans + 3 * n + 1);
    int32_t *rows = plan.order + n, *cols = rows + n;
    for (int i = 0; i < count; ++i) {
      rows[i] = d[i].rows;
      cols[i] = d[i].cols;
    }
    ns_plan(count, rows, cols, products, &plan);
    return true;
  }
};

bool spans_clash(Span* s, int n) {
  std::sort(s, s + n, [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t wend = 0, rend = 0;  // furthest end of a written and of a read span so far
  for (int i = 0; i < n; ++i) {
    // (an input written in place is one span, see the callers)
    if (s[i].at < wend || (s[i].written && s[i].at < rend)) return true;
    uintptr_t& e = s[i].written ? wend : rend;
    e = std::max(e, s[i].at + s[i].bytes);
  }
  return false;
}

fp16_status ns_call(int32_t count, const fp16_muon_desc* descs, fp16_t* const* w,
                    const fp16_t* const* g, fp16_t* const* m, bool update, float lr, float momentum,
                    float weight_decay, int32_t nesterov, int32_t steps, const float* coef,
                    int32_t products, void* ws, size_t ws_bytes, fp16_stream_t stream) {
  if (count == 0) return FP16_OK;
  if (count < 0 || count > kNsMaxJobs) return FP16_ERR_SHAPE;
  if (!descs || !w || !g || (update && !m)) return FP16_ERR_NULL;
  if (!ns_list_ok(count, descs, products) || steps < 1 || steps > kNsMaxSteps || !isfinite(lr) ||
      !isfinite(momentum) || !isfinite(weight_decay))
    return FP16_ERR_SHAPE;
  float table[3 * kNsMaxSteps];
  for (int i = 0; i < 3 * steps; ++i) {
    constexpr float quintic[3] = {3.4445f, -4.7750f, 2.0315f};
    table[i] = coef ? coef[i] : quintic[i % 3];
    if (!isfinite(table[i])) return FP16_ERR_SHAPE;
  }
  for (int i = 0; i < count; ++i) {
    if (!w[i] || !g[i] || (update && !m[i])) return FP16_ERR_NULL;
    if (((uintptr_t)w[i] | (uintptr_t)g[i] | (update ? (uintptr_t)m[i] : 0)) & 1u)
      return FP16_ERR_MISALIGNED;
  }
  NsHost host;
  if (!host.make(count, descs, products)) return FP16_ERR_HIP;
  NsPlan& plan = host.plan;
  if (!ws || ws_bytes < plan.bytes) return FP16_ERR_WORKSPACE;
  if (!aligned16(ws)) return FP16_ERR_MISALIGNED;
  Span* const spans = host.spans;
  int n = 0;
  for (int i = 0; i < count; ++i) {
    const size_t b = (size_t)descs[i].rows * descs[i].cols * 2;
    spans[n++] = {(uintptr_t)w[i], b, true};
    if (update) spans[n++] = {(uintptr_t)m[i], b, true};
    if (update || w[i] != g[i]) spans[n++] = {(uintptr_t)g[i], b, false};
  }
  spans[n++] = {(uintptr_t)ws, plan.bytes, true};
  if (spans_clash(spans, n)) return FP16_ERR_ALIASING;
  for (int i = 0; i < count; ++i) {
    const int o = plan.order[i];
    plan.jobs[i].g = reinterpret_cast<const h16*>(g[o]);
    plan.jobs[i].w = reinterpret_cast<h16*>(w[o]);
    plan.jobs[i].m = update ? reinterpret_cast<h16*>(m[o]) : nullptr;
    plan.jobs[i].alpha = update ? lr * descs[o].scale : descs[o].scale;
  }
  NsArgs a;
  a.steps = steps;
  a.products = products;
  a.coef = table;
  a.momentum = momentum;
  a.keep = 1.0f - lr * weight_decay;
  a.nesterov = nesterov != 0;
  return hip_status(launch_ns(plan, a, ws, static_cast<hipStream_t>(stream)));
}

// ---- 8-bit integer dense layers -----------------------------------------------------

bool i8_sides_ok(int64_t a, int64_t b) {
  return a >= 1 && b >= 1 && a < (1 << 22) && b < (1 << 22) && a * b < ((int64_t)1 << 40);
}
size_t i8_bytes(int64_t rows, int64_t n) { return (size_t)(rows * i8_row(n)); }

bool dense_ok(const fp16_int8_dense_desc* d) {
  return d->tokens >= 1 && d->inputs >= 1 && d->outputs >= 1 && d->tokens <= kI8MaxK &&
         d->inputs <= kI8MaxK && d->outputs <= kI8MaxK;
}

// Workspace places of the three calls.
struct DenseWs {
  size_t q1 = 0, s1 = 0, q2 = 0, s2 = 0, q3 = 0, s3 = 0, part = 0, part2 = 0, total = 0;
};
DenseWs dense_ws(const fp16_int8_dense_desc* d, int call) {
  DenseWs L;
  const int T = d->tokens, I = d->inputs, O = d->outputs;
  auto take = [&](size_t bytes) {
    const size_t at = L.total;
    L.total += align256(bytes);
    return at;
  };
  if (call == FP16_INT8_WEIGHTS) {
    L.part = take(i8_cols_ws_bytes(O, I, true, false));
  } else if (call == FP16_INT8_FWD) {
    if (!i8_fused_ok(T, O, I)) {
      L.q1 = take(i8_bytes(T, I));
      L.s1 = take((size_t)T * 4);
    }
  } else {
    // dy by rows, dy by columns, x by columns
    L.q1 = take(i8_bytes(T, O));
    L.s1 = take((size_t)T * 4);
    L.q2 = take(i8_bytes(O, T));
    L.s2 = take((size_t)O * 4);
    L.q3 = take(i8_bytes(I, T));
    L.s3 = take((size_t)I * 4);
    L.part = take(i8_cols_ws_bytes(T, O, true, true));
    L.part2 = take(i8_cols_ws_bytes(T, I, false, false));
  }
  return L;
}

template <class T>
T* ws_at(void* ws, size_t off) {
  return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

fp16_status ws_ok(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return FP16_OK;
  if (!ws || ws_bytes < need) return FP16_ERR_WORKSPACE;
  return aligned16(ws) ? FP16_OK : FP16_ERR_MISALIGNED;
}

// Whether a written buffer overlaps any other of the list.
struct Buf {
  const void* p;
  size_t bytes;
  bool written;
};
template <int N>
bool bufs_clash(const Buf (&b)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N; ++j)
      if (i != j && b[i].written && overlap(b[i].p, b[i].bytes, b[j].p, b[j].bytes)) return true;
  return false;
}
template <int N>
bool bufs_aligned(const Buf (&b)[N]) {
  for (int i = 0; i < N; ++i)
    if (!aligned16(b[i].p)) return false;
  return true;
}

const h16* hp(const fp16_t* p) { return reinterpret_cast<const h16*>(p); }
h16* hp(fp16_t* p) { return reinterpret_cast<h16*>(p); }

}  // namespace

extern "C" {

size_t fp16_muon_workspace_bytes(int32_t count, const fp16_muon_desc* descs, int32_t products) {
  if (!ns_list_ok(count, descs, products)) return 0;
  NsHost host;
  return host.make(count, descs, products) ? host.plan.bytes : 0;
}

const char* fp16_muon_kernels(int32_t count, const fp16_muon_desc* descs, int32_t products) {
  thread_local char name[64];
  if (!ns_list_ok(count, descs, products)) return "";
  NsHost host;
  if (!host.make(count, descs, products)) return "";
  const NsPlan& plan = host.plan;
  if (plan.small) return "one workgroup each";
  char* at = name;
  for (const NsTile& k : plan.kind) {
    at += snprintf(at, sizeof(name) - (size_t)(at - name), "%s%s", at == name ? "" : ", ", k.name);
    if (k.parts > 1) at += snprintf(at, sizeof(name) - (size_t)(at - name), " in %d", k.parts);
  }
  return name;
}

fp16_status fp16_orthogonalize(int32_t count, const fp16_muon_desc* descs, const fp16_t* const* x,
                               fp16_t* const* y, int32_t steps, const float* coef,
                               int32_t products, void* ws, size_t ws_bytes, fp16_stream_t stream) {
  return ns_call(count, descs, y, x, nullptr, false, 0.0f, 0.0f, 0.0f, 0, steps, coef, products, ws,
                 ws_bytes, stream);
}

fp16_status fp16_muon_step(int32_t count, const fp16_muon_desc* descs, fp16_t* const* w,
                           const fp16_t* const* g, fp16_t* const* m, float lr, float momentum,
                           float weight_decay, int32_t nesterov, int32_t steps, const float* coef,
                           int32_t products, void* ws, size_t ws_bytes, fp16_stream_t stream) {
  return ns_call(count, descs, w, g, m, true, lr, momentum, weight_decay, nesterov, steps, coef,
                 products, ws, ws_bytes, stream);
}

size_t fp16_int8_row_bytes(int32_t n) { return n < 1 ? 0 : (size_t)i8_row(n); }

fp16_status fp16_int8_quant_rows(int32_t rows, int32_t cols, const fp16_t* x, int8_t* q,
                                 float* scale, fp16_stream_t stream) {
  if (!i8_sides_ok(rows, cols)) return FP16_ERR_SHAPE;
  if (!x || !q || !scale) return FP16_ERR_NULL;
  const Buf b[] = {{x, (size_t)rows * cols * 2, false},
                   {q, i8_bytes(rows, cols), true},
                   {scale, (size_t)rows * 4, true}};
  if (!bufs_aligned(b)) return FP16_ERR_MISALIGNED;
  if (bufs_clash(b)) return FP16_ERR_ALIASING;
  return hip_status(launch_i8_rows(rows, cols, hp(x), q, scale, static_cast<hipStream_t>(stream)));
}

size_t fp16_int8_quant_workspace_bytes(int32_t rows, int32_t cols) {
  return i8_sides_ok(rows, cols) ? i8_cols_ws_bytes(rows, cols, false, false) : 0;
}

fp16_status fp16_int8_quant_cols(int32_t rows, int32_t cols, const fp16_t* x, int8_t* q,
                                 float* scale, void* ws, size_t ws_bytes, fp16_stream_t stream) {
  if (!i8_sides_ok(rows, cols)) return FP16_ERR_SHAPE;
  if (!x || !q || !scale) return FP16_ERR_NULL;
  const size_t need = i8_cols_ws_bytes(rows, cols, false, false);
  const fp16_status s = ws_ok(ws, ws_bytes, need);
  if (s != FP16_OK) return s;
  const Buf b[] = {{x, (size_t)rows * cols * 2, false},
                   {q, i8_bytes(cols, rows), true},
                   {scale, (size_t)cols * 4, true},
                   {ws, need, true}};
  if (!bufs_aligned(b)) return FP16_ERR_MISALIGNED;
  if (bufs_clash(b)) return FP16_ERR_ALIASING;
  const I8Cols j = i8_cols_job(rows, cols, hp(x), q, scale, nullptr, nullptr, nullptr, ws);
  return hip_status(launch_i8_cols(&j, 1, static_cast<hipStream_t>(stream)));
}

fp16_status fp16_int8_matmul(int32_t m, int32_t n, int32_t k, const int8_t* a, const float* sa,
                             const int8_t* b, const float* sb, const fp16_t* bias, fp16_t* y,
                             fp16_stream_t stream) {
  if (!i8_sides_ok(m, n) || k < 1 || k > kI8MaxK) return FP16_ERR_SHAPE;
  if (!a || !sa || !b || !sb || !y) return FP16_ERR_NULL;
  const Buf l[] = {{a, i8_bytes(m, k), false},          {sa, (size_t)m * 4, false},
                   {b, i8_bytes(n, k), false},          {sb, (size_t)n * 4, false},
                   {bias, bias ? (size_t)n * 2 : 0, false}, {y, (size_t)m * n * 2, true}};
  if (!bufs_aligned(l)) return FP16_ERR_MISALIGNED;
  if (bufs_clash(l)) return FP16_ERR_ALIASING;
  const I8Product p{m, n, k, a, b, sa, sb, hp(bias), hp(y)};
  return hip_status(launch_i8_product(p, static_cast<hipStream_t>(stream)));
}

const char* fp16_int8_kernel(int32_t m, int32_t n, int32_t k) {
  if (!i8_sides_ok(m, n) || k < 1 || k > kI8MaxK) return "";
  return i8_product_name(m, n, k);
}

size_t fp16_int8_dense_workspace_bytes(const fp16_int8_dense_desc* desc, int32_t call) {
  if (!desc || !dense_ok(desc) || call < FP16_INT8_FWD || call > FP16_INT8_WEIGHTS) return 0;
  return dense_ws(desc, call).total;
}

fp16_status fp16_int8_dense_weights(const fp16_int8_dense_desc* desc, const fp16_t* w, int8_t* wq,
                                    float* sw, int8_t* wqt, float* swt, void* ws, size_t ws_bytes,
                                    fp16_stream_t stream) {
  if (!desc || !w || !wq || !sw || (wqt == nullptr) != (swt == nullptr)) return FP16_ERR_NULL;
  if (!dense_ok(desc)) return FP16_ERR_SHAPE;
  const int I = desc->inputs, O = desc->outputs;
  const DenseWs L = dense_ws(desc, FP16_INT8_WEIGHTS);
  const size_t need = wqt ? L.total : 0;
  const fp16_status s = ws_ok(ws, ws_bytes, need);
  if (s != FP16_OK) return s;
  const Buf b[] = {{w, (size_t)I * O * 2, false},
                   {wq, i8_bytes(O, I), true},
                   {sw, (size_t)O * 4, true},
                   {wqt, wqt ? i8_bytes(I, O) : 0, true},
                   {swt, swt ? (size_t)I * 4 : 0, true},
                   {need ? ws : nullptr, need, true}};
  if (!bufs_aligned(b)) return FP16_ERR_MISALIGNED;
  if (bufs_clash(b)) return FP16_ERR_ALIASING;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (!wqt) return hip_status(launch_i8_rows(O, I, hp(w), wq, sw, st));
  const I8Cols j = i8_cols_job(O, I, hp(w), wqt, swt, wq, sw, nullptr, ws_at<void>(ws, L.part));
  return hip_status(launch_i8_cols(&j, 1, st));
}

fp16_status fp16_int8_dense_fwd(const fp16_int8_dense_desc* desc, const fp16_t* x, const int8_t* wq,
                                const float* sw, const fp16_t* bias, fp16_t* y, void* ws,
                                size_t ws_bytes, fp16_stream_t stream) {
  if (!desc || !x || !wq || !sw || !y) return FP16_ERR_NULL;
  if (!dense_ok(desc)) return FP16_ERR_SHAPE;
  const int T = desc->tokens, I = desc->inputs, O = desc->outputs;
  const DenseWs L = dense_ws(desc, FP16_INT8_FWD);
  const fp16_status s = ws_ok(ws, ws_bytes, L.total);
  if (s != FP16_OK) return s;
  const Buf b[] = {{x, (size_t)T * I * 2, false},
                   {wq, i8_bytes(O, I), false},
                   {sw, (size_t)O * 4, false},
                   {bias, bias ? (size_t)O * 2 : 0, false},
                   {y, (size_t)T * O * 2, true},
                   {L.total ? ws : nullptr, L.total, true}};
  if (!bufs_aligned(b)) return FP16_ERR_MISALIGNED;
  if (bufs_clash(b)) return FP16_ERR_ALIASING;
  hipStream_t st = static_cast<hipStream_t>(stream);
  I8Product p{T, O, I, nullptr, wq, nullptr, sw, hp(bias), hp(y)};
  if (i8_fused_ok(T, O, I)) return hip_status(launch_i8_fused(p, hp(x), st));
  int8_t* q = ws_at<int8_t>(ws, L.q1);
  float* sc = ws_at<float>(ws, L.s1);
  TRY(launch_i8_rows(T, I, hp(x), q, sc, st));
  p.a = q;
  p.sa = sc;
  return hip_status(launch_i8_product(p, st));
}

fp16_status fp16_int8_dense_bwd(const fp16_int8_dense_desc* desc, const fp16_t* x, const fp16_t* dy,
                                const int8_t* wqt, const float* swt, fp16_t* dx, fp16_t* dw,
                                fp16_t* dbias, void* ws, size_t ws_bytes, fp16_stream_t stream) {
  if (!desc || !dy || (dx && (!wqt || !swt)) || (dw && !x) || (dbias && !dw)) return FP16_ERR_NULL;
  if (!dense_ok(desc)) return FP16_ERR_SHAPE;
  const int T = desc->tokens, I = desc->inputs, O = desc->outputs;
  const DenseWs L = dense_ws(desc, FP16_INT8_BWD);
  const fp16_status s = ws_ok(ws, ws_bytes, L.total);
  if (s != FP16_OK) return s;
  const Buf b[] = {{dw ? x : nullptr, (size_t)T * I * 2, false},
                   {dy, (size_t)T * O * 2, false},
                   {dx ? wqt : nullptr, i8_bytes(I, O), false},
                   {dx ? swt : nullptr, (size_t)I * 4, false},
                   {dx, (size_t)T * I * 2, true},
                   {dw, (size_t)O * I * 2, true},
                   {dbias, (size_t)O * 2, true},
                   {ws, L.total, true}};
  if (!bufs_aligned(b)) return FP16_ERR_MISALIGNED;
  if (bufs_clash(b)) return FP16_ERR_ALIASING;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int8_t *q1 = ws_at<int8_t>(ws, L.q1), *q2 = ws_at<int8_t>(ws, L.q2), *q3 = ws_at<int8_t>(ws, L.q3);
  float *s1 = ws_at<float>(ws, L.s1), *s2 = ws_at<float>(ws, L.s2), *s3 = ws_at<float>(ws, L.s3);
  if (dw) {
    const I8Cols j[2] = {i8_cols_job(T, O, hp(dy), q2, s2, dx ? q1 : nullptr, dx ? s1 : nullptr,
                                     hp(dbias), ws_at<void>(ws, L.part)),
                         i8_cols_job(T, I, hp(x), q3, s3, nullptr, nullptr, nullptr,
                                     ws_at<void>(ws, L.part2))};
    TRY(launch_i8_cols(j, 2, st));
  } else if (dx) {
    TRY(launch_i8_rows(T, O, hp(dy), q1, s1, st));
  }
  if (dx) {
    const I8Product p{T, I, O, q1, wqt, s1, swt, nullptr, hp(dx)};
    TRY(launch_i8_product(p, st));
  }
  if (dw) {
    const I8Product p{O, I, T, q2, q3, s2, s3, nullptr, hp(dw)};
    TRY(launch_i8_product(p, st));
  }
  return FP16_OK;
}

}  // extern "C"
