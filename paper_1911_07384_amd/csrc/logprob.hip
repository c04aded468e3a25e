// Log probabilities of given classes, the entropy of each row's distribution and its
// most probable classes, and the logits' gradient from the gradients of the first two.
//
// For a row of logits z, with m its largest and d_j = scale (z_j - m):
//   S = sum_j exp(d_j),  T = sum_j exp(d_j) d_j
//   logp_j = d_j - log S,  H = log S - T / S   (every term of T is <= 0: no
//   cancellation), and, with p_j = exp(logp_j) and t the given class,
//   dz_j = scale (dlogp ([j = t] - p_j) - dH p_j (logp_j + H)).
// One pass over the row holds m, S and T by lane (each further group of elements may
// raise m, which scales S and T down), and they are joined over the lanes and, where
// few long rows are split over workgroups, over the parts.  How the exponents are
// computed, and what S and T are relative to, goes by the scale (see Sums).
//
// The most probable classes: the top-th largest of the lanes' maxima bounds the top-th
// largest element from below, so that a second look at the row (from the caches)
// gathers the few elements at or above it; those are ranked by counting, with the
// value and then the lower class as the key.  Where equal values make them more than
// kCand, the value that `top` elements reach is found by bisection, those above it are
// gathered and the first ones at it added in order.

#include "head.hpp"

#include <type_traits>

namespace fp16k {
namespace {

// Threads of a workgroup, NT: 256, and 512 for whole rows of more than kLong classes, of
// which fewer are then read at a time (4096 x 50001: 96 us with 256, 89 with 512: 410 MB at
// 4.6 TB/s; 128 x 1000 with 5 alternatives 5.4 us, a launch, one trip to memory and the ranking).
constexpr int kNT = 256, kU = 4, kLong = 16384;
constexpr int kCand = 1024;
constexpr int kPart = 4096, kMaxParts = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFloor = -1e30f;

typedef unsigned long long u64;

// 16-bit keys in the order of the values: NaN above all, +0 and -0 the same, 0 below all
__device__ __forceinline__ uint32_t value_key(uint16_t b) {
  if ((b & 0x7FFF) > 0x7C00) return 0xFFFF;
  if (b == 0x8000) return 0x8000;
  return (b & 0x8000) ? (uint16_t)~b : (b | 0x8000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  const uint16_t b = (k & 0x8000) ? (uint16_t)(k ^ 0x8000) : (uint16_t)~k;
  return k == 0xFFFF ? __builtin_nanf("") : to_f32(__builtin_bit_cast(h16, b));
}
__device__ __forceinline__ u64 full_key(uint32_t value, int cls) {
  return ((u64)value << 32) | (0xFFFFFFFFu - (uint32_t)cls);
}

// With c = fl(scale / ln 2), a term's exponent is fl(z c - r), r = fl(m c), where the scale
// allows it (!DIFF): one instruction with one rounding (a factor may be binary16).  The
// sums are then relative to r and not to m c, and what r is off by, known exactly, is put
// right at the end:
//   log sum exp(scale (z - m)) = log s + ln 2 (r - m c),  H = log s - ln 2 t / s.
// While kLargest c < 2^24 (scales up to 177) r is off by at most 1/2, for any logits: the
// largest term is 2^-1/2 to 2^1/2, and H's two parts cancel by ln 2 / 2 at most.  Larger
// scales let r be off by enough for the largest term to overflow or vanish: there the
// differences are taken first (DIFF), fl(fl(z - m) c), the largest exponent is 0 and no
// term of t is positive.  They have kernels of their own, so that usual scales do not pay
// for them (32768 x 1000: 56 us, 49 without; 4096 x 50048: 74 and 73).
struct Sums {
  float m, s, t;  // m: a binary16 value; t in units of ln 2
};
constexpr float kLargest = 65504.0f;  // of binary16
bool differences_first(float scale) { return !(kLargest * (scale * kLog2e) < 16777216.0f); }

// exponent by which sums of maximum m count towards a maximum of top
template <bool DIFF>
__device__ __forceinline__ float shift(float m, float top, float c) {
  // (the floor also where both are -inf)
  return __builtin_fmaxf(DIFF ? (m - top) * c : m * c - top * c, kFloor);
}
template <bool DIFF>
__device__ __forceinline__ void rescale(Sums& a, float top, float c) {
  const float d = shift<DIFF>(a.m, top, c), f = __builtin_amdgcn_exp2f(d);
  a.t = f * (a.t + d * a.s);
  a.s *= f;
  a.m = top;
}

__device__ __forceinline__ V8 low8() {
  V8 v;
  v.u = u32x4{0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u};
  return v;
}
// (Loops that few lanes enter are kept as loops: these kernels run once over a row, and
// instructions that have to be fetched for one use cost more than they do.)
__device__ __forceinline__ V8 load8_low(const h16* p, int left) {
  if (left >= 8) return load16u(p);
  u64 lo = 0xFC00FC00FC00FC00ull, hi = lo;
  const uint16_t* const from = reinterpret_cast<const uint16_t*>(p);
#pragma unroll 1
  for (int e = left - 1; e >= 0; --e) {
    hi = hi << 16 | lo >> 48;
    lo = lo << 16 | from[e];
  }
  V8 v;
  v.d[0] = (uint32_t)lo;
  v.d[1] = (uint32_t)(lo >> 32);
  v.d[2] = (uint32_t)hi;
  v.d[3] = (uint32_t)(hi >> 32);
  return v;
}
__device__ __forceinline__ half2 top2(const V8& v) {
  half2 t = __builtin_bit_cast(half2, v.d[0]);
#pragma unroll
  for (int k = 1; k < 4; ++k) t = __builtin_elementwise_max(t, __builtin_bit_cast(half2, v.d[k]));
  return t;
}
// f(value key, e) for the elements e of v, -inf past the first `left`
template <class F>
__device__ __forceinline__ void each8(const V8& v, int left, F f) {
  u64 w = v.d[0] | (u64)v.d[1] << 32, hi = v.d[2] | (u64)v.d[3] << 32;
#pragma unroll 1
  for (int e = 0; e < 8 && e < left; ++e) {
    f(value_key((uint16_t)w), e);
    w = w >> 16 | hi << 48;
    hi >>= 16;
  }
}
// the largest value key of a vector (of a NaN's, if it has one)
__device__ __forceinline__ uint32_t top_key(const V8& v) {
  const half2 t = top2(v);
  const float f = __builtin_fmaxf(to_f32(t[0]), to_f32(t[1]));
  bool nan = false;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const half2 h = __builtin_bit_cast(half2, v.d[k]);
    nan |= __builtin_isnan(h[0]) | __builtin_isnan(h[1]);
  }
  return nan ? 0xFFFFu : value_key(__builtin_bit_cast(uint16_t, (h16)f));
}

// A lane's elements of z[0 .. n): vectors of 8, kU at a time, -inf past the end.
template <int NT>
__device__ __forceinline__ void lane_load(const h16* z, int n, int i, V8 (&v)[kU]) {
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const int at = i + u * NT * 8;
    v[u] = at < n ? load8_low(z + at, n - at) : low8();
  }
}

template <bool DIFF>
__device__ __forceinline__ void lane_add(const V8 (&v)[kU], float c, Sums& a) {
  half2 top = top2(v[0]);
#pragma unroll
  for (int u = 1; u < kU; ++u) top = __builtin_elementwise_max(top, top2(v[u]));
  // (a NaN is no maximum here; it reaches the sums below)
  float m = __builtin_fmaxf(to_f32(top[0]), to_f32(top[1]));
  m = __builtin_fmaxf(m, a.m);
  rescale<DIFF>(a, m, c);
  const float r = m == -__builtin_inff() ? 0.0f : DIFF ? m : m * c;
#pragma unroll
  for (int u = 0; u < kU; ++u)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float z = to_f32(v[u].h[k]);
      const float d = DIFF ? (z - r) * c : __builtin_fmaf(z, c, -r);
      const float e = __builtin_amdgcn_exp2f(d);
      a.s += e;
      a.t = __builtin_fmaf(e, __builtin_fmaxf(d, kFloor), a.t);
    }
}

// This lane's sums over z[0 .. n); v holds the last turn's elements.
template <int NT, bool DIFF>
__device__ __forceinline__ Sums lane_sums(const h16* z, int n, float c, V8 (&v)[kU]) {
  Sums a = {-__builtin_inff(), 0.0f, 0.0f};
  for (int i = threadIdx.x * 8; i < n; i += NT * 8 * kU) {
    lane_load<NT>(z, n, i, v);
    lane_add<DIFF>(v, c, a);
  }
  return a;
}

// f(x, i) for a lane's vectors x from z + i on, read again if they are not all in v
template <int NT, class F>
__device__ __forceinline__ void lane_each(const h16* z, int n, V8 (&v)[kU], F f) {
  for (int i = threadIdx.x * 8; i < n; i += NT * 8 * kU) {
    if (n > NT * 8 * kU) lane_load<NT>(z, n, i, v);
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (i + u * NT * 8 < n) f(v[u], i + u * NT * 8);
  }
}

// Over the 64 lanes of a wave, in every one of them, by register permutes alone: quads,
// eights, sixteens, the rows of 16 and the halves.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL,
                                                               0xf, 0xf, false));
}
template <class F>
__device__ __forceinline__ float wave_all(float v, F f) {
  v = f(v, dpp<0xB1>(v));   // lanes 1 0 3 2 of each quad
  v = f(v, dpp<0x4E>(v));   // 2 3 0 1
  v = f(v, dpp<0x141>(v));  // 7 .. 0 of each eight
  v = f(v, dpp<0x140>(v));  // 15 .. 0 of each sixteen
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  v = f(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
  const uint32_t d = __builtin_bit_cast(uint32_t, v);
  const auto q = __builtin_amdgcn_permlane32_swap(d, d, false, false);
  return f(__builtin_bit_cast(float, (uint32_t)q[0]), __builtin_bit_cast(float, (uint32_t)q[1]));
}

// Joined over the workgroup, the same in every lane.
template <int NT, bool DIFF>
__device__ __forceinline__ Sums block_sums(Sums a, float c, float (*red)[3]) {
  constexpr int kWaves = NT / 64;
  const auto larger = [](float x, float y) { return __builtin_fmaxf(x, y); };
  const auto sum = [](float x, float y) { return x + y; };
  float m = wave_all(a.m, larger);
  rescale<DIFF>(a, m, c);
  a.s = wave_all(a.s, sum);
  a.t = wave_all(a.t, sum);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[wave][0] = a.m;
    red[wave][1] = a.s;
    red[wave][2] = a.t;
  }
  __syncthreads();
  m = red[0][0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = __builtin_fmaxf(m, red[w][0]);
  Sums r = {m, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    Sums b = {red[w][0], red[w][1], red[w][2]};
    rescale<DIFF>(b, m, c);
    r.s += b.s;
    r.t += b.t;
  }
  __syncthreads();
  return r;
}

template <int NT>
struct TopLds {
  __attribute__((aligned(16))) u64 cand[kCand + 8];
  u64 best[kTopMax];
  uint16_t lane[NT];
  int count, scan[NT / 64];
};

// A workgroup's `top` largest keys into l.best, in order, from `count` distinct ones
// in l.cand (0s where there are fewer).
template <int NT>
__device__ __forceinline__ void rank_candidates(TopLds<NT>& l, int count, int top) {
  for (int i = threadIdx.x; i < top; i += NT) l.best[i] = 0;
  if (threadIdx.x < 8) l.cand[count + threadIdx.x] = 0;  // (whole eights)
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += NT) {
    const u64 k = l.cand[i];
    int r = 0;
    for (int j = 0; j < count; j += 8) {
      u64 o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = l.cand[j + e];
#pragma unroll
      for (int e = 0; e < 8; ++e) r += o[e] > k;
    }
    if (r < top) l.best[r] = k;
  }
  __syncthreads();
}

template <int NT>
__device__ __forceinline__ int block_count(int n, TopLds<NT>& l) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) l.scan[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) n += l.scan[w];
  __syncthreads();
  return n;
}

// The `top` largest elements of z[0 .. n), classes first + i, into l.best.  m: the
// largest of this lane's elements, v as lane_sums left it.
template <int NT>
__device__ __forceinline__ void block_top(const h16* z, int n, int first, int top, float m,
                                          V8 (&v)[kU], TopLds<NT>& l) {
  constexpr int kWaves = NT / 64;
  l.lane[threadIdx.x] = (uint16_t)value_key(__builtin_bit_cast(uint16_t, (h16)m));
  __syncthreads();
  // the largest value that `top` lanes' maxima reach, to its highest twelve bits (1.6 %,
  // and a few more candidates), bit by bit, in every wave alike
  uint32_t bound = 0;
  {
    uint32_t key[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) key[w] = l.lane[w * 64 + (threadIdx.x & 63)];
#pragma unroll 1
    for (int b = 15; b >= 4; --b) {
      const uint32_t up = bound | (1u << b);
      int c = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) c += __popcll(__ballot(key[w] >= up));
      if (c >= top) bound = up;
    }
  }
  // gathers what is at or above `from`
  auto gather = [&](uint32_t from) {
    if (threadIdx.x == 0) l.count = 0;
    __syncthreads();
    lane_each<NT>(z, n, v, [&](const V8& x, int i) {
      if (top_key(x) < from) return;
      each8(x, n - i, [&](uint32_t k, int e) {
        if (k >= from) {
          const int at = atomicAdd(&l.count, 1);
          if (at < kCand) l.cand[at] = full_key(k, first + i + e);
        }
      });
    });
    __syncthreads();
    const int count = l.count;
    __syncthreads();
    return count;
  };
  // (masked classes are at -inf and many)
  constexpr uint32_t kLow = 0x3FF;
  if (bound <= kLow) bound = kLow;  // (no value is below)
  int count = gather(bound == kLow ? kLow + 1 : bound);
  if (count > kCand || count < top) {
    // too many of one value: those above it ..
    uint32_t value = bound;
    if (count > kCand) {
      // (the largest value that `top` elements reach, bit by bit)
      value = 0;
#pragma unroll 1
      for (int b = 15; b >= 0; --b) {
        const uint32_t up = value | (1u << b);
        int c = 0;
        lane_each<NT>(z, n, v, [&](const V8& x, int i) {
          each8(x, n - i, [&](uint32_t k, int) { c += k >= up; });
        });
        if (block_count<NT>(c, l) >= top) value = up;
      }
      count = gather(value + 1);
    }
    // .. and the first of those equal to it, in the order of the classes
#pragma unroll 1
    for (int i0 = 0; i0 < n && count < top; i0 += NT * 8) {
      const int i = i0 + threadIdx.x * 8;
      const V8 x = i < n ? load8_low(z + i, n - i) : low8();
      uint32_t eq = 0;
      each8(x, n - i, [&](uint32_t k, int e) { eq |= (uint32_t)(k == value) << e; });
      const int mine8 = __popc(eq);
      int before = mine8;  // inclusive, over the wave
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int other = __shfl_up(before, o, 64);
        if ((int)(threadIdx.x & 63) >= o) before += other;
      }
      if ((threadIdx.x & 63) == 63) l.scan[threadIdx.x >> 6] = before;
      __syncthreads();
      int at = count + before - mine8, all = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        if (w < (int)(threadIdx.x >> 6)) at += l.scan[w];
        all += l.scan[w];
      }
#pragma unroll 1
      for (int e = 0; e < 8; ++e)
        if ((eq >> e) & 1) {
          if (at < top) l.cand[at] = full_key(value, first + i + e);
          ++at;
        }
      count = count + all < top ? count + all : top;
      __syncthreads();
    }
  }
  rank_candidates<NT>(l, count, top);
}

// What a row's sums and largest keys give.
template <int NT, bool DIFF>
__device__ __forceinline__ void finish(const LogprobArgs& a, int row, const Sums& r,
                                       const u64* best) {
  const bool none = r.m == -__builtin_inff() && r.s == 0.0f;  // every class is at -inf
  const float c = a.scale * kLog2e, ln = logf(r.s);
  const float log_s =
      DIFF ? ln : __builtin_fmaf(kLn2, __builtin_fmaf(-r.m, c, r.m * c), ln);
  if (threadIdx.x == 0) {
    a.stats[3 * (int64_t)row] = r.m;
    a.stats[3 * (int64_t)row + 1] = none ? -__builtin_inff() : log_s;
    a.stats[3 * (int64_t)row + 2] = none ? 0.0f : ln - kLn2 * (r.t / r.s);
    if (a.logp) {
      const int t = a.token[row];
      float lp = 0.0f;
      if (t >= a.classes)
        lp = __builtin_nanf("");
      else if (t >= 0)
        lp = none ? -__builtin_inff()
                  : (to_f32(a.z[row * a.stride + t]) - r.m) * a.scale - log_s;
      a.logp[row] = lp;
    }
  }
  for (int i = threadIdx.x; i < a.top; i += NT) {
    const u64 k = best[i];
    const float v = key_value((uint32_t)(k >> 32));
    a.top_id[(int64_t)row * a.top + i] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
    a.top_logp[(int64_t)row * a.top + i] =
        none ? -__builtin_inff() : (v - r.m) * a.scale - log_s;
  }
}

// What a part of a row leaves for the join.
__host__ __device__ inline size_t part_bytes(int top) { return 16 + (size_t)top * 8; }

template <int NT, bool PARTS, bool TOP, bool DIFF>
__global__ __launch_bounds__(NT) void logprob_kernel(const LogprobArgs a, int parts, int per) {
  __shared__ float red[NT / 64][3];
  __shared__ typename std::conditional<TOP, TopLds<NT>, u64>::type l;
  const int row = PARTS ? blockIdx.x / parts : blockIdx.x;
  const int first = PARTS ? (blockIdx.x % parts) * per : 0;
  const int n = PARTS && a.classes - first > per ? per : a.classes - first;
  const h16* z = a.z + row * a.stride + first;
  const float c = a.scale * kLog2e;
  V8 v[kU];
  const Sums mine = lane_sums<NT, DIFF>(z, n, c, v);
  const Sums r = block_sums<NT, DIFF>(mine, c, red);
  const u64* best = nullptr;
  if constexpr (TOP) {
    block_top<NT>(z, n, first, a.top, mine.m, v, l);
    best = l.best;
  }
  if (!PARTS) {
    finish<NT, DIFF>(a, row, r, best);
  } else {
    char* to = static_cast<char*>(a.ws) + blockIdx.x * part_bytes(a.top);
    if (threadIdx.x == 0) {
      float* f = reinterpret_cast<float*>(to);
      f[0] = r.m;
      f[1] = r.s;
      f[2] = r.t;
    }
    u64* k = reinterpret_cast<u64*>(to + 16);
    for (int i = threadIdx.x; i < a.top; i += NT) k[i] = best[i];
  }
}

// A row from its parts: the sums, and the largest of their keys by counting.  32 parts with 20
// keys each 5.0 us, a launch and two dependent trips to memory and LDS.
template <bool DIFF>
__global__ __launch_bounds__(kNT) void logprob_join(const LogprobArgs a, int parts) {
  __shared__ float red[kNT / 64][3];
  __shared__ TopLds<kNT> l;
  const int row = blockIdx.x;
  const float c = a.scale * kLog2e;
  const char* from = static_cast<const char*>(a.ws) + (int64_t)row * parts * part_bytes(a.top);
  Sums mine = {-__builtin_inff(), 0.0f, 0.0f};
  if ((int)threadIdx.x < parts) {
    const float* f = reinterpret_cast<const float*>(from + threadIdx.x * part_bytes(a.top));
    mine = {f[0], f[1], f[2]};
  }
  const Sums r = block_sums<kNT, DIFF>(mine, c, red);
  if (a.top) {
    // a lane holds up to kPer of a part's keys; as in block_top, the lanes' maxima bound
    // what is ranked, and only `top` lanes reach the bound
    constexpr int kLanes = kNT / kMaxParts, kPer = kTopMax / kLanes;  // of a part; keys
    static_assert(kPer * kTopMax <= kCand, "candidates");
    const int p = threadIdx.x / kLanes;
    const u64* const keys = reinterpret_cast<const u64*>(from + p * part_bytes(a.top) + 16);
    u64 key[kPer], most = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * kLanes + threadIdx.x % kLanes;
      key[i] = p < parts && at < a.top ? keys[at] : 0;
      most = key[i] > most ? key[i] : most;
    }
    l.cand[threadIdx.x] = most;
    if (threadIdx.x == 0) {
      l.count = 0;
      l.best[0] = 0;
    }
    __syncthreads();
    int rank = 0;
    const int lanes = parts * kLanes;
    for (int j = 0; j < lanes; j += 16) {  // (parts past the last hold zeros)
      u64 o[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = l.cand[j + e];
#pragma unroll
      for (int e = 0; e < 16; ++e) rank += o[e] > most;
    }
    if (rank == a.top - 1 && most) l.best[0] = most;  // (lanes without keys share 0)
    __syncthreads();
    const u64 bound = l.best[0];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (key[i] && key[i] >= bound) {
        const int at = atomicAdd(&l.count, 1);
        if (at < kCand) l.cand[at] = key[i];
      }
    __syncthreads();
    rank_candidates<kNT>(l, l.count < kCand ? l.count : kCand, a.top);
  }
  finish<kNT, DIFF>(a, row, r, l.best);
}

// The gradient: each lane 8 classes of a row at a time, no sums, bound by its bytes: 4096 x
// 50001 after the forward 129 us, 819 MB at 6.4 TB/s (some of them from the caches).
__global__ __launch_bounds__(kNT) void logprob_bwd_kernel(const LogprobArgs a, int parts, int per) {
  // the last rows first: a forward before read them last, and they may still be cached
  const int row = a.rows - 1 - (int)(blockIdx.x / parts), first = (blockIdx.x % parts) * per;
  const int end = a.classes - first > per ? first + per : a.classes;
  const float m = a.stats[3 * (int64_t)row], log_s = a.stats[3 * (int64_t)row + 1],
              h = a.stats[3 * (int64_t)row + 2];
  const int t = a.token ? a.token[row] : -1;
  const float dl = a.dlogp && t >= 0 ? a.dlogp[row] : 0.0f;
  const float dh = a.dentropy ? a.dentropy[row] : 0.0f;
  const bool none = m == -__builtin_inff() && log_s == -__builtin_inff();
  const h16* z = a.z + row * a.stride;
  h16* dz = a.dz + row * a.stride;
  for (int i = first + threadIdx.x * 8; i < end; i += kNT * 8) {
    const V8 v = load8_upto(z + i, end - i);
    V8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float lp = (to_f32(v.h[e]) - m) * a.scale - log_s;
      const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
      // (p before dh: with any finite dh a class of p = 0, at any lp from -200 down, adds 0)
      const float q = p * (__builtin_fmaxf(lp, -200.0f) + h);
      float g = -__builtin_fmaf(dh, q, dl * p);
      if (i + e == t) g += dl;
      o.h[e] = to_h16(none ? 0.0f : g * a.scale);
    }
    store8_upto(dz + i, o, end - i);
  }
}

// Parts of a row: as many as fill the device, of kPart classes at least.
int row_parts(int rows, int classes) {
  const int fill = (512 + rows - 1) / rows, most = (classes + kPart - 1) / kPart;
  const int parts = fill < most ? fill : most;
  return parts < 1 ? 1 : parts > kMaxParts ? kMaxParts : parts;
}
int part_len(int classes, int parts) { return ((classes + parts - 1) / parts + 7) & ~7; }

}  // namespace

size_t logprob_ws_bytes(int rows, int classes, int top) {
  const int parts = row_parts(rows, classes);
  return parts == 1 ? 0 : (size_t)rows * parts * part_bytes(top);
}

namespace {
template <bool DIFF>
hipError_t launch_sums(const LogprobArgs& a, hipStream_t st) {
  int parts = row_parts(a.rows, a.classes);
  const int per = part_len(a.classes, parts);
  parts = (a.classes + per - 1) / per;  // (none is empty)
  const unsigned grid = (unsigned)((int64_t)a.rows * parts);
  const auto go = [&](auto nt, auto split, auto top) {
    constexpr int NT = decltype(nt)::value;
    logprob_kernel<NT, decltype(split)::value, decltype(top)::value, DIFF>
        <<<grid, NT, 0, st>>>(a, parts, per);
  };
  const auto pick = [&](auto nt, auto split) {
    if (a.top)
      go(nt, split, std::true_type{});
    else
      go(nt, split, std::false_type{});
  };
  constexpr std::integral_constant<int, 256> small{};
  if (parts == 1) {
    if (a.classes > kLong)
      pick(std::integral_constant<int, 512>{}, std::false_type{});
    else
      pick(small, std::false_type{});
    return hipGetLastError();
  }
  pick(small, std::true_type{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  logprob_join<DIFF><<<a.rows, kNT, 0, st>>>(a, parts);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_logprob(const LogprobArgs& a, hipStream_t st) {
  return differences_first(a.scale) ? launch_sums<true>(a, st) : launch_sums<false>(a, st);
}

hipError_t launch_logprob_bwd(const LogprobArgs& a, hipStream_t st) {
  const int per = 8 * kNT * 4, parts = (a.classes + per - 1) / per;
  logprob_bwd_kernel<<<(unsigned)((int64_t)a.rows * parts), kNT, 0, st>>>(a, parts, per);
  return hipGetLastError();
}

}  // namespace fp16k
