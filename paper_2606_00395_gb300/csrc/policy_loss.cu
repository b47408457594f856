// Clipped policy loss with a KL term over a vocabulary, and the gradient of the logits
// (pr2_policy_loss).
//
// A row needs, relative to any m, l = sum exp(z - m) and, for the entropy H = log l - e / l,
// e = sum exp(z - m) (z - m): one pass.  The token's loss and the factor of its gradient,
//   c = w (beta (1 - exp(gap)) - (shut ? 0 : r A)),
// depend on the target's log-probability alone, so a second pass over the row writes
//   grad_v = f [v = a] - (f / l) exp(z_v - m),  f = grad_scale inv_temp c
// (not exp(z - lse): where the row's values are large, lse = m + log l rounds to m).
// Exponentials are powers of two of y = logit scale - M, scale = inv_temp log2 e, one fused operation.  Its
// rounding moves a term by up to 2^-25 |y| log 2, 1.3e-6 at the |y| of 40 to 64 that an M of 0 allows, and a
// logit of nothing like that does not need its row's maximum first: so M is 0 to begin with and is set to
// the entries' maximum (rounded: it shifts l and the target's term alike) only where the sums over- or
// underrun it.  Where M would be too large to keep its fraction (a row at a
// large mask value) the difference logit - m is taken first.
//
// A row is read from HBM once.  A producer warp streams it, by bulk copies, through a ring of chunks
// in shared memory, and the chunks that fit stay there between the passes.  Of a longer row the first
// chunks are let go after the first pass and come again, from L2, after the others in the second; in
// the order of loading and of release the ring is first in, first out throughout.  The slots that the
// second pass frees take the next row's chunks.  The CTAs of a cluster may split a row: they exchange
// their three sums through distributed shared memory.  Short rows go to one warp each.
// Bound by HBM (logits read once, gradient written once), and per row by its serial part, some 3 us of
// joins, exchange and the token's own arithmetic, which the CTAs of an SM overlap.  Rows of a few KB are
// bound by that part, of which a CTA has one at a time (8192 entries of bf16 with the gradient: HBM 54 %, issue
// slots 60 %), so they have CTAs of fewer warps.  Back to back, without weights: 4096 x 131072 bf16 364 us
// with the gradient (87 % of the copy rate), 162 without (98 %); 8192 x 32001 180 us (86 %); 2048 x 131072
// fp32 349 us (91 %); 32768 x 2048 (warps) 74 us (53 %); one token of 131072 7.2 us.
// Tokens are dealt to clusters (warps) by their numbers and masks; each sums its tokens' terms in double and
// policy_finish_kernel the clusters' in order, so the loss does not depend on timing.
#include <math_constants.h>

#include <mutex>

#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLn2Rest = static_cast<float>(0.6931471805599453 - static_cast<double>(kLn2));

// ---- packed pairs of fp32 -------------------------------------------------------------------
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// ---- 16-byte vectors of a row ---------------------------------------------------------------
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int kElems = 4;
  static constexpr uint32_t kNegInf = 0xff800000u;
  static __device__ __forceinline__ float top(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
                 fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ void pairs(const uint4& v, uint64_t (&p)[2]) {
    p[0] = pack2(__uint_as_float(v.x), __uint_as_float(v.y));
    p[1] = pack2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ uint4 from_pairs(const uint64_t (&p)[2]) {
    float a, b, c, d;
    unpack2(p[0], a, b);
    unpack2(p[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kElems = 8;
  static constexpr uint32_t kNegInf = 0xff80ff80u;
  static __device__ __forceinline__ float top(const uint4& v) {
    const __nv_bfloat162 a = __hmax2(reinterpret_cast<const __nv_bfloat162&>(v.x),
                                     reinterpret_cast<const __nv_bfloat162&>(v.y));
    const __nv_bfloat162 b = __hmax2(reinterpret_cast<const __nv_bfloat162&>(v.z),
                                     reinterpret_cast<const __nv_bfloat162&>(v.w));
    const __nv_bfloat162 c = __hmax2(a, b);
    return fmaxf(__low2float(c), __high2float(c));
  }
  static __device__ __forceinline__ void pairs(const uint4& v, uint64_t (&p)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      p[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 from_pairs(const uint64_t (&p)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      unpack2(p[i], a, b);
      w[i] = pack_bf16x2(a, b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Running softmax sums over the logits above -inf relative to the logit m: with y = logit scale - M(m),
// l = sum 2^y, e = sum 2^y y.  Nothing seen: l = 0, and m means nothing.  A NaN or +inf makes l NaN.
struct RowSum {
  float m = 0.f, l = 0.f, e = 0.f;
};

// M(m) is m scale in 32 bits while its rounding, which moves every y by as much, stays below 2^-4.  Beyond
// that (finite mask values among them: at -1e10 m scale - M may be 440, whose power is infinite) it is NaN,
// and y = (logit - m) scale.
constexpr float kMostRef = 1048576.f;  // 2^20
__device__ __forceinline__ float scaled_ref(float m, float scale) {
  const float M = m * scale;
  return fabsf(M) <= kMostRef ? M : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ float power_of(float z, float m, float M, float scale) {
  return M == M ? fmaf(z, scale, -M) : (z - m) * scale;
}

// The sums relative to another logit.  (The gap is between what was subtracted and what is to be: the
// rounded M where there is one, else the product itself.)
__device__ __forceinline__ void raise(RowSum& s, float m, float scale) {
  if (s.m == m || s.l == 0.f) {
    s.m = m;
    return;
  }
  const float from = scaled_ref(s.m, scale), to = scaled_ref(m, scale);
  const float gap = from == from ? (to == to ? from - to : fmaf(-m, scale, from))
                                 : (to == to ? fmaf(s.m, scale, -to) : (s.m - m) * scale);
  const float f = exp2_approx(gap);
  s.e = f == 0.f ? s.l * f : fmaf(gap, s.l, s.e) * f;
  s.l *= f;
  s.m = m;
}

__device__ __forceinline__ void add_one(RowSum& s, float z, float scale) {
  if (z == -CUDART_INF_F) return;
  if (z > s.m || s.l == 0.f) raise(s, z, scale);
  const float y = power_of(z, s.m, scaled_ref(s.m, scale), scale), p = exp2_approx(y);
  s.l += p;
  s.e = p != 0.f ? fmaf(p, y, s.e) : s.e;  // (y may be -inf)
}

// Vectors src[v], src[v + stride], ... below n, kVecs of them at most, relative to their maximum or
// s.m, whichever is larger (if s has sums); entries of -inf left out.
template <typename T, int kVecs>
__device__ __noinline__ RowSum add_careful(RowSum s, const uint4* src, int v, int stride, int n, float scale) {
  constexpr int kPairs = Vec<T>::kElems / 2;
  float top = -CUDART_INF_F;
#pragma unroll
  for (int j = 0; j < kVecs; ++j)
    if (v + j * stride < n) top = fmaxf(top, Vec<T>::top(src[v + j * stride]));
  if (top > s.m || s.l == 0.f) raise(s, top, scale);
  const float M = scaled_ref(s.m, scale);
#pragma unroll 1
  for (int j = 0; j < kVecs; ++j) {
    if (v + j * stride >= n) break;
    uint64_t z[kPairs];
    Vec<T>::pairs(src[v + j * stride], z);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      float x[2];
      unpack2(z[i], x[0], x[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float y = power_of(x[h], s.m, M, scale), p = exp2_approx(y);
        if (x[h] != -CUDART_INF_F) {
          s.l += p;
          s.e = p != 0.f ? fmaf(p, y, s.e) : s.e;
        }
      }
    }
  }
  return s;
}

// y, or if it is lower a power far below 2^-126 (so that an entry of -inf gives 0 in both sums); a NaN
// stays one.
__device__ __forceinline__ float at_least(float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(y), "f"(-16384.f));
  return r;
}

// The two sums over 16 entries relative to M, in the order of pairs.
template <typename T>
__device__ __forceinline__ void sum_16(const uint4 (&raw)[16 / Vec<T>::kElems], float M, float scale, float& l,
                                       float& e) {
  constexpr int kVecs = 16 / Vec<T>::kElems, kPairs = Vec<T>::kElems / 2;
  const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(-M, -M);
  uint64_t l2 = 0, e2 = 0;
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    uint64_t z[kPairs];
    Vec<T>::pairs(raw[j], z);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      float a, b;
      unpack2(fma2(z[i], scale2, ref2), a, b);
      a = at_least(a);
      b = at_least(b);
      const uint64_t p2 = pack2(exp2_approx(a), exp2_approx(b));
      l2 = add2(l2, p2);
      e2 = fma2(p2, pack2(a, b), e2);
    }
  }
  float a, b;
  unpack2(l2, a, b);
  l = a + b;
  unpack2(e2, a, b);
  e = a + b;
}

// 16 entries, the vectors src[v], src[v + stride], ... which are in raw.  They are summed relative to
// s.m as it is; where that does not do (M is NaN, the sum is too large for it or so small that entries
// that matter may have vanished, an entry is NaN) they go the careful way.  M: scaled_ref(s.m), kept by
// the caller.
template <typename T>
__device__ __forceinline__ void add_vectors(RowSum& s, float& M, const uint4 (&raw)[16 / Vec<T>::kElems],
                                            const uint4* src, int v, int stride, int n, float scale) {
  constexpr float kMost = 1.0995116e12f, kLeast = 8.6736174e-19f;  // 2^40, 2^-60
  float l, e;
  sum_16<T>(raw, M, scale, l, e);
  if (l > kLeast && l < kMost) {
    s.l += l;
    s.e += e;
  } else {
    s = add_careful<T, 16 / Vec<T>::kElems>(s, src, v, stride, n, scale);
    M = scaled_ref(s.m, scale);
  }
}

// Where a row lies: `head` entries before its first 16-byte boundary, nvec whole vectors, then
// `tail` entries.
struct RowShape {
  int head, tail, nvec;
};
template <typename T>
__device__ __forceinline__ RowShape row_shape(const T* row, int V) {
  constexpr int E = Vec<T>::kElems;
  const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
  RowShape s;
  s.head = off != 0 ? E - off : 0;
  if (s.head > V) s.head = V;
  s.nvec = (V - s.head) / E;
  s.tail = V - s.head - s.nvec * E;
  return s;
}

template <typename T>
__device__ __forceinline__ uint4 no_entries() {
  return make_uint4(Vec<T>::kNegInf, Vec<T>::kNegInf, Vec<T>::kNegInf, Vec<T>::kNegInf);
}

// Sums over vectors src[0 .. n), thread `tid` of kStride taking each kStride-th.  kWhole vectors (a
// multiple of 16 kStride entries) go without bounds.
template <typename T, int kStride, int kWhole>
__device__ __forceinline__ void sum_span(RowSum& s, const uint4* src, int n, int tid, float scale) {
  constexpr int kVecs = 16 / Vec<T>::kElems;
  static_assert(kWhole % (kStride * kVecs) == 0, "whole steps");
  float M = scaled_ref(s.m, scale);
  if (n == kWhole) {
#pragma unroll
    for (int base = 0; base < kWhole; base += kStride * kVecs) {
      uint4 raw[kVecs];
#pragma unroll
      for (int j = 0; j < kVecs; ++j) raw[j] = src[base + j * kStride + tid];
      add_vectors<T>(s, M, raw, src, base + tid, kStride, n, scale);
    }
    return;
  }
  for (int base = 0; base < n; base += kStride * kVecs) {
    uint4 raw[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const int v = base + j * kStride + tid;
      raw[j] = v < n ? src[v] : no_entries<T>();
    }
    add_vectors<T>(s, M, raw, src, base + tid, kStride, n, scale);
  }
}

// What the second pass needs of a row.
struct RowGrad {
  float f, fl, m, M, za;  // factor, factor / l, the sums' m and M(m), the target's logit
};

template <typename T>
__device__ __forceinline__ T grad_one(float z, const RowGrad& g, float scale, bool target) {
  return from_f32<T>(fmaf(-g.fl, exp2_approx(power_of(z, g.m, g.M, scale)), target ? g.f : 0.f));
}

// The gradient of one vector but for the target's f.
template <typename T>
__device__ __forceinline__ uint4 grad_vector(const uint4& v, const RowGrad& g, float scale) {
  constexpr int kPairs = Vec<T>::kElems / 2;
  const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(-g.M, -g.M), fl2 = pack2(-g.fl, -g.fl);
  uint64_t z[kPairs];
  Vec<T>::pairs(v, z);
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    float a, b;
    unpack2(fma2(z[i], scale2, ref2), a, b);
    z[i] = mul2(pack2(exp2_approx(a), exp2_approx(b)), fl2);
  }
  return Vec<T>::from_pairs(z);
}

// Gradient of vectors 0 .. n - 1, which load(v) gives, to out (the entry of vector 0; 16-byte aligned
// or not), thread `tid` of kStride taking each kStride-th.  f = 0 writes zeros and loads nothing.
// `at`: the target's entry relative to out, or outside.
template <typename T, int kStride, int kWhole, typename Load>
__device__ __forceinline__ void grad_span(Load load, T* out, int n, int tid, const RowGrad& g, float scale,
                                          int at) {
  constexpr int E = Vec<T>::kElems;
  if ((reinterpret_cast<uintptr_t>(out) & 15u) != 0 || (g.f != 0.f && g.M != g.M)) {
    // rows of another alignment than the logits', rows without an M
    for (int v = tid; v < n; v += kStride) {
      const uint4 w = g.f != 0.f ? load(v) : make_uint4(0u, 0u, 0u, 0u);
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int i = 0; i < E; ++i)
        out[v * E + i] = g.f != 0.f ? grad_one<T>(to_f32<T>(e[i]), g, scale, false) : from_f32<T>(0.f);
    }
  } else {
    uint4* dst = reinterpret_cast<uint4*>(out);
    if (g.f == 0.f) {
      for (int v = tid; v < n; v += kStride) __stcs(dst + v, make_uint4(0u, 0u, 0u, 0u));
    } else if (n == kWhole) {
#pragma unroll
      for (int v = 0; v < kWhole; v += kStride) __stcs(dst + v + tid, grad_vector<T>(load(v + tid), g, scale));
    } else {
      for (int v = tid; v < n; v += kStride) __stcs(dst + v, grad_vector<T>(load(v), g, scale));
    }
  }
  if (g.f != 0.f && at >= 0 && at < n * E && (at / E) % kStride == tid)  // by the thread that wrote its vector
    out[at] = grad_one<T>(g.za, g, scale, true);
}

// ---- a warp's entries joined ------------------------------------------------------------------
// (of kLanes neighbouring lanes, in all of them)
template <int kLanes>
__device__ __forceinline__ RowSum join_lanes(RowSum s, float scale) {
  float m = s.l == 0.f ? -CUDART_INF_F : s.m;
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  raise(s, m, scale);
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    s.l += __shfl_xor_sync(0xffffffffu, s.l, o);
    s.e += __shfl_xor_sync(0xffffffffu, s.e, o);
  }
  return s;
}

// ---- a token ------------------------------------------------------------------------------------
struct Token {
  int t;
  float w;  // 0: does not count (or beyond the batch)
  int target;
};
__device__ __forceinline__ Token load_token(const PolicyArgs& a, int t) {
  Token k{t, 0.f, 0};
  if (t < a.T) {
    k.w = a.weight != nullptr ? a.weight[t] : 1.f / static_cast<float>(a.T);
    k.target = a.target[t];
  }
  return k;
}
// A target out of range counts as weight 0.  `flag`: this thread records it.
__device__ __forceinline__ void check_token(const PolicyArgs& a, Token& k, bool flag) {
  if (k.w != 0.f && (k.target < 0 || k.target >= a.V)) {
    k.w = 0.f;
    if (flag && a.status != nullptr) atomicOr(a.status, PR2_STATUS_BAD_INDEX);
  }
}

struct TokenIn {
  float A, old, ref, za;
};
// (all but za, which needs a checked token)
__device__ __forceinline__ TokenIn load_inputs(const PolicyArgs& a, int t) {
  TokenIn in{0.f, 0.f, 0.f, 0.f};
  if (t < a.T) {
    in.A = a.advantage[t];
    if (a.logp_old != nullptr) in.old = a.logp_old[t];
    if (a.logp_ref != nullptr) in.ref = a.logp_ref[t];
  }
  return in;
}
template <typename T>
__device__ __forceinline__ float load_target(const PolicyArgs& a, const Token& k) {
  if (k.w == 0.f) return 0.f;
  return to_f32<T>(static_cast<const T*>(a.logits)[static_cast<int64_t>(k.t) * a.ld_logits + k.target]);
}

// The token's terms from its row's sums: adds them to sums[] (policy part, KL part, clip flag, each
// times the weight) and gives the row's gradient factors.  `write`: this thread stores logp and
// entropy and keeps the sums.
__device__ __forceinline__ RowGrad finish_token(const PolicyArgs& a, const Token& k, const TokenIn& in,
                                                const RowSum& s, float scale, bool write,
                                                double (&sums)[3]) {
  RowGrad g{0.f, 0.f, 0.f, 0.f, in.za};
  if (s.l == 0.f) {  // no entry above -inf
    if (write) {
      if (a.logp != nullptr) a.logp[k.t] = -CUDART_INF_F;
      if (a.entropy != nullptr) a.entropy[k.t] = 0.f;
    }
    return g;
  }
  const float mean = s.e / s.l;
  const float M = scaled_ref(s.m, scale);
  // The target's y, as the sums took it, and in `slip` what log 2 times it lacks: the rest of its product and
  // differences, less what its own power in l has of that (an l that is mostly the target's moves with it),
  // and what rounding scale and log 2 to 32 bits did (the same to all tokens, so that it would not average
  // out in the loss): to first order scale_slip moves a y by its own multiple, log l by that of the mean
  // y, and log 2 is a factor of y - n.  l = 2^n part with 1 <= part < 2, so logp = (y - n) log 2 - log part, and its
  // distance from another log-probability x is taken as one fused product less x: the ratio does not
  // lose what the logarithm of a large l would.  (A NaN or infinity stays in part; an infinite y, a
  // target that is banned, has no rest.)
  const uint32_t bits = __float_as_uint(s.l);
  const int n = bits < 0x7f800000u ? static_cast<int>(bits >> 23) - 127 : 0;
  const float log_part = logf(__uint_as_float(bits - (static_cast<uint32_t>(n) << 23)));
  const float nf = static_cast<float>(n), y = power_of(in.za, s.m, M, scale), yn = y - nf;
  float slip = 0.f;
  if (fabsf(y) < CUDART_INF_F) {
    const float back_n = yn - y;
    float rest = (y - (yn - back_n)) - (nf + back_n);
    if (M == M) {
      const float p = in.za * scale, d = p - M, back = d - p;
      const float lacks = (d - y) + ((p - (d - back)) - (M + back)) + fmaf(in.za, scale, -p);
      rest = fmaf(lacks, 1.f - __fdividef(exp2_approx(y), s.l), rest);
    }
    slip = fmaf(rest, kLn2, fmaf(yn, kLn2Rest, a.scale_slip * (y - mean)));
  }
  auto logp_less = [&](float x) { return fmaf(yn, kLn2, -x) - log_part + slip; };
  // (a finite logit may be infinite as a multiple of log 2; of l only a NaN counts beside it)
  const float far = (M == M ? in.za : in.za - s.m) * a.inv_temp - log_part;
  const float logp = y == -CUDART_INF_F ? far : logp_less(0.f);
  if (write) {  // (no log-probability is above 0, no entropy below; a NaN stays one)
    if (a.logp != nullptr) a.logp[k.t] = logp > 0.f ? 0.f : logp;
    const float entropy = fmaf(kLn2, nf - mean, log_part);
    if (a.entropy != nullptr) a.entropy[k.t] = entropy < 0.f ? 0.f : entropy;
  }
  const float A = in.A;
  const float r = a.logp_old != nullptr ? expf(logp_less(in.old)) : 1.f;
  const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
  // min(r A, clip(r) A) takes the clipped side exactly where the clip shuts the gradient off; a NaN
  // ratio goes through.  A token of advantage 0 has no policy part, however large its ratio.
  const bool shut = A > 0.f ? r > hi : A < 0.f && r < lo;
  const float part = A == 0.f ? 0.f : (shut ? (A > 0.f ? hi : lo) : r) * A;
  float c = shut || A == 0.f ? 0.f : -r * A;
  float kl = 0.f;
  if (a.logp_ref != nullptr) {
    const float gap = -logp_less(in.ref), x = expm1f(gap);
    kl = isinf(x) ? x : x - gap;
    if (a.kl_coef > 0.f) c -= a.kl_coef * x;
  }
  if (write) {
    sums[0] -= k.w * part;
    sums[1] += k.w * kl;
    sums[2] += shut ? k.w : 0.f;
  }
  g.f = k.w * c * a.inv_temp * a.grad_scale;
  g.fl = g.f / s.l;
  g.m = s.m;
  g.M = M;
  return g;
}

__device__ __forceinline__ void spoil(double (&s)[3], bool timed_out) {
  if (timed_out)
#pragma unroll
    for (int j = 0; j < 3; ++j) s[j] = CUDART_NAN;
}
__device__ __forceinline__ void write_loss(const PolicyArgs& a, const double (&s)[3]) {
  a.loss[0] = static_cast<float>(a.kl_coef > 0.f ? s[0] + a.kl_coef * s[1] : s[0]);
#pragma unroll
  for (int j = 0; j < 3; ++j) a.loss[1 + j] = static_cast<float>(s[j]);
}

// ---- rows through a ring of chunks -----------------------------------------------------------------
// Consumer warps of a CTA, its ring, and CTAs an SM.  Bf16 rows, T = 4096, us with wide / narrow: V = 5128
// 40.0 / 31.1, 8192 40.8 / 36.0, 12000 52.5 / 45.4, 24000 74.8 / 77.5, 50001 155 / 169.
struct WideRows {
  static constexpr int kWarps = 8, kRing = 4, kChunkVecs = 1024, kCtas = 3;
};
struct NarrowRows {
  static constexpr int kWarps = 4, kRing = 5, kChunkVecs = 512, kCtas = 5;
};
// With the gradient a CTA's loads pause while its row's sums are joined, and a round has that cost however
// short the slices are: long rows in large batches take fewer CTAs an SM with longer slices.  Bf16, T = 4096,
// us with wide / deep: V = 50000 152 / 146, 65000 208 / 179, 98000 296 / 311, 131072 396 / 360, 260000 815 / 731;
// T = 450, V = 65536 26.5 / 29.9 (two rounds against one and a half).  Forward alone wide is faster, 161 / 174.
struct DeepRows {
  static constexpr int kWarps = 8, kRing = 7, kChunkVecs = 1024, kCtas = 2;
};
// Without the gradient, where a row need not stay in the ring.  Bf16, us with wide / forward: 8192 x 16384
// 61.0 / 58.6, 8192 x 50001 145.9 / 136.0, 700 x 50001 23.1 / 20.2, 8192 x 65536 164 / 172.
struct ForwardRows {
  static constexpr int kWarps = 4, kRing = 4, kChunkVecs = 512, kCtas = 6;
};
constexpr int kNarrowVecs = 1536;   // most vectors of a row for NarrowRows
constexpr int kForwardVecs = 6400;  // for ForwardRows
constexpr int kDeepVecs = 6400;     // fewest vectors of a CTA's slice for DeepRows
constexpr int kTokens = 3;  // rows between the producer and the last to be done with them

// A row's token as the producer hands it to the consumers.
struct TokenRecord {
  int t;  // T: no more
  float w;
  int target;
  TokenIn in;
};

// A place in the ring: slot and how often the ring went round (its parity).
template <int kRing>
struct RingAt {
  int slot;
  uint32_t round;
  __device__ __forceinline__ void step() {
    if (++slot == kRing) {
      slot = 0;
      round ^= 1u;
    }
  }
};

__device__ __forceinline__ void arrive_cluster(uint64_t* bar, uint32_t rank) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                   mapa_shared(smem_u32(bar), rank))
               : "memory");
}
__device__ __forceinline__ void st_cluster(int* shared, uint32_t rank, int v) {
  asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(mapa_shared(smem_u32(shared), rank)), "r"(v) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded, as mbar_wait.
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag,
                                             int32_t* status) {
  if (try_wait_cluster(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t it = 1;; ++it) {
    if (try_wait_cluster(bar, parity)) return true;
    if ((it & 63u) == 0u) {
      if (*abort_flag) return false;
      if (globaltimer_ns() - t0 > kWaitLimitNs) {
        *abort_flag = 1;
        if (status != nullptr) atomicOr(status, PR2_STATUS_TIMEOUT);
        return false;
      }
    }
  }
}

// ---- which cluster takes which token ---------------------------------------------------------------
// Masked tokens take a fraction of the others' time, so with weights both kinds are dealt out evenly where that
// pays.  The first `groups` tokens go to the clusters in order: a cluster's first row is asked for before the
// deal is read.  The others stand in a list, those that count first, and its first D, D the masked tokens among
// the first `groups`, go to the clusters that began with those; from there on all take turns.  order: D;
// [groups] a cluster's place among the D, -1: none; [T - groups] the list.
// The deal is a launch in front of the rows, which wait for it (1 to 3 us), and reading the list costs each row
// something, so it is made for long rows in batches of some size only (deals).  us by number / dealt, with none, a
// tenth, three tenths and half of the tokens masked:
//   gradient, bf16  4096 x 131072 367/369 361/343 328/305 289/267    8192 x 32001 178/180 175/168 175/148 158/137
//                   32768 x 16384 369/380 350/351 310/307 296/271
//                   1200 x 32001 39.2/41.2 37.6/40.0 35.5/35.1 32.7/32.2
//                   8192 x 8192 60.9/64.5 60.0/60.5 56.2/53.0 51.1/45.9   65536 x 16384 727/748 691/695 607/607 561/538
//   forward, bf16   4096 x 131072 163/168 156/150 138/120 114/91     8192 x 50001 134/138 131/126 123/103 100/79
//                   1500 x 131072 66.5/71.3 64.2/65.5 61.3/53.3 55.7/45.7
//                   2048 x 65000 49.1/54.0 48.2/50.1 45.0/43.3 41.6/35.5
//                   16384 x 16384 100/107 96/99 86/83 71/69    65536 x 32000 654/675 612/615 507/499 393/381
//   forward, fp32   8192 x 32768 162/166 149/152 123/122 91/93
//                   2400 x 32001 53.6/58.2 50.1/53.4 42.1/44.0 35.8/34.7
constexpr int kDealThreads = 1024, kDealVecs = 8;

__global__ void __launch_bounds__(kDealThreads) policy_deal_kernel(const float* weight, int T, int groups,
                                                                   int* order) {
  __shared__ int3 warp_sum[32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int* place = order + 1;
  int* list = place + groups;
  int3 all = make_int3(0, 0, 0);  // tokens so far: that count, masked, masked among the first
  for (int base = 0; base < T; base += kDealThreads * kDealVecs) {
    const int t0 = base + warp * 32 * kDealVecs + lane;
    float w[kDealVecs];
#pragma unroll
    for (int j = 0; j < kDealVecs; ++j) w[j] = t0 + j * 32 < T ? weight[t0 + j * 32] : 0.f;
    uint32_t live[kDealVecs], dead[kDealVecs], head[kDealVecs];
    int3 mine = make_int3(0, 0, 0);
#pragma unroll
    for (int j = 0; j < kDealVecs; ++j) {
      const int t = t0 + j * 32;
      live[j] = __ballot_sync(0xffffffffu, t >= groups && t < T && w[j] != 0.f);
      dead[j] = __ballot_sync(0xffffffffu, t >= groups && t < T && w[j] == 0.f);
      head[j] = __ballot_sync(0xffffffffu, t < groups && w[j] == 0.f);
      mine.x += __popc(live[j]);
      mine.y += __popc(dead[j]);
      mine.z += __popc(head[j]);
    }
    __syncthreads();  // (the sums of the tokens before have been read)
    if (lane == 0) warp_sum[warp] = mine;
    __syncthreads();
    int3 s = warp_sum[lane];
    const int3 own = s;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, s.x, o), y = __shfl_up_sync(0xffffffffu, s.y, o);
      const int z = __shfl_up_sync(0xffffffffu, s.z, o);
      if (lane >= o) s.x += x, s.y += y, s.z += z;
    }
    int l = all.x + __shfl_sync(0xffffffffu, s.x - own.x, warp);
    int d = all.y + __shfl_sync(0xffffffffu, s.y - own.y, warp);
    int h = all.z + __shfl_sync(0xffffffffu, s.z - own.z, warp);
    all.x += __shfl_sync(0xffffffffu, s.x, 31);
    all.y += __shfl_sync(0xffffffffu, s.y, 31);
    all.z += __shfl_sync(0xffffffffu, s.z, 31);
    const uint32_t lower = (1u << lane) - 1u;
#pragma unroll
    for (int j = 0; j < kDealVecs; ++j) {
      const int t = t0 + j * 32;
      if (live[j] >> lane & 1u) list[l + __popc(live[j] & lower)] = t;
      if (dead[j] >> lane & 1u) list[T - groups - 1 - (d + __popc(dead[j] & lower))] = t;
      if (t < groups) place[t] = head[j] >> lane & 1u ? h + __popc(head[j] & lower) : -1;
      l += __popc(live[j]);
      d += __popc(dead[j]);
      h += __popc(head[j]);
    }
  }
  if (threadIdx.x == 0) *order = all.z;
}

// A cluster's tokens after its first.
struct Turns {
  const int* list;  // NULL: by number
  int T, groups, own, at, n, extra;

  __device__ __forceinline__ void begin(const int* order) {
    if (order == nullptr) {
      list = nullptr;
      at = own + groups;
      return;
    }
    list = order + 1 + groups;
    n = T - groups;
    extra = __ldcg(order);
    at = __ldcg(order + 1 + own);
    if (at < 0) at = extra + own;
  }
  __device__ __forceinline__ int next() {  // T: none left
    if (list == nullptr) {
      const int t = at < T ? at : T;
      at = t < T ? t + groups : T;
      return t;
    }
    if (at >= n) return T;
    const int t = __ldcg(list + at);
    at = at < extra ? extra + own : at + groups;
    return t;
  }
};

// A CTA's part of a row: `n` vectors from vector v0 on, in `chunks` chunks.
struct Slice {
  RowShape sh;
  int n, chunks;
};

// Warps of a CTA: consumers, a producer and without the gradient a finisher, which joins a row's sums while the
// consumers take the next row (with it they wait for the row's factors anyway: one of them joins).  Forward, bf16,
// T = 8192, us with a consumer / a finisher: V = 8192 47.0 / 40.7, 16384 72.5 / 61.3, 32000 108.6 / 97.2.
template <typename Rows, bool kGrad>
constexpr int warps_of() {
  return Rows::kWarps + (kGrad ? 1 : 2);
}

// C CTAs a row, `cap` vectors each at most.
template <typename T, typename Rows, bool kGrad>
__global__ void __launch_bounds__(32 * warps_of<Rows, kGrad>(), Rows::kCtas)
    policy_row_kernel(const PolicyArgs a, int C, int cap) {
  constexpr int kWarps = Rows::kWarps, kThreads = 32 * kWarps, kRing = Rows::kRing;
  constexpr int kChunkVecs = Rows::kChunkVecs;
  extern __shared__ uint4 ring[];
  __shared__ float4 part[kTokens][kWarps];
  __shared__ float4 xchg[2][kMaxCluster];
  __shared__ RowGrad row_grad;
  __shared__ TokenRecord record[kTokens];
  __shared__ uint64_t full[kRing], empty[kRing], met[2], told[kTokens], read[kTokens];
  __shared__ uint64_t joined[kTokens], graded;
  __shared__ int abort_flag_s;
  volatile int* abort_flag = &abort_flag_s;
  constexpr int E = Vec<T>::kElems;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  if (tid == 0) {
    abort_flag_s = 0;
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], kWarps);
    }
    for (int i = 0; i < kTokens; ++i) {
      mbar_init(&told[i], 1);
      mbar_init(&read[i], kWarps + (kGrad ? 0 : 1));
      mbar_init(&joined[i], kWarps);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&met[i], C);
    mbar_init(&graded, 1);
    fence_mbar_init();
  }
  if (C > 1)
    cluster_sync();  // peers arrive here from the first row on
  else
    __syncthreads();
  pdl_wait();
  pdl_trigger();
  const T* logits = static_cast<const T*>(a.logits);
  const int groups = static_cast<int>(gridDim.x) / C, first = static_cast<int>(blockIdx.x) / C;
  const int v0 = rank * cap;
  auto row_of = [&](int t) { return logits + t * a.ld_logits; };
  auto slice_of = [&](int t) {
    Slice s;
    s.sh = row_shape(row_of(t), static_cast<int>(a.V));
    const int left = s.sh.nvec - v0;
    s.n = left < 0 ? 0 : left < cap ? left : cap;
    s.chunks = static_cast<int>((s.n + kChunkVecs - 1) / kChunkVecs);
    return s;
  };

  // Every wait is bounded and decided by the whole warp; a warp whose wait ran out leaves.
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, a.status)) != 0;
  };
  const float scale = a.scale;
  // A warp joins the sums of the CTA's row number `live` and finishes its token.
  auto join_row = [&](const Token& cur, const TokenIn& in, uint32_t live, double (&sums)[3], RowGrad& g) {
    const uint32_t third = live % kTokens, half = live & 1u;
    if (!wait(&joined[third], (live / kTokens) & 1u)) return false;
    const float4 own = part[third][lane % kWarps];
    RowSum s = join_lanes<kWarps>(RowSum{own.x, own.y, own.z}, scale);
    if (C > 1) {
      // A peer one row ahead writes the other half of xchg, and none is two ahead.
      if (lane < C) {
        st_cluster_v4(mapa_shared(smem_u32(&xchg[half][rank]), lane), __float_as_uint(s.m), __float_as_uint(s.l),
                      __float_as_uint(s.e), 0u);
        arrive_cluster(&met[half], lane);
      }
      if (!__all_sync(0xffffffffu, wait_cluster(&met[half], (live >> 1) & 1u, abort_flag, a.status))) return false;
      const int r = lane % kMaxCluster;
      const float4 x = r < C ? xchg[half][r] : make_float4(0.f, 0.f, 0.f, 0.f);
      s = join_lanes<kMaxCluster>(RowSum{x.x, x.y, x.z}, scale);
    }
    g = finish_token(a, cur, in, s, scale, rank == 0 && lane == 0, sums);
    return true;
  };
  auto masked = [&](int t) {
    if (a.logp != nullptr) a.logp[t] = 0.f;
    if (a.entropy != nullptr) a.entropy[t] = 0.f;
  };
  // Where a wait ran out the sums are NaN: those of the tokens done by then would pass for all of them.
  auto store_sums = [&](double (&sums)[3]) {
    spoil(sums, *abort_flag);
    if (groups == 1) {
      write_loss(a, sums);
    } else {
      double* p = a.partial + static_cast<int64_t>(first) * 4;
#pragma unroll
      for (int j = 0; j < 3; ++j) p[j] = sums[j];
    }
  };

  if (warp == kWarps) {
    // ---------------- producer ----------------
    if (lane == 0) {
      RingAt<kRing> at{0, 0u};
      uint32_t landing = 0, last_round = 0;  // slots with a copy issued, and its round
      // a token's number is read three rows ahead, its weight and inputs two, its target's logit one
      const int T_all = static_cast<int>(a.T);
      const bool dealt = a.order != nullptr;
      Turns turns{nullptr, T_all, groups, first, 0, 0, 0};
      const bool late = status_timed_out(a.status);
      Token cur = load_token(a, first), next{T_all, 0.f, 0}, after = next;
      TokenIn cur_in = load_inputs(a, first), next_in{}, after_in{};
      int ahead = T_all;
      auto begin_turns = [&] {
        turns.begin(a.order);
        const int t = turns.next();
        ahead = turns.next();
        next = load_token(a, t);
        next_in = load_inputs(a, t);
      };
      auto look_ahead = [&] {
        after = load_token(a, ahead);
        after_in = load_inputs(a, ahead);
        ahead = turns.next();
        check_token(a, next, rank == 0);
        next_in.za = load_target<T>(a, next);
      };
      if (!dealt) begin_turns();
      check_token(a, cur, rank == 0);
      cur_in.za = load_target<T>(a, cur);
      if (late) *abort_flag = 1;  // an earlier call's wait ran out: the inputs may be unwritten
      uint32_t row = 0;
      bool ok = true;
      for (;;) {
        if (row > 0 || !dealt) look_ahead();
        Slice s{};
        const char* src = nullptr;
        int again = 0;
        if (cur.w != 0.f) {
          s = slice_of(cur.t);
          src = reinterpret_cast<const char*>(row_of(cur.t) + s.sh.head) + static_cast<int64_t>(v0) * 16;
          again = kGrad && s.chunks > kRing ? s.chunks - kRing : 0;
        }
        auto load_chunks = [&](int from, int to) {
          for (int i = from; i < to && ok; ++i) {
            const int v = (i < s.chunks ? i : i - s.chunks) * kChunkVecs;
            const int left = s.n - v;
            const uint32_t bytes = static_cast<uint32_t>(left < kChunkVecs ? left : kChunkVecs) * 16u;
            ok = mbar_wait(&empty[at.slot], at.round ^ 1u, abort_flag, a.status);
            if (!ok) break;
            mbar_arrive_expect_tx(&full[at.slot], bytes);
            bulk_load(smem_u32(ring + at.slot * kChunkVecs), src + static_cast<int64_t>(v) * 16, bytes, &full[at.slot]);
            landing |= 1u << at.slot;
            last_round = (last_round & ~(1u << at.slot)) | (at.round << at.slot);
            at.step();
          }
        };
        // The first row's chunks go on their way before the record is told, which waits for the target's
        // logit; later on the consumers may need the record to free a chunk.
        const int chunks = s.chunks + again, early = row > 0 ? 0 : chunks < kRing ? chunks : kRing;
        load_chunks(0, early);
        const int rec = row % kTokens;
        if (ok) ok = mbar_wait(&read[rec], ((row / kTokens) & 1u) ^ 1u, abort_flag, a.status);
        if (!ok) break;
        record[rec] = TokenRecord{cur.t, cur.w, cur.target, cur_in};
        mbar_arrive(&told[rec]);
        load_chunks(early, chunks);
        if (!ok || cur.t >= T_all) break;
        if (row == 0 && dealt) {
          begin_turns();
          look_ahead();
        }
        cur = next;
        cur_in = next_in;
        next = after;
        next_in = after_in;
        ++row;
      }
      // no copy may still be landing when the CTA leaves (the consumers may have given up)
      for (int i = 0; i < kRing; ++i)
        if ((landing >> i) & 1u)
          mbar_wait_slow(&full[i], (last_round >> i) & 1u, nullptr, nullptr, kDrainLimitNs);
    }
  } else if (!kGrad && warp > kWarps) {
    // ---------------- finisher ----------------
    double sums[3] = {0.0, 0.0, 0.0};
    uint32_t live = 0;  // rows joined so far
    for (uint32_t turn = 0;; ++turn) {
      const int rec = turn % kTokens;
      if (!wait(&told[rec], (turn / kTokens) & 1u)) break;
      const Token cur{record[rec].t, record[rec].w, record[rec].target};
      if (cur.t >= a.T) break;
      RowGrad g;
      if (cur.w != 0.f) {
        if (!join_row(cur, record[rec].in, live++, sums, g)) break;
      } else if (rank == 0 && lane == 0) {
        masked(cur.t);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&read[rec]);
    }
    if (rank == 0 && lane == 0) store_sums(sums);
  } else {
    // ---------------- consumers ----------------
    // A warp writes part and joined of a row only when their reader is done with the row kTokens before: it has
    // the row's record, for which the producer waits for all readers.
    T* grad = static_cast<T*>(a.grad);
    RingAt<kRing> in_at{0, 0u}, out_at{0, 0u};  // the next chunk to come, the next one to let go
    double sums[3] = {0.0, 0.0, 0.0};
    uint32_t live = 0;  // rows joined so far
    auto let_go = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[out_at.slot]);
      out_at.step();
    };
    auto vecs_of = [&](const Slice& s, int c) {
      const int left = s.n - c * kChunkVecs;
      return left < kChunkVecs ? left : kChunkVecs;
    };
    bool ok = true;
    for (uint32_t turn = 0;; ++turn) {
      const int rec = turn % kTokens;
      if (!wait(&told[rec], (turn / kTokens) & 1u)) break;
      const Token cur{record[rec].t, record[rec].w, record[rec].target};
      if (cur.t >= a.T) break;
      const Slice sl = slice_of(cur.t);
      // the entries outside whole vectors: threads 0-7 the head's, 8-15 the tail's, of rank 0
      int edge = -1;
      if (rank == 0 && tid < 16) {
        if (tid < 8 && tid < sl.sh.head) edge = tid;
        if (tid >= 8 && tid - 8 < sl.sh.tail) edge = static_cast<int>(a.V) - sl.sh.tail + (tid - 8);
      }
      float ez = 0.f;
      RowGrad g{0.f, 0.f, 0.f, 0.f, 0.f};
      const bool counts = cur.w != 0.f;
      const int again = !kGrad ? sl.chunks : sl.chunks > kRing ? sl.chunks - kRing : 0;
      if (counts) {
        RowSum s;
        if (edge >= 0) ez = to_f32<T>(row_of(cur.t)[edge]);
        for (int c = 0; c < sl.chunks; ++c) {
          if (!(ok = wait(&full[in_at.slot], in_at.round))) break;
          sum_span<T, kThreads, kChunkVecs>(s, ring + in_at.slot * kChunkVecs, vecs_of(sl, c), tid, scale);
          in_at.step();
          if (c < again) let_go();
        }
        if (!ok) break;
        if (edge >= 0) add_one(s, ez, scale);
        s = join_lanes<32>(s, scale);
        if (lane == 0) {
          part[live % kTokens][warp] = make_float4(s.m, s.l, s.e, 0.f);
          mbar_arrive(&joined[live % kTokens]);
        }
        if (kGrad) {
          if (warp == 0) {
            if (!join_row(cur, record[rec].in, live, sums, g)) break;
            if (lane == 0) {
              row_grad = g;
              mbar_arrive(&graded);
            }
          }
          if (!wait(&graded, live & 1u)) break;
          g = row_grad;
        }
        ++live;
      } else if (kGrad && rank == 0 && tid == 0) {
        masked(cur.t);
      }
      if (kGrad) {
        const int start = sl.sh.head + v0 * E;
        T* out = grad + cur.t * a.ld_grad + start;
        if (counts) {
          for (int i = again; i < sl.chunks + again; ++i) {
            const int c = i < sl.chunks ? i : i - sl.chunks;
            if (i >= sl.chunks) {
              if (!(ok = wait(&full[in_at.slot], in_at.round))) break;
              in_at.step();
            }
            const int e0 = c * kChunkVecs * E;
            grad_span<T, kThreads, kChunkVecs>([&](int v) { return ring[out_at.slot * kChunkVecs + v]; }, out + e0,
                                               vecs_of(sl, c), tid, g, scale, cur.target - start - e0);
            let_go();
          }
          if (!ok) break;
        } else {
          grad_span<T, kThreads, kChunkVecs>([](int) { return make_uint4(0u, 0u, 0u, 0u); }, out, sl.n, tid, g, scale,
                                             -1);
        }
        if (edge >= 0)
          grad[cur.t * a.ld_grad + edge] =
              g.f != 0.f ? grad_one<T>(ez, g, scale, edge == cur.target) : from_f32<T>(0.f);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&read[rec]);
    }
    if (kGrad && rank == 0 && tid == 0) store_sums(sums);
  }
  if (C > 1) {
    __syncwarp();
    if (rank != 0 && lane == 0 && *abort_flag) st_cluster(&abort_flag_s, 0, 1);
    cluster_sync();  // no peer writes here any more (every wait before is bounded)
    if (rank == 0 && tid == 0 && *abort_flag) {
      double none[3] = {0.0, 0.0, 0.0};
      store_sums(none);
    }
  }
}

// ---- a warp per row --------------------------------------------------------------------------------
// A lane holds up to kHeld vectors of the row between the passes.
template <typename T, int kHeld>
__global__ void __launch_bounds__(kThreads, kHeld <= 8 ? 3 : 2) policy_warp_kernel(const PolicyArgs a) {
  constexpr int kVecs = 16 / Vec<T>::kElems;
  __shared__ double part[kWarps][3];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float scale = a.scale;
  const bool late = threadIdx.x == 0 && status_timed_out(a.status);  // (as in the row kernel)
  double sums[3] = {0.0, 0.0, 0.0};
  const int rows = static_cast<int>(gridDim.x) * kWarps;
  for (int t = static_cast<int>(blockIdx.x) * kWarps + warp; t < a.T; t += rows) {
    Token k = load_token(a, t);
    const T* row = static_cast<const T*>(a.logits) + t * a.ld_logits;
    const RowShape sh = row_shape(row, static_cast<int>(a.V));
    const uint4* src = reinterpret_cast<const uint4*>(row + sh.head);
    check_token(a, k, lane == 0);
    int edge = -1;
    if (lane < 8 && lane < sh.head) edge = lane;
    if (lane >= 8 && lane - 8 < sh.tail) edge = static_cast<int>(a.V) - sh.tail + (lane - 8);
    float ez = 0.f;
    RowGrad g{0.f, 0.f, 0.f, 0.f, 0.f};
    uint4 raw[kHeld];
    if (k.w != 0.f) {
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int v = j * 32 + lane;
        raw[j] = v < sh.nvec ? src[v] : no_entries<T>();
      }
      RowSum s;
      float M = scaled_ref(s.m, scale);
      TokenIn in = load_inputs(a, t);
      in.za = load_target<T>(a, k);
      if (edge >= 0) ez = to_f32<T>(row[edge]);
#pragma unroll
      for (int j = 0; j < kHeld; j += kVecs)
        if (j * 32 < sh.nvec)
          add_vectors<T>(s, M, reinterpret_cast<const uint4(&)[kVecs]>(raw[j]), src, j * 32 + lane, 32, sh.nvec, scale);
      if (edge >= 0) add_one(s, ez, scale);
      s = join_lanes<32>(s, scale);
      g = finish_token(a, k, in, s, scale, lane == 0, sums);
    } else if (lane == 0) {
      if (a.logp != nullptr) a.logp[t] = 0.f;
      if (a.entropy != nullptr) a.entropy[t] = 0.f;
    }
    if (a.grad != nullptr) {
      __syncwarp();  // (in place: every lane has read the target's logit)
      T* out = static_cast<T*>(a.grad) + t * a.ld_grad;
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int left = sh.nvec - j * 32, e0 = sh.head + j * 32 * Vec<T>::kElems;
        if (left > 0)
          grad_span<T, 32, 32>([&](int) { return raw[j]; }, out + e0, left < 32 ? left : 32, lane, g, scale,
                               k.target - e0);
      }
      if (edge >= 0)
        out[edge] = g.f != 0.f ? grad_one<T>(ez, g, scale, edge == k.target) : from_f32<T>(0.f);
    }
  }
  if (lane == 0)
#pragma unroll
    for (int j = 0; j < 3; ++j) part[warp][j] = sums[j];
  __syncthreads();
  if (threadIdx.x == 0) {
    double s[3] = {0.0, 0.0, 0.0};
    for (int w = 0; w < kWarps; ++w)
#pragma unroll
      for (int j = 0; j < 3; ++j) s[j] += part[w][j];
    spoil(s, late);
    if (gridDim.x == 1) {
      write_loss(a, s);
    } else {
      double* p = a.partial + static_cast<int64_t>(blockIdx.x) * 4;
#pragma unroll
      for (int j = 0; j < 3; ++j) p[j] = s[j];
    }
  }
}

__global__ void __launch_bounds__(256) policy_finish_kernel(const PolicyArgs a, int n) {
  __shared__ double sh[3][256];
  pdl_wait();
  pdl_trigger();
  // (64-bit additions are slow here: none of zeros)
  const int tid = threadIdx.x;
  double s[3] = {0.0, 0.0, 0.0};
  if (tid < n)
    for (int j = 0; j < 3; ++j) s[j] = a.partial[tid * 4 + j];
  for (int i = tid + 256; i < n; i += 256)
    for (int j = 0; j < 3; ++j) s[j] += a.partial[i * 4 + j];
  for (int j = 0; j < 3; ++j) sh[j][tid] = s[j];
  for (int o = 128; o > 0; o >>= 1) {
    __syncthreads();
    if (tid < o && tid + o < n)
      for (int j = 0; j < 3; ++j) sh[j][tid] += sh[j][tid + o];
  }
  if (threadIdx.x == 0) {
    const double all[3] = {sh[0][0], sh[1][0], sh[2][0]};
    write_loss(a, all);
  }
}

// ---- host ----------------------------------------------------------------------------------------
template <typename Rows>
constexpr size_t ring_bytes() {
  return static_cast<size_t>(Rows::kRing) * Rows::kChunkVecs * 16;
}
// (an SM has 228 KB, a CTA 1 KB of them for the system and less than 1 KB of its own beside the ring)
static_assert(WideRows::kCtas * (ring_bytes<WideRows>() + 2048) <= 228 * 1024 &&
                  NarrowRows::kCtas * (ring_bytes<NarrowRows>() + 2048) <= 228 * 1024 &&
                  DeepRows::kCtas * (ring_bytes<DeepRows>() + 2048) <= 228 * 1024 &&
                  ForwardRows::kCtas * (ring_bytes<ForwardRows>() + 2048) <= 228 * 1024,
              "the CTAs' rings fit an SM");
static_assert(kNarrowVecs <= NarrowRows::kRing * NarrowRows::kChunkVecs, "a narrow row fits its ring");

// Clusters of C CTAs of the row kernel that run at once (0 on error), cached per device and C.
template <typename T, typename Rows, bool kGrad>
int active_clusters(int C) {
  struct Entry {
    int dev, C, clusters;
  };
  static std::mutex mu;
  static Entry cache[32];
  static int used = 0;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < used; ++i)
    if (cache[i].dev == dev && cache[i].C == C) return cache[i].clusters;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C);
  cfg.blockDim = dim3(32 * warps_of<Rows, kGrad>());
  cfg.dynamicSmemBytes = ring_bytes<Rows>();
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  auto* kernel = policy_row_kernel<T, Rows, kGrad>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(ring_bytes<Rows>())) !=
          cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    return 0;
  }
  if (used < 32) cache[used++] = Entry{dev, C, n};
  return n;
}

// Whether the deal pays (figures at policy_deal_kernel).
bool deals(const PolicyArgs& a, int64_t nvec, int64_t groups) {
  const bool grad = a.grad != nullptr;
  const int64_t row = nvec * 16;  // bytes
  return a.weight != nullptr && a.T > groups && a.T <= kPolicyDealt && row >= (grad ? 32 << 10 : 64 << 10) &&
         a.T * row >= (grad ? 100000000 : 350000000);
}

// Rows over clusters of C CTAs; *parts: the clusters that take rows.
template <typename T, typename Rows, bool kGrad>
cudaError_t launch_rows(const PolicyArgs& args, int64_t nvec, int C, int64_t* parts, cudaStream_t st) {
  PolicyArgs a = args;
  int64_t groups = active_clusters<T, Rows, kGrad>(C);
  if (groups <= 0) return cudaErrorInvalidConfiguration;
  if (groups > a.T) groups = a.T;
  if (groups > kPolicyParts) groups = kPolicyParts;
  *parts = groups;
  if (deals(a, nvec, groups)) {
    const cudaError_t err = launch_pdl(policy_deal_kernel, dim3(1), dim3(kDealThreads), 0, st, 1, a.weight,
                                       static_cast<int>(a.T), static_cast<int>(groups), a.order);
    if (err != cudaSuccess) return err;
  } else {
    a.order = nullptr;
  }
  return launch_pdl(policy_row_kernel<T, Rows, kGrad>, dim3(static_cast<unsigned>(groups * C)),
                    dim3(32 * warps_of<Rows, kGrad>()), ring_bytes<Rows>(), st, C, a, C,
                    static_cast<int>((nvec + C - 1) / C));
}

// CTAs a row with the gradient.  A row that does not fit the rings is read again from L2, so the rows in
// flight have to stay there (with the gradients on their way, `bytes` of its 129 MB: with WideRows 4096 bf16
// rows of 65536 take 220 us with one CTA a row, 204 with two; with DeepRows 3400 rows of 175000 412 with two,
// 472 with four, and of 103000 282 with one, 260 with two).  No more than that, because a round's exchange of
// the sums takes its time however small the slices are (rows of 131072: 397 us with four, 510 with eight).
template <typename Rows>
int grad_cluster(int64_t T, int64_t nvec, int num_sms, int64_t bytes) {
  int C = 1;
  for (; C < kMaxCluster && nvec * 16 > static_cast<int64_t>(C * ring_bytes<Rows>()); C *= 2) {
    const int64_t rows = static_cast<int64_t>(num_sms) * Rows::kCtas / C;
    if ((T < rows ? T : rows) * nvec * 16 <= bytes) break;
  }
  return C;
}

template <typename T>
cudaError_t launch(const PolicyArgs& args, int num_sms, cudaStream_t st) {
  PolicyArgs a = args;
  const double exact = static_cast<double>(a.inv_temp) * 1.4426950408889634;
  a.scale = static_cast<float>(exact);
  a.scale_slip = static_cast<float>(0.6931471805599453 * (exact / a.scale - 1.0));
  constexpr int E = Vec<T>::kElems;
  const int64_t nvec = a.V / E;  // most whole vectors of a row
  const int64_t resident = static_cast<int64_t>(num_sms) * WideRows::kCtas;
  int64_t parts = 0;
  cudaError_t err;
  // A warp a row up to 4 KB, and up to 8 KB where the rows outnumber the CTAs that the row kernel keeps
  // resident (bf16 rows of 4096, us: 256 rows 11.3 by warps, 8.8 by rows; 2432 rows 13.3 / 24.6; rows
  // of 8192, 2432 of them 31 / 25).
  if (nvec <= 256 || (nvec <= 512 && a.T > resident)) {
    int64_t blocks = (a.T + kWarps - 1) / kWarps;
    if (blocks > kPolicyParts) blocks = kPolicyParts;
    parts = blocks;
    const dim3 grid(static_cast<unsigned>(blocks));
    err = nvec <= 128 ? launch_pdl(policy_warp_kernel<T, 4>, grid, dim3(kThreads), 0, st, 1, a)
          : nvec <= 256 ? launch_pdl(policy_warp_kernel<T, 8>, grid, dim3(kThreads), 0, st, 1, a)
                      : launch_pdl(policy_warp_kernel<T, 16>, grid, dim3(kThreads), 0, st, 1, a);
  } else if (nvec <= (a.grad != nullptr ? kNarrowVecs : kForwardVecs) && a.T > resident) {
    err = a.grad != nullptr ? launch_rows<T, NarrowRows, true>(a, nvec, 1, &parts, st)
                            : launch_rows<T, ForwardRows, false>(a, nvec, 1, &parts, st);
  } else {
    // Wider clusters also where that puts idle CTAs to work and leaves every thread four vectors.
    const int deep = a.grad == nullptr ? 1 : grad_cluster<DeepRows>(a.T, nvec, num_sms, int64_t{54} << 20);
    if (a.grad != nullptr && nvec >= static_cast<int64_t>(deep) * kDeepVecs &&
        a.T >= int64_t{4} * num_sms * DeepRows::kCtas) {
      err = launch_rows<T, DeepRows, true>(a, nvec, deep, &parts, st);
    } else {
      int C = a.grad == nullptr ? 1 : grad_cluster<WideRows>(a.T, nvec, num_sms, int64_t{48} << 20);
      while (C < kMaxCluster && a.T * C * 2 <= resident && nvec >= C * 4 * kThreads) C *= 2;
      err = a.grad != nullptr ? launch_rows<T, WideRows, true>(a, nvec, C, &parts, st)
                              : launch_rows<T, WideRows, false>(a, nvec, C, &parts, st);
    }
  }
  if (err != cudaSuccess || parts == 1) return err;  // one cluster (block) writes the loss itself
  return launch_pdl(policy_finish_kernel, dim3(1), dim3(256), 0, st, 1, a, static_cast<int>(parts));
}

}  // namespace

cudaError_t launch_policy_loss(const PolicyArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? launch<__nv_bfloat16>(a, num_sms, st) : launch<float>(a, num_sms, st);
}

}  // namespace pr2
