// Clipped policy loss with a KL term over a vocabulary, and the gradient of the logits
// (pr2_policy_loss).
//
// A row needs its maximum m, l = sum exp(z - m) and, for the entropy H = log l - e / l,
// e = sum exp(z - m) (z - m): one pass keeps a running maximum with the two sums, rescaled when it
// grows.  The token's loss and the factor of its gradient,
//   c = w (beta (1 - exp(gap)) - (shut ? 0 : r A)),
// depend on the target's log-probability alone, so a second pass over the row writes
//   grad_v = f [v = a] - (f / l) exp(z_v - m),  f = grad_scale inv_temp c
// (not exp(z - lse): where the row's values are large, lse = m + log l rounds to m).
// Exponentials are powers of two of (logit - m) (inv_temp log2 e), m the largest logit: the
// difference first, which is exact or nearly so and cannot overflow where a scaled logit could (a
// row at the type's lowest value).
//
// A row is read from HBM once: the CTAs of a cluster split it and each keeps its slice in shared
// memory (bulk copies, the next row's slice in flight) between the two passes; they exchange their
// three sums through distributed shared memory.  Short rows go to one warp each, and rows that no
// cluster's shared memory holds are read twice.
// Tokens are dealt to clusters (warps) by their number; each sums its tokens' terms in double and
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
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

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

// Running softmax sums over the logits above -inf: maximum m, and with y = (logit - m) scale
// l = sum 2^y, e = sum 2^y y.  Nothing seen: m = -inf, l = 0.  A NaN or +inf makes l NaN.
struct RowSum {
  float m, l, e;
};

// The sums relative to a larger maximum.
__device__ __forceinline__ void raise(RowSum& s, float m, float scale) {
  if (s.m == m) return;
  const float gap = (s.m - m) * scale;
  const float f = exp2_approx(gap);  // 0 from m = -inf
  s.e = s.m == -CUDART_INF_F ? s.l * f : fmaf(gap, s.l, s.e) * f;
  s.l *= f;
  s.m = m;
}

__device__ __forceinline__ void add_one(RowSum& s, float z, float scale) {
  if (z == -CUDART_INF_F) return;
  if (z > s.m) raise(s, z, scale);
  const float y = (z - s.m) * scale, p = exp2_approx(y);
  s.l += p;
  s.e = fmaf(p, y, s.e);
}

// 16 entries: their maximum first, then powers relative to the running one.  Entries of -inf give
// 0 inf in the second sum; it is taken again without them where it comes out NaN.
template <typename T>
__device__ __forceinline__ void add_vectors(RowSum& s, const uint4 (&raw)[16 / Vec<T>::kElems],
                                            float scale) {
  constexpr int kVecs = 16 / Vec<T>::kElems, kPairs = Vec<T>::kElems / 2;
  float top = Vec<T>::top(raw[0]);
#pragma unroll
  for (int j = 1; j < kVecs; ++j) top = fmaxf(top, Vec<T>::top(raw[j]));
  if (top > s.m) raise(s, top, scale);
  const float ref = s.m == -CUDART_INF_F ? 0.f : -s.m;
  const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(ref, ref);
  uint64_t l2 = 0, e2 = 0;
  float y[16];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    uint64_t z[kPairs];
    Vec<T>::pairs(raw[j], z);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const uint64_t x2 = mul2(add2(z[i], ref2), scale2);
      float a, b;
      unpack2(x2, a, b);
      const uint64_t p2 = pack2(exp2_approx(a), exp2_approx(b));
      l2 = add2(l2, p2);
      e2 = fma2(p2, x2, e2);
      y[(j * kPairs + i) * 2] = a;
      y[(j * kPairs + i) * 2 + 1] = b;
    }
  }
  float a, b;
  unpack2(l2, a, b);
  s.l += a + b;
  unpack2(e2, a, b);
  float e = a + b;
  if (e != e) {
    e = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (y[i] != -CUDART_INF_F) e = fmaf(exp2_approx(y[i]), y[i], e);
  }
  s.e += e;
}

// Where a row lies: `head` entries before its first 16-byte boundary, nvec whole vectors, then
// `tail` entries.
struct RowShape {
  int head, tail;
  int64_t nvec;
};
template <typename T>
__device__ __forceinline__ RowShape row_shape(const T* row, int64_t V) {
  constexpr int E = Vec<T>::kElems;
  const int off = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T));
  RowShape s;
  s.head = off != 0 ? E - off : 0;
  if (s.head > V) s.head = static_cast<int>(V);
  s.nvec = (V - s.head) / E;
  s.tail = static_cast<int>(V - s.head - s.nvec * E);
  return s;
}

// Sums over vectors src[0 .. n), thread `tid` of kStride taking each kStride-th.
template <typename T, int kStride>
__device__ __forceinline__ void sum_span(RowSum& s, const uint4* src, int64_t n, int tid, float scale) {
  constexpr int kVecs = 16 / Vec<T>::kElems;
  for (int64_t base = 0; base < n; base += kStride * kVecs) {
    uint4 raw[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      const int64_t v = base + j * kStride + tid;
      raw[j] = v < n ? src[v]
                     : make_uint4(Vec<T>::kNegInf, Vec<T>::kNegInf, Vec<T>::kNegInf, Vec<T>::kNegInf);
    }
    add_vectors<T>(s, raw, scale);
  }
}

// What the second pass needs of a row.
struct RowGrad {
  float f, fl, m, za;  // factor, factor / l, maximum, the target's logit
};

template <typename T>
__device__ __forceinline__ T grad_one(float z, const RowGrad& g, float scale, bool target) {
  return from_f32<T>(fmaf(-g.fl, exp2_approx((z - g.m) * scale), target ? g.f : 0.f));
}

// Gradient of vectors src[0 .. n) to out (entry `first` of the row on; 16-byte aligned or not).
// f = 0 writes zeros and reads nothing.  `at`: the target's entry relative to src, or outside.
template <typename T, int kStride>
__device__ __forceinline__ void grad_span(const uint4* src, T* out, int64_t n, int tid, const RowGrad& g,
                                          float scale, int64_t at) {
  constexpr int E = Vec<T>::kElems, kPairs = E / 2;
  if ((reinterpret_cast<uintptr_t>(out) & 15u) != 0) {  // rows of another alignment than the logits'
    const T* one = reinterpret_cast<const T*>(src);
    for (int64_t i = tid; i < n * E; i += kStride)
      out[i] = g.f != 0.f ? grad_one<T>(to_f32<T>(one[i]), g, scale, i == at) : from_f32<T>(0.f);
    return;
  }
  uint4* dst = reinterpret_cast<uint4*>(out);
  if (g.f == 0.f) {
    for (int64_t v = tid; v < n; v += kStride) __stcs(dst + v, make_uint4(0u, 0u, 0u, 0u));
    return;
  }
  const uint64_t scale2 = pack2(scale, scale), ref2 = pack2(-g.m, -g.m), fl2 = pack2(-g.fl, -g.fl);
#pragma unroll 2
  for (int64_t v = tid; v < n; v += kStride) {
    uint64_t z[kPairs];
    Vec<T>::pairs(src[v], z);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      float a, b;
      unpack2(mul2(add2(z[i], ref2), scale2), a, b);
      z[i] = mul2(pack2(exp2_approx(a), exp2_approx(b)), fl2);
    }
    __stcs(dst + v, Vec<T>::from_pairs(z));
  }
  if (at >= 0 && at < n * E && (at / E) % kStride == tid)  // by the thread that wrote its vector
    out[at] = grad_one<T>(g.za, g, scale, true);
}

// ---- a warp's entries joined ------------------------------------------------------------------
__device__ __forceinline__ RowSum join_warp(RowSum s, float scale) {
  float m = s.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  raise(s, m, scale);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s.l += __shfl_xor_sync(0xffffffffu, s.l, o);
    s.e += __shfl_xor_sync(0xffffffffu, s.e, o);
  }
  return s;
}

// ---- a token ------------------------------------------------------------------------------------
struct Token {
  int64_t t;
  float w;  // 0: does not count (or beyond the batch)
  int target;
};
__device__ __forceinline__ Token load_token(const PolicyArgs& a, int64_t t, bool flag) {
  Token k{t, 0.f, 0};
  if (t >= a.T) return k;
  k.w = a.weight != nullptr ? a.weight[t] : 1.f / static_cast<float>(a.T);
  if (k.w == 0.f) return k;
  k.target = a.target[t];
  if (k.target < 0 || k.target >= a.V) {
    k.w = 0.f;
    if (flag && a.status != nullptr) atomicOr(a.status, PR2_STATUS_BAD_INDEX);
  }
  return k;
}

struct TokenIn {
  float A, old, ref, za;
};
template <typename T>
__device__ __forceinline__ TokenIn load_inputs(const PolicyArgs& a, const Token& k) {
  TokenIn in{0.f, 0.f, 0.f, 0.f};
  if (k.w == 0.f) return in;
  in.A = a.advantage[k.t];
  if (a.logp_old != nullptr) in.old = a.logp_old[k.t];
  if (a.logp_ref != nullptr) in.ref = a.logp_ref[k.t];
  in.za = to_f32<T>(static_cast<const T*>(a.logits)[k.t * a.ld_logits + k.target]);
  return in;
}

// The token's terms from its row's sums: adds them to sums[] (policy part, KL part, clip flag, each
// times the weight) and gives the row's gradient factors.  `write`: this thread stores logp, entropy.
__device__ __forceinline__ RowGrad finish_token(const PolicyArgs& a, const Token& k, const TokenIn& in,
                                                const RowSum& s, bool write,
                                                double (&sums)[3]) {
  RowGrad g{0.f, 0.f, 0.f, in.za};
  if (s.m == -CUDART_INF_F && s.l == 0.f) {  // no entry above -inf
    if (write) {
      if (a.logp != nullptr) a.logp[k.t] = -CUDART_INF_F;
      if (a.entropy != nullptr) a.entropy[k.t] = 0.f;
    }
    return g;
  }
  const float logl = logf(s.l);
  const float logp = fmaf(in.za - s.m, a.inv_temp, -logl);
  if (write) {
    if (a.logp != nullptr) a.logp[k.t] = logp;
    if (a.entropy != nullptr) a.entropy[k.t] = fmaf(-kLn2, s.e / s.l, logl);
  }
  const float A = in.A;
  const float r = a.logp_old != nullptr ? expf(logp - in.old) : 1.f;
  const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
  // min(r A, clip(r) A) takes the clipped side exactly where the clip shuts the gradient off; a NaN
  // ratio goes through.  A token of advantage 0 has no policy part, however large its ratio.
  const bool shut = A > 0.f ? r > hi : A < 0.f && r < lo;
  const float part = A == 0.f ? 0.f : (shut ? (A > 0.f ? hi : lo) : r) * A;
  float c = shut || A == 0.f ? 0.f : -r * A;
  sums[0] -= k.w * part;
  sums[2] += shut ? k.w : 0.f;
  if (a.logp_ref != nullptr) {
    const float gap = in.ref - logp, x = expm1f(gap);
    sums[1] += k.w * (isinf(x) ? x : x - gap);
    if (a.kl_coef > 0.f) c -= a.kl_coef * x;
  }
  g.f = k.w * c * a.inv_temp * a.grad_scale;
  g.fl = g.f / s.l;
  g.m = s.m;
  return g;
}

__device__ __forceinline__ void write_loss(const PolicyArgs& a, const double (&s)[3]) {
  a.loss[0] = static_cast<float>(a.kl_coef > 0.f ? s[0] + a.kl_coef * s[1] : s[0]);
#pragma unroll
  for (int j = 0; j < 3; ++j) a.loss[1 + j] = static_cast<float>(s[j]);
}

// ---- rows split over a cluster -------------------------------------------------------------------
// `cap` vectors a CTA at most; kResident: they stay in shared memory (`slots` buffers, one row each),
// else both passes read them from global memory.
template <typename T, bool kResident>
__global__ void __launch_bounds__(kThreads)
    policy_cluster_kernel(const PolicyArgs a, int C, int64_t cap, int slots) {
  extern __shared__ uint4 data[];
  __shared__ RowSum part[kWarps];
  __shared__ float4 xchg[2][kMaxCluster];
  __shared__ RowGrad row_grad;
  __shared__ uint64_t full[2];
  __shared__ int abort_flag_s;
  volatile int* abort_flag = &abort_flag_s;
  constexpr int E = Vec<T>::kElems;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = C > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  if (tid == 0) {
    abort_flag_s = 0;
    mbar_init(&full[0], 1);
    mbar_init(&full[1], 1);
    fence_mbar_init();
  }
  if (C > 1)
    cluster_sync();  // peers write here from the first row on
  else
    __syncthreads();
  pdl_wait();
  pdl_trigger();
  const float scale = a.inv_temp * kLog2e;
  const T* logits = static_cast<const T*>(a.logits);
  T* grad = static_cast<T*>(a.grad);
  const int64_t groups = gridDim.x / C, first = blockIdx.x / C;
  const int64_t v0 = rank * cap;
  auto span = [&](const RowShape& sh) {
    const int64_t left = sh.nvec - v0;
    return left < 0 ? int64_t{0} : left < cap ? left : cap;
  };
  int issued[2] = {0, 0};
  auto issue = [&](const Token& k, int slot) {  // by thread 0
    if (k.w == 0.f) return;
    const T* row = logits + k.t * a.ld_logits;
    const RowShape sh = row_shape(row, a.V);
    const int64_t n = span(sh);
    if (n == 0) return;
    const char* src = reinterpret_cast<const char*>(row + sh.head) + v0 * 16;
    ++issued[slot];
    mbar_arrive_expect_tx(&full[slot], static_cast<uint32_t>(n * 16));
    constexpr int64_t kPiece = 8192;
    for (int64_t at = 0; at < n * 16; at += kPiece) {
      const int64_t left = n * 16 - at;
      bulk_load(smem_u32(data + slot * cap) + static_cast<uint32_t>(at), src + at,
                static_cast<uint32_t>(left < kPiece ? left : kPiece), &full[slot]);
    }
  };
  Token cur = load_token(a, first, rank == 0 && tid == 0);
  Token next = load_token(a, first + groups, rank == 0 && tid == 0);
  if (kResident && tid == 0) {
    issue(cur, 0);
    if (slots == 2) issue(next, 1);
  }
  uint32_t phases = 0;
  double sums[3] = {0.0, 0.0, 0.0};
  int parity = 0, slot = 0;
  for (; cur.t < a.T;) {
    const Token after = load_token(a, cur.t + 2 * groups, rank == 0 && tid == 0);
    const T* row = logits + cur.t * a.ld_logits;
    const RowShape sh = row_shape(row, a.V);
    const int64_t n = span(sh);
    const uint4* src = kResident ? data + slot * cap
                                 : reinterpret_cast<const uint4*>(row + sh.head) + v0;
    // the entries outside whole vectors: threads 0-7 the head's, 8-15 the tail's, of rank 0
    int64_t edge = -1;
    if (rank == 0 && tid < 16) {
      if (tid < 8 && tid < sh.head) edge = tid;
      if (tid >= 8 && tid - 8 < sh.tail) edge = a.V - sh.tail + (tid - 8);
    }
    float ez = 0.f;
    RowGrad g{0.f, 0.f, 0.f, 0.f};
    if (cur.w != 0.f) {
      RowSum s{-CUDART_INF_F, 0.f, 0.f};
      if (edge >= 0) {
        ez = to_f32<T>(row[edge]);
        add_one(s, ez, scale);
      }
      TokenIn in{};
      if (warp == 0) in = load_inputs<T>(a, cur);
      if (kResident && n > 0) {
        mbar_wait(&full[slot], (phases >> slot) & 1u, abort_flag, a.status);
        phases ^= 1u << slot;
      }
      sum_span<T, kThreads>(s, src, n, tid, scale);
      s = join_warp(s, scale);
      if (lane == 0) part[warp] = s;
      __syncthreads();
      if (warp == 0) {
        s = lane < kWarps ? part[lane] : RowSum{-CUDART_INF_F, 0.f, 0.f};
        s = join_warp(s, scale);
        if (C > 1 && lane < C)
          st_cluster_v4(mapa_shared(smem_u32(&xchg[parity][rank]), lane), __float_as_uint(s.m),
                        __float_as_uint(s.l), __float_as_uint(s.e), 0u);
      }
      if (C > 1) cluster_sync();
      // (a peer that is a row ahead writes the other half of xchg, and none is two ahead)
      if (warp == 0) {
        if (C > 1) {
          const float4 x = lane < C ? xchg[parity][lane] : make_float4(-CUDART_INF_F, 0.f, 0.f, 0.f);
          s = join_warp(RowSum{x.x, x.y, x.z}, scale);
        }
        g = finish_token(a, cur, in, s, rank == 0 && lane == 0, sums);
        if (lane == 0) row_grad = g;
      }
      __syncthreads();
      g = row_grad;
      parity ^= 1;
    } else if (rank == 0 && tid == 0) {
      if (a.logp != nullptr) a.logp[cur.t] = 0.f;
      if (a.entropy != nullptr) a.entropy[cur.t] = 0.f;
    }
    if (grad != nullptr) {
      T* out = grad + cur.t * a.ld_grad;
      const int64_t start = sh.head + v0 * E;
      grad_span<T, kThreads>(src, out + start, n, tid, g, scale, cur.target - start);
      if (edge >= 0)
        out[edge] = g.f != 0.f ? grad_one<T>(ez, g, scale, edge == cur.target) : from_f32<T>(0.f);
    }
    __syncthreads();  // the slot, part and row_grad are free
    if (kResident && tid == 0) issue(slots == 2 ? after : next, slot);
    if (slots == 2) slot ^= 1;
    cur = next;
    next = after;
  }
  // a wait ran out: no copy may still be landing when the CTA leaves
  if (kResident && tid == 0 && *abort_flag)
    for (int s = 0; s < 2; ++s)
      if (issued[s] > 0)
        mbar_wait_slow(&full[s], (issued[s] - 1) & 1, nullptr, nullptr, kDrainLimitNs);
  if (rank == 0 && tid == 0) {
    if (groups == 1) {
      write_loss(a, sums);
    } else {
      double* p = a.partial + first * 4;
#pragma unroll
      for (int j = 0; j < 3; ++j) p[j] = sums[j];
    }
  }
}

// ---- a warp per row ------------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_warp_kernel(const PolicyArgs a) {
  __shared__ double part[kWarps][3];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float scale = a.inv_temp * kLog2e;
  double sums[3] = {0.0, 0.0, 0.0};
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWarps + warp; t < a.T;
       t += static_cast<int64_t>(gridDim.x) * kWarps) {
    const Token k = load_token(a, t, lane == 0);
    const T* row = static_cast<const T*>(a.logits) + t * a.ld_logits;
    const RowShape sh = row_shape(row, a.V);
    const uint4* src = reinterpret_cast<const uint4*>(row + sh.head);
    int64_t edge = -1;
    if (lane < 8 && lane < sh.head) edge = lane;
    if (lane >= 8 && lane - 8 < sh.tail) edge = a.V - sh.tail + (lane - 8);
    float ez = 0.f;
    RowGrad g{0.f, 0.f, 0.f, 0.f};
    if (k.w != 0.f) {
      RowSum s{-CUDART_INF_F, 0.f, 0.f};
      const TokenIn in = load_inputs<T>(a, k);
      if (edge >= 0) {
        ez = to_f32<T>(row[edge]);
        add_one(s, ez, scale);
      }
      sum_span<T, 32>(s, src, sh.nvec, lane, scale);
      s = join_warp(s, scale);
      g = finish_token(a, k, in, s, lane == 0, sums);
    } else if (lane == 0) {
      if (a.logp != nullptr) a.logp[t] = 0.f;
      if (a.entropy != nullptr) a.entropy[t] = 0.f;
    }
    if (a.grad != nullptr) {
      __syncwarp();  // (in place: the target's logit has been read)
      T* out = static_cast<T*>(a.grad) + t * a.ld_grad;
      grad_span<T, 32>(src, out + sh.head, sh.nvec, lane, g, scale, k.target - sh.head);
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
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < n; i += 256)
    for (int j = 0; j < 3; ++j) s[j] += a.partial[i * 4 + j];
  for (int j = 0; j < 3; ++j) sh[j][threadIdx.x] = s[j];
  for (int o = 128; o > 0; o >>= 1) {
    __syncthreads();
    if (threadIdx.x < o)
      for (int j = 0; j < 3; ++j) sh[j][threadIdx.x] += sh[j][threadIdx.x + o];
  }
  if (threadIdx.x == 0) {
    const double all[3] = {sh[0][0], sh[1][0], sh[2][0]};
    write_loss(a, all);
  }
}

// ---- host ----------------------------------------------------------------------------------------
constexpr int64_t kSmemSm = 227 * 1024;  // shared memory of an SM that CTAs may take
constexpr int64_t kSmemStatic = 2048;    // at most what a CTA takes beside its slots, with the reserve

template <typename T>
cudaError_t set_smem() {
  // the kernel's limit, the same for every call
  return cudaFuncSetAttribute(policy_cluster_kernel<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(kSmemSm - kSmemStatic));
}

// Clusters of the resident kernel that run at once (0 on error), cached per device and launch shape.
template <typename T>
int active_clusters(int C, size_t smem) {
  struct Entry {
    int dev, C, clusters;
    size_t smem;
  };
  static std::mutex mu;
  static Entry cache[32];
  static int used = 0;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  std::lock_guard<std::mutex> lock(mu);
  for (int i = 0; i < used; ++i)
    if (cache[i].dev == dev && cache[i].C == C && cache[i].smem == smem) return cache[i].clusters;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (set_smem<T>() != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, policy_cluster_kernel<T, true>, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    n = 0;
  }
  cache[used < 32 ? used++ : 31] = Entry{dev, C, n, smem};
  return n;
}

template <typename T>
cudaError_t launch(const PolicyArgs& a, int num_sms, cudaStream_t st) {
  constexpr int E = Vec<T>::kElems;
  const int64_t nvec = a.V / E;  // most whole vectors of a row
  int64_t parts;
  cudaError_t err;
  if (nvec <= 256) {  // at most 8 vectors a lane
    int64_t blocks = (a.T + kWarps - 1) / kWarps;
    const int64_t cap = static_cast<int64_t>(num_sms) * 8;
    if (blocks > cap) blocks = cap;
    parts = blocks;
    err = launch_pdl(policy_warp_kernel<T>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, 1, a);
  } else {
    // Slices of which three CTAs an SM hold two each, in as narrow a cluster as gives them; a wider
    // one while that puts idle SMs to work and leaves every thread a vector.
    int C = 1;
    while (C < kMaxCluster && (nvec + C - 1) / C * 16 * 6 > kSmemSm - 3 * kSmemStatic) C *= 2;
    while (C < kMaxCluster && a.T * C * 2 <= num_sms && nvec >= C * 2 * kThreads) C *= 2;
    const int64_t cap = (nvec + C - 1) / C;
    const int64_t bytes = cap * 16;
    const bool resident = bytes <= kSmemSm - kSmemStatic;
    const int slots = 3 * (2 * bytes + kSmemStatic) <= kSmemSm ? 2 : 1;
    const size_t smem = resident ? static_cast<size_t>(bytes * slots) : 0;
    int64_t groups = resident ? active_clusters<T>(C, smem) : static_cast<int64_t>(num_sms) * 4 / C;
    if (groups <= 0) return cudaErrorInvalidConfiguration;
    if (groups > a.T) groups = a.T;
    if (groups > kPolicyParts) groups = kPolicyParts;
    parts = groups;
    const dim3 grid(static_cast<unsigned>(groups * C)), block(kThreads);
    err = resident ? launch_pdl(policy_cluster_kernel<T, true>, grid, block, smem, st, C, a, C, cap, slots)
                   : launch_pdl(policy_cluster_kernel<T, false>, grid, block, 0, st, C, a, C, cap, 1);
  }
  if (err != cudaSuccess || parts == 1) return err;  // one cluster (block) writes the loss itself
  return launch_pdl(policy_finish_kernel, dim3(1), dim3(256), 0, st, 1, a, static_cast<int>(parts));
}

}  // namespace

cudaError_t launch_policy_loss(const PolicyArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? launch<__nv_bfloat16>(a, num_sms, st) : launch<float>(a, num_sms, st);
}

}  // namespace pr2
