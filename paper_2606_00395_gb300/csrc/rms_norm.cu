// Residual addition and root-mean-square norm of rows, with the normed rows in the layer dtype, in 8
// bits with a scale for each row, or both; rows in 8 bits alone; and the norm's backward pass.
//
//   s = x + residual,  rstd = 1 / sqrt(sum s^2 / d + eps),  p = s w,  y = p rstd,
//   q = e4m3(p 448 / top),  scale = top / 448 rstd,  top = max |p|.
// Backward, with g = w dy and xhat = s rstd:
//   ds = dsum + rstd (g - xhat (sum g xhat) / d),  dweight = sum over rows of dy xhat.
//
// Bound by HBM: a row is read once and stays in registers between its sum and its results, so the two
// sums of a row (forward: of squares, and the maximum) cost one exchange between its threads.  A row
// is a warp's, several warps' or a whole block's, by its width: 32 elements of it a thread.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr float kTop8 = 448.f;                                  // largest e4m3 value
constexpr float kInvTop8 = static_cast<float>(1.0 / 448.0);
constexpr float kTinyTop8 = 1e-30f;                             // rows below are held as zeros

// 8 V elements of a row per thread.  kVec: vector v of thread t holds elements 8 (v G + t) .., else
// element j of it is 8 v G + j G + t.
template <int G, bool kVec>
__device__ __forceinline__ int column(int t, int v, int j) {
  return kVec ? (v * G + t) * 8 + j : (v * 8 + j) * G + t;
}

// Elements as loaded.
template <typename T, int V, bool kVec>
struct Held;
template <int V>
struct Held<__nv_bfloat16, V, true> {
  uint4 v[V];
};
template <int V>
struct Held<float, V, true> {
  float4 v[2 * V];
};
template <typename T, int V>
struct Held<T, V, false> {
  T e[8 * V];
};

// The vectors from v0 on that h holds.
template <typename T, int G, int V, bool kVec>
__device__ __forceinline__ void load_row(Held<T, V, kVec>& h, const T* row, int t, int d, int v0 = 0) {
  if constexpr (kVec) {  // (d is a multiple of 8)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = column<G, true>(t, v0 + v, 0);
      if constexpr (sizeof(T) == 2) {
        h.v[v] = c < d ? __ldcs(reinterpret_cast<const uint4*>(row + c)) : make_uint4(0u, 0u, 0u, 0u);
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          h.v[2 * v + i] = c < d ? __ldcs(reinterpret_cast<const float4*>(row + c) + i)
                                 : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) {
      const int c = column<G, false>(t, v0 + (i >> 3), i & 7);
      h.e[i] = c < d ? row[c] : from_f32<T>(0.f);
    }
  }
}

template <typename T, int V, bool kVec>
__device__ __forceinline__ void unpack(const Held<T, V, kVec>& h, float (&f)[8 * V]) {
  if constexpr (!kVec) {
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) f[i] = to_f32<T>(h.e[i]);
  } else if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t w[4] = {h.v[v].x, h.v[v].y, h.v[v].z, h.v[v].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[8 * v + 2 * i] = __uint_as_float(w[i] << 16);
        f[8 * v + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < 2 * V; ++v) {
      f[4 * v] = h.v[v].x;
      f[4 * v + 1] = h.v[v].y;
      f[4 * v + 2] = h.v[v].z;
      f[4 * v + 3] = h.v[v].w;
    }
  }
}

// Vector v of a thread's elements.
template <typename T, int G, bool kVec>
__device__ __forceinline__ void store8(T* row, const float* g, int t, int v, int d) {
  if constexpr (kVec) {
    const int c = column<G, true>(t, v, 0);
    if (c >= d) return;
    if constexpr (sizeof(T) == 2) {
      __stcs(reinterpret_cast<uint4*>(row + c), make_uint4(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]),
                                                           pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7])));
    } else {
      __stcs(reinterpret_cast<float4*>(row + c), make_float4(g[0], g[1], g[2], g[3]));
      __stcs(reinterpret_cast<float4*>(row + c) + 1, make_float4(g[4], g[5], g[6], g[7]));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = column<G, false>(t, v, j);
      if (c < d) row[c] = from_f32<T>(g[j]);
    }
  }
}
template <typename T, int G, int V, bool kVec>
__device__ __forceinline__ void store_row(T* row, const float (&f)[8 * V], int t, int d) {
#pragma unroll
  for (int v = 0; v < V; ++v) store8<T, G, kVec>(row, f + 8 * v, t, v, d);
}

// The weight, small and read by every row: through L1.
template <typename T, int G, int V, bool kVec>
__device__ __forceinline__ void load_weight(Held<T, V, kVec>& h, const T* w, int t, int d, int v0 = 0) {
  if constexpr (kVec) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = column<G, true>(t, v0 + v, 0);
      if constexpr (sizeof(T) == 2) {
        h.v[v] = c < d ? __ldg(reinterpret_cast<const uint4*>(w + c)) : make_uint4(0u, 0u, 0u, 0u);
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          h.v[2 * v + i] = c < d ? __ldg(reinterpret_cast<const float4*>(w + c) + i)
                                 : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
  } else {
    load_row<T, G, V, false>(h, w, t, d, v0);
  }
}

// Two floats in e4m3, to nearest, ties to even: the first in the low byte.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int G, int V, bool kVec>
__device__ __forceinline__ void store_row8(uint8_t* row, const float (&f)[8 * V], float r, int t, int d) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      b[i] = pack_e4m3x2(__fmul_rn(f[8 * v + 2 * i], r), __fmul_rn(f[8 * v + 2 * i + 1], r));
    if constexpr (kVec) {
      const int c = column<G, true>(t, v, 0);
      if (c < d) __stcs(reinterpret_cast<uint2*>(row + c), make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = column<G, false>(t, v, j);
        if (c < d) row[c] = static_cast<uint8_t>(b[j >> 1] >> (8 * (j & 1)));
      }
    }
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename T, int G, int V, bool kVec>
__global__ void __launch_bounds__(G < 256 ? 256 : G) norm_kernel(NormArgs a) {
  constexpr int kThreads = G < 256 ? 256 : G;
  constexpr int kWarps = G / 32;  // of a row
  __shared__ float red_sum[kThreads / 32];
  __shared__ uint32_t red_top[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x % G;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / G) + threadIdx.x / G;
  if (row >= a.rows) return;
  const int d = a.d;
  float f[8 * V];
  {
    Held<T, V, kVec> x, res;
    load_row<T, G, V, kVec>(x, static_cast<const T*>(a.x) + row * a.ld, t, d);
    if (a.end != nullptr && row >= *a.end) return;  // (read beside the row, not before it)
    if (a.residual != nullptr) {
      load_row<T, G, V, kVec>(res, static_cast<const T*>(a.residual) + row * a.ld, t, d);
      float g[8 * V];
      unpack<T, V, kVec>(x, f);
      unpack<T, V, kVec>(res, g);
#pragma unroll
      for (int i = 0; i < 8 * V; ++i) f[i] = to_f32<T>(from_f32<T>(f[i] + g[i]));
    } else {
      unpack<T, V, kVec>(x, f);
    }
  }
  if (a.sum != nullptr) store_row<T, G, V, kVec>(static_cast<T*>(a.sum) + row * a.ld, f, t, d);
  float ss = 0.f;
  if (a.weight != nullptr) {
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) ss = fmaf(f[i], f[i], ss);
    Held<T, V, kVec> hw;
    load_weight<T, G, V, kVec>(hw, static_cast<const T*>(a.weight), t, d);
    float w[8 * V];
    unpack<T, V, kVec>(hw, w);
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) f[i] = __fmul_rn(f[i], w[i]);
  }
  // largest magnitude as a bit pattern: ordered as the values are, NaN above all of them
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8 * V; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
  ss = warp_sum(ss);
  top = __reduce_max_sync(0xffffffffu, top);
  if constexpr (G > 32) {
    const int lane = threadIdx.x & 31, group = threadIdx.x / G;
    if (lane == 0) {
      red_sum[threadIdx.x >> 5] = ss;
      red_top[threadIdx.x >> 5] = top;
    }
    named_bar_sync(1 + group, G);
    ss = warp_sum(lane < kWarps ? red_sum[group * kWarps + lane] : 0.f);
    top = __reduce_max_sync(0xffffffffu, lane < kWarps ? red_top[group * kWarps + lane] : 0u);
  }
  float rstd = 1.f;
  if (a.weight != nullptr) rstd = __frsqrt_rn(ss * a.inv_d + a.eps);
  if (a.q != nullptr) {
    const float m = __uint_as_float(top);
    const bool finite = top < 0x7f800000u;
    const bool some = finite && m >= kTinyTop8;
    const float r = some ? __fdiv_rn(kTop8, m) : 0.f;
    if (t == 0)
      a.scale[row] = !finite ? __uint_as_float(0x7fc00000u)
                             : some ? __fmul_rn(__fmul_rn(m, kInvTop8), rstd) : 0.f;
    store_row8<G, V, kVec>(a.q + row * d, f, r, t, d);
  }
  if (a.y != nullptr) {
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) f[i] = __fmul_rn(f[i], rstd);
    store_row<T, G, V, kVec>(static_cast<T*>(a.y) + row * d, f, t, d);
  }
}

// Pairs of fp32 for the packed FMAs, which do the backward pass's arithmetic in half the instructions.
struct Pair {
  uint64_t v;
};
__device__ __forceinline__ Pair make_pair(float lo, float hi) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p.v));
}
__device__ __forceinline__ Pair mul(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// Elements 2 i and 2 i + 1 of a thread's.
template <typename T, int V, bool kVec>
__device__ __forceinline__ Pair pair_of(const Held<T, V, kVec>& h, int i) {
  if constexpr (!kVec) {
    return make_pair(to_f32<T>(h.e[2 * i]), to_f32<T>(h.e[2 * i + 1]));
  } else if constexpr (sizeof(T) == 2) {
    const uint4& q = h.v[i >> 2];
    const uint32_t w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
    return make_pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  } else {
    const float4& q = h.v[i >> 1];
    return (i & 1) ? make_pair(q.z, q.w) : make_pair(q.x, q.y);
  }
}

// Rows on their way (bf16 rows that start on 16 bytes): each thread copies its own 8 elements of s, dy and dsum
// into slots of its own, so that nothing but its own wait stands between the copy and the use.  fp32 rows are
// twice the bytes, of which two blocks an SM have enough in flight without it (16384 x 2048: 96 us, with
// copies two rows ahead 152).
template <typename T, int V, bool kVec, int kThreads>
struct Ahead {
  static constexpr bool kUsed = V == 1 && kVec && sizeof(T) == 2;
  static constexpr int kDepth = 4;
  static constexpr int kBytes = kUsed ? kDepth * 3 * kThreads * 16 : 0;
  __device__ __forceinline__ static uint32_t at(const uint8_t* base, int slot, int which) {
    return smem_u32(base) + ((slot * 3 + which) * kThreads + threadIdx.x) * 16;
  }
  __device__ __forceinline__ static void copy(const uint8_t* base, int slot, int which, const T* row, int t, int d) {
    const bool in = t * 8 < d;
    cp_async_16(at(base, slot, which), in ? row + t * 8 : row, in ? 16u : 0u);
  }
  __device__ __forceinline__ static void read(const uint8_t* base, int slot, int which, Held<T, V, kVec>& h) {
    if constexpr (kUsed) {
      uint32_t w[4];
      ld_shared_v4(at(base, slot, which), w);
      h.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

// A group of G threads walks rows.  The row stays packed as loaded between its sums and its gradient, so
// that two blocks of 512 threads fit an SM; rows above 8192 are read twice, the second time from L2.  Each
// thread keeps the weight's gradient of its columns, which the block's groups join at the end and weight_kernel
// over the blocks.
//   ds = dsum + c1 (w dy) + c2 s,  c1 = rstd,  c2 = -rstd^3 (sum w dy s) / d,   dweight += (dy s) rstd
template <int G>
constexpr int kBackThreads = G < 512 ? 512 : G;

template <typename T, int G, int V, bool kVec>
__global__ void __launch_bounds__(kBackThreads<G>, kBackThreads<G> == 512 ? 2 : 1) norm_backward_kernel(NormArgs a) {
  constexpr int kThreads = kBackThreads<G>;
  constexpr int kGroups = kThreads / G;
  constexpr int kWarps = G / 32;  // of a group
  constexpr bool kTwice = V > 1;
  __shared__ __align__(8) float red[2][kThreads / 32][2];  // a warp's sums, read as pairs
  __shared__ float join[kGroups > 1 ? kGroups : 1][kGroups > 1 ? G * 8 * V : 1];
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x % G, group = threadIdx.x / G, lane = threadIdx.x & 31;
  const int d = a.d;
  const T* s = static_cast<const T*>(a.x);
  const T* dy = static_cast<const T*>(a.dy);
  const T* dsum = static_cast<const T*>(a.residual);
  T* ds = static_cast<T*>(a.sum);
  const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
  const T* weight = static_cast<const T*>(a.weight);
  Held<T, 1, kVec> hw;
  if constexpr (!kTwice) load_weight<T, G, 1, kVec>(hw, weight, t, d);
  Pair acc[4 * V];
#pragma unroll
  for (int i = 0; i < 4 * V; ++i) acc[i] = make_pair(0.f, 0.f);
  extern __shared__ __align__(16) uint8_t ahead[];
  using Slot = Ahead<T, V, kVec, kThreads>;  // the next rows of this thread's columns
  auto fetch = [&](int64_t r, int slot) {
    if (r < a.rows) {
      Slot::copy(ahead, slot, 0, s + r * a.ld, t, d);
      Slot::copy(ahead, slot, 1, dy + r * d, t, d);
      if (dsum != nullptr) Slot::copy(ahead, slot, 2, dsum + r * a.ld, t, d);
    }
    cp_async_commit();
  };
  int odd = 0, slot = 0;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kGroups + group;
  if constexpr (Slot::kUsed) {
#pragma unroll
    for (int i = 0; i < Slot::kDepth - 1; ++i) fetch(row0 + i * step, i);
  }
  for (int64_t row = row0; row < a.rows; row += step, odd ^= 1) {
    Held<T, 1, kVec> hs, hd, hr;
    auto load = [&](int v, bool all) {
      load_row<T, G, 1, kVec>(hs, s + row * a.ld, t, d, v);
      load_row<T, G, 1, kVec>(hd, dy + row * d, t, d, v);
      if (all && dsum != nullptr) load_row<T, G, 1, kVec>(hr, dsum + row * a.ld, t, d, v);
    };
    if constexpr (Slot::kUsed) {
      fetch(row + (Slot::kDepth - 1) * step, slot == 0 ? Slot::kDepth - 1 : slot - 1);
      cp_async_wait<Slot::kDepth - 1>();
      Slot::read(ahead, slot, 0, hs);
      Slot::read(ahead, slot, 1, hd);
      if (dsum != nullptr) Slot::read(ahead, slot, 2, hr);
      if (++slot == Slot::kDepth) slot = 0;
    } else if constexpr (!kTwice) {
      load(0, true);
    }
    Pair ss2 = make_pair(0.f, 0.f), gs2 = ss2;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (kTwice) {
        load(v, false);
        load_weight<T, G, 1, kVec>(hw, weight, t, d, v);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Pair x = pair_of<T, 1, kVec>(hs, i), g = pair_of<T, 1, kVec>(hd, i);
        ss2 = fma(x, x, ss2);
        gs2 = fma(pair_of<T, 1, kVec>(hw, i), mul(g, x), gs2);
      }
    }
    float s0, s1, g0, g1;
    split(ss2, s0, s1);
    split(gs2, g0, g1);
    // both sums of the warp in one tree: the lower half-warp goes on with one, the upper with the other
    const float ss = s0 + s1, gs = g0 + g1;
    const bool upper = lane & 16;
    float v = (upper ? gs : ss) + __shfl_xor_sync(0xffffffffu, upper ? ss : gs, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    float sum_s, sum_g;
    if constexpr (kWarps > 1) {
      if ((lane & 15) == 0) red[odd][threadIdx.x >> 5][lane >> 4] = v;
      named_bar_sync(1 + group, G);  // (the other buffer's readers are behind it too)
      sum_s = sum_g = 0.f;
      if constexpr (kWarps <= 8) {
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          const float2 r = *reinterpret_cast<const float2*>(red[odd][group * kWarps + i]);
          sum_s += r.x;
          sum_g += r.y;
        }
      } else {
        const float2 r = lane < kWarps ? *reinterpret_cast<const float2*>(red[odd][group * kWarps + lane])
                                       : make_float2(0.f, 0.f);
        sum_s = warp_sum(r.x);
        sum_g = warp_sum(r.y);
      }
    } else {
      sum_s = __shfl_sync(0xffffffffu, v, 0);
      sum_g = __shfl_sync(0xffffffffu, v, 16);
    }
    const float rstd = __frsqrt_rn(sum_s * a.inv_d + a.eps);
    const float c = -(sum_g * a.inv_d) * rstd * rstd * rstd;
    const Pair c1 = make_pair(rstd, rstd), c2 = make_pair(c, c);
    T* to = ds + row * a.ld;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if constexpr (kTwice) {
        load(i, true);
        load_weight<T, G, 1, kVec>(hw, weight, t, d, i);
      }
      float out[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const Pair x = pair_of<T, 1, kVec>(hs, k), g = pair_of<T, 1, kVec>(hd, k);
        const Pair add = dsum != nullptr ? pair_of<T, 1, kVec>(hr, k) : make_pair(0.f, 0.f);
        acc[4 * i + k] = fma(mul(g, x), c1, acc[4 * i + k]);
        split(fma(mul(pair_of<T, 1, kVec>(hw, k), g), c1, fma(x, c2, add)), out[2 * k], out[2 * k + 1]);
      }
      store8<T, G, kVec>(to, out, t, i, d);
    }
  }
  float* part = a.partial + static_cast<int64_t>(blockIdx.x) * d;
  if constexpr (kGroups > 1) {
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) {
      float lo, hi;
      split(acc[i], lo, hi);
      join[group][column<G, kVec>(t, i >> 2, (2 * i) & 7)] = lo;
      join[group][column<G, kVec>(t, i >> 2, (2 * i + 1) & 7)] = hi;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < d; c += kThreads) {
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < kGroups; ++j) v += join[j][c];
      part[c] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4 * V; ++i) {
      float v[2];
      split(acc[i], v[0], v[1]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = column<G, kVec>(t, i >> 2, (2 * i + k) & 7);
        if (c < d) part[c] = v[k];
      }
    }
  }
}

// dweight[c] = sum of the blocks' parts, in order within 32 interleaved sums.
__global__ void __launch_bounds__(1024) weight_kernel(const float* partial, int parts, int d, float* dweight) {
  __shared__ float join[32][33];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, j = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (c < d) {
#pragma unroll 10
    for (int i = j; i < parts; i += 32) v += partial[static_cast<int64_t>(i) * d + c];
  }
  join[j][lane] = v;
  __syncthreads();
  v = warp_sum(join[lane][j]);  // column j of the block's 32
  const int mine = blockIdx.x * 32 + j;
  if (lane == 0 && mine < d) dweight[mine] = v;
}

bool at16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename T, int G, int V>
cudaError_t launch_norm_rows(const NormArgs& a, bool vec, cudaStream_t st) {
  constexpr int kThreads = G < 256 ? 256 : G;
  const int64_t blocks = (a.rows + kThreads / G - 1) / (kThreads / G);
  return launch_pdl(vec ? norm_kernel<T, G, V, true> : norm_kernel<T, G, V, false>,
                    dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, 1, a);
}

template <typename T>
cudaError_t launch_norm_t(const NormArgs& a, cudaStream_t st) {
  const bool vec = a.d % 8 == 0 && a.ld * sizeof(T) % 16 == 0 && at16(a.x) && at16(a.residual) &&
                   at16(a.sum) && at16(a.weight) && at16(a.y) && reinterpret_cast<uintptr_t>(a.q) % 8 == 0;
  if (a.d <= 256) return launch_norm_rows<T, 32, 1>(a, vec, st);
  if (a.d <= 512) return launch_norm_rows<T, 32, 2>(a, vec, st);
  if (a.d <= 1024) return launch_norm_rows<T, 32, 4>(a, vec, st);
  if (a.d <= 2048) return launch_norm_rows<T, 64, 4>(a, vec, st);
  if (a.d <= 4096) return launch_norm_rows<T, 128, 4>(a, vec, st);
  if (a.d <= 8192) return launch_norm_rows<T, 256, 4>(a, vec, st);
  return launch_norm_rows<T, 1024, 4>(a, vec, st);
}

template <typename T, int G, int V>
cudaError_t launch_backward_rows(const NormArgs& a, bool vec, int num_sms, cudaStream_t st) {
  constexpr int kThreads = kBackThreads<G>;
  const int64_t blocks = (a.rows + kThreads / G - 1) / (kThreads / G);
  const int most = 2 * num_sms < kNormParts ? 2 * num_sms : kNormParts;
  const int grid = static_cast<int>(blocks < most ? blocks : most);
  auto* kernel = vec ? norm_backward_kernel<T, G, V, true> : norm_backward_kernel<T, G, V, false>;
  const int smem = vec ? Ahead<T, V, true, kThreads>::kBytes : Ahead<T, V, false, kThreads>::kBytes;
  cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  err = launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, st, 1, a);
  if (err != cudaSuccess) return err;
  return launch_pdl(weight_kernel, dim3((a.d + 31) / 32), dim3(1024), 0, st, 1,
                    static_cast<const float*>(a.partial), grid, a.d, a.dweight);
}

template <typename T>
cudaError_t launch_backward_t(const NormArgs& a, bool vec, int num_sms, cudaStream_t st) {
  if (a.d <= 256) return launch_backward_rows<T, 32, 1>(a, vec, num_sms, st);
  if (a.d <= 1024) return launch_backward_rows<T, 128, 1>(a, vec, num_sms, st);
  if (a.d <= 2048) return launch_backward_rows<T, 256, 1>(a, vec, num_sms, st);
  if (a.d <= 4096) return launch_backward_rows<T, 512, 1>(a, vec, num_sms, st);
  if (a.d <= 8192) return launch_backward_rows<T, 1024, 1>(a, vec, num_sms, st);
  return launch_backward_rows<T, 1024, 4>(a, vec, num_sms, st);
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  return a.bf16 ? launch_norm_t<__nv_bfloat16>(a, st) : launch_norm_t<float>(a, st);
}

cudaError_t launch_norm_backward(const NormArgs& a, int num_sms, cudaStream_t st) {
  const size_t es = a.bf16 ? 2 : 4;
  const bool vec = a.d % 8 == 0 && a.ld * es % 16 == 0 && at16(a.x) && at16(a.residual) && at16(a.sum) &&
                   at16(a.weight) && at16(a.dy);
  return a.bf16 ? launch_backward_t<__nv_bfloat16>(a, vec, num_sms, st) : launch_backward_t<float>(a, vec, num_sms, st);
}

}  // namespace pr2
