// SwiGLU activation with an 8-bit checkpoint of its inputs, and its backward pass.
//
// act = silu(gate) up; a run of 128 elements of a row of gate or up is held as q = round(x 127 / top),
// scale = top / 127, top = max |x|.  Backward, from g = q scale: s = 1 / (1 + exp(-g)),
//   dgate = dact u s (1 + g (1 - s)),  dup = dact g s,  act = g s u.
// Bound by HBM: bf16 reads 4 bytes and writes 4 per element forward, reads 4 and writes 6 backward.
// Lanes take 8 neighbouring elements (two 16-byte vectors of fp32, one of bf16; 8 bytes of q), so 16
// lanes hold a run and a warp two; where a row's start or width does not allow that, single elements.
// 32768 x 768 bf16: forward 38 us (79 % of the copy rate; it issues about 30 instructions an element, 79 %
// of all slots), backward 41 us (91 %); 65536 x 2048 88 % and 95 %; 767 columns 64 and 68 us.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kGroup = PR2_CKPT_GROUP;
constexpr int kLane = 8;                    // elements of a lane
constexpr int kRunLanes = kGroup / kLane;   // 16
constexpr float kInv127 = static_cast<float>(1.0 / 127.0);
constexpr float kTinyTop = 1e-30f;

// From the exponential that cannot overflow: with exp(-x) the sigmoid of x < -88 would be 0 where
// x sigmoid(x) is still a normal number.  __expf rounds its argument, which is 4e-6 of the result at x = -85:
// enough before a rounding to bf16, while fp32 takes the full function (act then 2.7e-7 off at most).  fp32,
// forward and backward, us with __expf / expf: 32768 x 768 58, 83 / 57, 82; 32768 x 767 68, 95 / 70, 94.
template <typename T>
__device__ __forceinline__ float sigmoid(float x) {
  const float e = sizeof(T) == 4 ? expf(-fabsf(x)) : __expf(-fabsf(x));
  return __fdividef(x >= 0.f ? 1.f : e, 1.f + e);
}

// Scale of a run and the factor that takes its values to integers, from the largest bit pattern
// of |x| (ordered as the values are; infinities and NaN above every finite one).
__device__ __forceinline__ void run_scale(uint32_t top_bits, float* scale, float* factor) {
  const float top = __uint_as_float(top_bits);
  const bool finite = top_bits < 0x7f800000u;
  const bool some = finite && top >= kTinyTop;
  *scale = !finite ? __uint_as_float(0x7fc00000u) : some ? __fmul_rn(top, kInv127) : 0.f;
  *factor = some ? __fdiv_rn(127.f, top) : 0.f;
}

// round(x factor) to the nearest integer, ties to even, in two's complement in the low byte: the
// product is at most 127 (1 + 2^-23) and adding 1.5 2^23 rounds it to the last place of the sum.
__device__ __forceinline__ uint32_t quantize(float x, float factor) {
  return __float_as_uint(__fadd_rn(__fmul_rn(x, factor), 12582912.f));
}
__device__ __forceinline__ uint32_t quantize4(const float* x, float factor) {
  const uint32_t lo = __byte_perm(quantize(x[0], factor), quantize(x[1], factor), 0x0040);
  const uint32_t hi = __byte_perm(quantize(x[2], factor), quantize(x[3], factor), 0x0040);
  return __byte_perm(lo, hi, 0x5410);
}
// The larger of two magnitudes' bit patterns; of two bf16 pairs' at once.
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Byte i of w as a signed number: 2^23 + 128 + q as a bit pattern, less that.
template <int i>
__device__ __forceinline__ float byte_value(uint32_t flipped) {  // w ^ 0x80808080
  return __uint_as_float(__byte_perm(flipped, 0x4b000000u, 0x7440 | i)) - 8388736.f;
}

// 8 elements as loaded, and as fp32.
template <typename T>
struct Raw8 {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) v[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) v[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[4 * i] = __uint_as_float(v[i].x);
        f[4 * i + 1] = __uint_as_float(v[i].y);
        f[4 * i + 2] = __uint_as_float(v[i].z);
        f[4 * i + 3] = __uint_as_float(v[i].w);
      }
    }
  }
};
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]);
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]),
                                            pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
template <>
__device__ __forceinline__ void store8<float>(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Largest magnitudes of a run's gate and up, as fp32 bit patterns, over its 16 lanes.
template <typename T>
__device__ __forceinline__ void run_tops(const Raw8<T> (&raw)[2], uint32_t (&top)[2]) {
  if constexpr (sizeof(T) == 2) {  // in pairs of bf16; a NaN stays one
    uint32_t m[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4& v = raw[h].v[0];
      m[h] = max_bf16x2(max_bf16x2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu),
                        max_bf16x2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    }
    uint32_t both = max_bf16x2(__byte_perm(m[0], m[1], 0x5410), __byte_perm(m[0], m[1], 0x7632));
#pragma unroll
    for (int o = kRunLanes / 2; o > 0; o >>= 1) both = max_bf16x2(both, __shfl_xor_sync(0xffffffffu, both, o));
    top[0] = both << 16;
    top[1] = both & 0xffff0000u;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4& v = raw[h].v[i];
        m = max(max(max(m, v.x & 0x7fffffffu), v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu));
      }
#pragma unroll
      for (int o = kRunLanes / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      top[h] = m;
    }
  }
}

// m % 8 == 0 and every row starts on 16 bytes (q: 8).  A half warp per run; a run's last lanes may lie
// past m.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    checkpoint_kernel(const T* __restrict__ gate, const T* __restrict__ up, int64_t rows, int64_t ld,
                      int m, int G, T* __restrict__ act, int8_t* __restrict__ q, float* __restrict__ scale) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, sub = lane % kRunLanes;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (kThreads / kRunLanes);
  const int64_t mine = static_cast<int64_t>(blockIdx.x) * (kThreads / kRunLanes) + threadIdx.x / kRunLanes;
  // The next run is loaded before the present one is worked on.
  RowWalk at(mine, step, G);
  Raw8<T> raw[2];
  auto load = [&](const RowWalk& w) {
    const int c = w.col * kGroup + sub * kLane;
    if (w.row < rows && c < m) {
      raw[0].load(gate + w.row * ld + c);
      raw[1].load(up + w.row * ld + c);
    } else {
      raw[0].zero();
      raw[1].zero();
    }
  };
  load(at);
  while (__any_sync(0xffffffffu, at.row < rows)) {  // (both halves of a warp go round together)
    const int64_t r = at.row;
    const int grp = at.col, c = grp * kGroup + sub * kLane;
    const bool own = r < rows && c < m;
    float x[2][8];
    uint32_t top[2];
    run_tops<T>(raw, top);
    raw[0].unpack(x[0]);
    raw[1].unpack(x[1]);
    at.next();
    load(at);
    // even lanes work out gate's scale, odd lanes up's
    float sc, f;
    run_scale(top[sub & 1], &sc, &f);
    const float factor[2] = {__shfl_sync(0xffffffffu, f, lane & ~1), __shfl_sync(0xffffffffu, f, lane | 1)};
    if (sub < 2 && r < rows) scale[(r * 2 + sub) * G + grp] = sc;  // (up's lane may lie past m)
    if (!own) continue;
    const int64_t rm = r * m;
    float a[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = x[0][j] * sigmoid<T>(x[0][j]) * x[1][j];
    store8(act + rm + c, a);
    int8_t* qr = q + 2 * rm + c;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint2 w = make_uint2(quantize4(x[h], factor[h]), quantize4(x[h] + 4, factor[h]));
      *reinterpret_cast<uint2*>(qr + (h == 0 ? 0 : m)) = factor[h] > 0.f ? w : make_uint2(0u, 0u);
    }
  }
}

struct Grads {
  float dgate, dup, act;
};
template <typename T>
__device__ __forceinline__ Grads swiglu_grads(float g, float u, float d) {
  const float s = sigmoid<T>(g), gs = g * s;
  return Grads{d * u * s * (1.f + g * (1.f - s)), d * gs, gs * u};
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    backward_kernel(const T* dact, const int8_t* __restrict__ q, const float* __restrict__ scale,
                    int64_t rows, int64_t ld, int m, int G, T* __restrict__ dgate, T* __restrict__ dup, T* act) {
  pdl_wait();
  pdl_trigger();
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x, static_cast<int64_t>(gridDim.x) * kThreads,
             m / kLane);
  for (; at.row < rows; at.next()) {
    const int64_t r = at.row;
    const int c = at.col * kLane;
    const uint2 qg = __ldcs(reinterpret_cast<const uint2*>(q + r * 2 * m + c));
    const uint2 qu = __ldcs(reinterpret_cast<const uint2*>(q + (r * 2 + 1) * m + c));
    const float sg = scale[r * 2 * G + c / kGroup], su = scale[(r * 2 + 1) * G + c / kGroup];
    float d[8], dg[8], du[8], a[8];
    Raw8<T> rd;
    rd.load(dact + r * m + c);
    rd.unpack(d);
    const uint32_t wg[2] = {qg.x ^ 0x80808080u, qg.y ^ 0x80808080u};
    const uint32_t wu[2] = {qu.x ^ 0x80808080u, qu.y ^ 0x80808080u};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float g[4] = {byte_value<0>(wg[h]), byte_value<1>(wg[h]), byte_value<2>(wg[h]), byte_value<3>(wg[h])};
      const float u[4] = {byte_value<0>(wu[h]), byte_value<1>(wu[h]), byte_value<2>(wu[h]), byte_value<3>(wu[h])};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Grads o = swiglu_grads<T>(__fmul_rn(g[j], sg), __fmul_rn(u[j], su), d[4 * h + j]);
        dg[4 * h + j] = o.dgate;
        du[4 * h + j] = o.dup;
        a[4 * h + j] = o.act;
      }
    }
    store8(dgate + r * ld + c, dg);
    store8(dup + r * ld + c, du);
    if (act != nullptr) store8(act + r * m + c, a);
  }
}

// Any width and alignment: a warp per run.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    checkpoint_any_kernel(const T* __restrict__ gate, const T* __restrict__ up, int64_t rows,
                          int64_t ld, int m, int G, T* __restrict__ act, int8_t* __restrict__ q,
                          float* __restrict__ scale) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x) * kWarps,
             G);
  for (; at.row < rows; at.next()) {
    const int64_t r = at.row;
    const int grp = at.col;
    float x[2][4];
    uint32_t top[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = grp * kGroup + j * 32 + lane;
      x[0][j] = c < m ? to_f32<T>(gate[r * ld + c]) : 0.f;
      x[1][j] = c < m ? to_f32<T>(up[r * ld + c]) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = grp * kGroup + j * 32 + lane;
#pragma unroll
      for (int h = 0; h < 2; ++h) top[h] = max(top[h], __float_as_uint(x[h][j]) & 0x7fffffffu);
      if (c < m) act[r * m + c] = from_f32<T>(x[0][j] * sigmoid<T>(x[0][j]) * x[1][j]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      top[h] = __reduce_max_sync(0xffffffffu, top[h]);
      float sc, f;
      run_scale(top[h], &sc, &f);
      if (lane == 0) scale[(r * 2 + h) * G + grp] = sc;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int c = grp * kGroup + j * 32 + lane;
        if (c < m) q[(r * 2 + h) * m + c] = f > 0.f ? static_cast<int8_t>(quantize(x[h][j], f) & 0xffu) : 0;
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    backward_any_kernel(const T* dact, const int8_t* __restrict__ q, const float* __restrict__ scale,
                        int64_t rows, int64_t ld, int m, int G, T* __restrict__ dgate, T* __restrict__ dup, T* act) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x) * kWarps,
             G);
  for (; at.row < rows; at.next()) {
    const int64_t r = at.row;
    const int grp = at.col;
    const float sg = scale[r * 2 * G + grp], su = scale[(r * 2 + 1) * G + grp];
    float d[4];
    int8_t qg[4], qu[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = grp * kGroup + j * 32 + lane;
      if (c < m) {
        d[j] = to_f32<T>(dact[r * m + c]);
        qg[j] = q[r * 2 * m + c];
        qu[j] = q[(r * 2 + 1) * m + c];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = grp * kGroup + j * 32 + lane;
      if (c >= m) continue;
      const Grads o = swiglu_grads<T>(__fmul_rn(qg[j], sg), __fmul_rn(qu[j], su), d[j]);
      dgate[r * ld + c] = from_f32<T>(o.dgate);
      dup[r * ld + c] = from_f32<T>(o.dup);
      if (act != nullptr) act[r * m + c] = from_f32<T>(o.act);
    }
  }
}

unsigned blocks_for(int64_t items, int64_t per_block, int num_sms) {
  const int64_t want = (items + per_block - 1) / per_block, cap = static_cast<int64_t>(num_sms) * 16;
  return static_cast<unsigned>(want < cap ? want : cap);
}

// Whether every row of the matrices at `ps` (row stride ld, and m) starts on 16 bytes and q's on 8.
bool vectors(const ActArgs& a, int es) {
  const void* ps[] = {a.gate, a.up, a.dact, a.act, a.dgate, a.dup};
  uintptr_t all = reinterpret_cast<uintptr_t>(a.q) << 1;
  for (const void* p : ps) all |= reinterpret_cast<uintptr_t>(p);
  return (all & 15u) == 0 && a.ld * es % 16 == 0 && a.m % kLane == 0;
}

template <typename T>
cudaError_t forward(const ActArgs& a, int num_sms, cudaStream_t st) {
  const int G = (a.m + kGroup - 1) / kGroup;
  const bool vec = vectors(a, sizeof(T));
  return launch_pdl(vec ? checkpoint_kernel<T> : checkpoint_any_kernel<T>,
                    dim3(blocks_for(a.rows * G, vec ? kThreads / kRunLanes : kWarps, num_sms)), dim3(kThreads), 0,
                    st, 1, static_cast<const T*>(a.gate), static_cast<const T*>(a.up), a.rows, a.ld, a.m, G,
                    static_cast<T*>(a.act), a.q, a.scale);
}

template <typename T>
cudaError_t backward(const ActArgs& a, int num_sms, cudaStream_t st) {
  const int G = (a.m + kGroup - 1) / kGroup;
  const bool vec = vectors(a, sizeof(T));
  const unsigned blocks = vec ? blocks_for(a.rows * (a.m / kLane), kThreads, num_sms)
                              : blocks_for(a.rows * G, kWarps, num_sms);
  return launch_pdl(vec ? backward_kernel<T> : backward_any_kernel<T>, dim3(blocks), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.dact), static_cast<const int8_t*>(a.q),
                    static_cast<const float*>(a.scale), a.rows, a.ld, a.m, G, static_cast<T*>(a.dgate),
                    static_cast<T*>(a.dup), static_cast<T*>(a.act));
}

}  // namespace

cudaError_t launch_swiglu_checkpoint(const ActArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? forward<__nv_bfloat16>(a, num_sms, st) : forward<float>(a, num_sms, st);
}

cudaError_t launch_swiglu_backward(const ActArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? backward<__nv_bfloat16>(a, num_sms, st) : backward<float>(a, num_sms, st);
}

}  // namespace pr2
