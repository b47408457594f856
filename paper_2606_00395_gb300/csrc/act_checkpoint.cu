// SwiGLU activation with an 8-bit checkpoint of its inputs, and its backward pass.
//
// act = silu(gate) up; a run of 128 elements of a row of gate or up is held as q = round(x 127 / top),
// scale = top / 127, top = max |x|.  Backward, from g = q scale: s = 1 / (1 + exp(-g)),
//   dgate = dact u s (1 + g (1 - s)),  dup = dact g s,  act = g s u.
// One warp per run.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;
constexpr int kGroup = PR2_CKPT_GROUP;
constexpr float kInv127 = static_cast<float>(1.0 / 127.0);
constexpr float kTinyTop = 1e-30f;

// From the exponential that cannot overflow: with exp(-x) the sigmoid of x < -88 would be 0 where
// x sigmoid(x) is still a normal number.
__device__ __forceinline__ float sigmoid(float x) {
  const float e = __expf(-fabsf(x));
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

template <typename T>
__global__ void __launch_bounds__(kWarps * 32)
    checkpoint_any_kernel(const T* __restrict__ gate, const T* __restrict__ up, int64_t rows,
                          int64_t ld, int m, T* __restrict__ act, int8_t* __restrict__ q,
                          float* __restrict__ scale) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int G = (m + kGroup - 1) / kGroup;
  const int64_t n = rows * G;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); i < n;
       i += static_cast<int64_t>(gridDim.x) * kWarps) {
    const int64_t r = i / G;
    const int grp = static_cast<int>(i - r * G);
    float x[2][4];
    uint32_t top[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = grp * kGroup + j * 32 + lane;
      x[0][j] = c < m ? to_f32<T>(gate[r * ld + c]) : 0.f;
      x[1][j] = c < m ? to_f32<T>(up[r * ld + c]) : 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) top[h] = max(top[h], __float_as_uint(x[h][j]) & 0x7fffffffu);
      if (c < m) act[r * m + c] = from_f32<T>(x[0][j] * sigmoid(x[0][j]) * x[1][j]);
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
        if (c < m) q[(r * 2 + h) * m + c] = f > 0.f ? static_cast<int8_t>(__float2int_rn(__fmul_rn(x[h][j], f))) : 0;
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256)
    backward_any_kernel(const T* dact, const int8_t* __restrict__ q,
                        const float* __restrict__ scale, int64_t rows, int64_t ld, int m,
                        T* __restrict__ dgate, T* __restrict__ dup, T* act) {
  pdl_wait();
  pdl_trigger();
  const int G = (m + kGroup - 1) / kGroup;
  const int64_t n = rows * m;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < n;
       i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    const int64_t r = i / m;
    const int c = static_cast<int>(i - r * m);
    const float g = __fmul_rn(q[r * 2 * m + c], scale[r * 2 * G + c / kGroup]);
    const float u = __fmul_rn(q[(r * 2 + 1) * m + c], scale[(r * 2 + 1) * G + c / kGroup]);
    const float d = to_f32<T>(dact[i]);
    const float s = sigmoid(g);
    dup[r * ld + c] = from_f32<T>(d * g * s);
    dgate[r * ld + c] = from_f32<T>(d * u * s * (1.f + g * (1.f - s)));
    if (act != nullptr) act[i] = from_f32<T>(g * s * u);
  }
}

unsigned blocks_for(int64_t items, int64_t per_block, int num_sms) {
  const int64_t want = (items + per_block - 1) / per_block, cap = static_cast<int64_t>(num_sms) * 8;
  return static_cast<unsigned>(want < cap ? want : cap);
}

template <typename T>
cudaError_t forward(const ActArgs& a, int num_sms, cudaStream_t st) {
  const int64_t runs = a.rows * ((a.m + kGroup - 1) / kGroup);
  return launch_pdl(checkpoint_any_kernel<T>, dim3(blocks_for(runs, kWarps, num_sms)),
                    dim3(kWarps * 32), 0, st, 1, static_cast<const T*>(a.gate),
                    static_cast<const T*>(a.up), a.rows, a.ld, a.m, static_cast<T*>(a.act), a.q,
                    a.scale);
}

template <typename T>
cudaError_t backward(const ActArgs& a, int num_sms, cudaStream_t st) {
  return launch_pdl(backward_any_kernel<T>, dim3(blocks_for(a.rows * a.m, 256, num_sms)), dim3(256),
                    0, st, 1, static_cast<const T*>(a.dact), static_cast<const int8_t*>(a.q),
                    static_cast<const float*>(a.scale), a.rows, a.ld, a.m, static_cast<T*>(a.dgate),
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
