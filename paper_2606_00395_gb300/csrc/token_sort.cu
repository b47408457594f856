// Rows of tokens in expert order and back, with their gradients (pr2_token_*).
//
//   sort:            x[inv[t,s]] = h[t];            backward  dh[t] = sum_s dx[inv[t,s]]
//   unsort:          out[t] = sum_s g[t,s] y[inv[t,s]]
//   unsort_backward: dy[inv[t,s]] = g[t,s] dout[t],  dg[t,s] = <dout[t], y[inv[t,s]]>
// Every kernel walks tokens: a token's row is read or written once and its k rows in the other
// order are found through inv, so nothing is written twice and no sum is split over blocks (the
// results do not depend on the launch).  Rows past offsets[N], which no slot names, are zeroed.
// A row number outside [0, T k) is taken as an invalid slot.
// One block per token.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kThreads = 128;
constexpr int kMaxK = kMaxTopKSimt;

__device__ __forceinline__ int64_t row_of(const int32_t* __restrict__ inv, int64_t f, int64_t F) {
  const int64_t p = inv[f];
  return p >= 0 && p < F ? p : -1;
}

// First row that no slot names.
__device__ __forceinline__ int64_t rows_used(const int32_t* __restrict__ offsets, int N, int64_t F) {
  const int64_t n = offsets[N];
  return n < 0 ? 0 : n < F ? n : F;
}

template <typename T>
__device__ __forceinline__ void zero_rows(T* x, int64_t from, int64_t F, int d) {
  for (int64_t r = from + blockIdx.x; r < F; r += gridDim.x)
    for (int c = threadIdx.x; c < d; c += blockDim.x) x[r * d + c] = from_f32<T>(0.f);
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    sort_any_kernel(const T* __restrict__ h, const int32_t* __restrict__ inv,
                    const int32_t* __restrict__ offsets, int64_t Tn, int d, int N, int k,
                    T* __restrict__ x, int32_t* __restrict__ perm, const int32_t* status) {
  pdl_wait();
  pdl_trigger();
  if (status_timed_out(status)) return;  // dispatch gave up: its tables may be unwritten
  const int64_t F = Tn * k;
  const int64_t used = rows_used(offsets, N, F);
  if (perm != nullptr)
    for (int64_t r = used + static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; r < F;
         r += static_cast<int64_t>(gridDim.x) * blockDim.x)
      perm[r] = -1;
  if (x == nullptr) return;
  for (int64_t t = blockIdx.x; t < Tn; t += gridDim.x)
    for (int s = 0; s < k; ++s) {
      const int64_t r = row_of(inv, t * k + s, F);
      if (r < 0) continue;
      for (int c = threadIdx.x; c < d; c += blockDim.x) x[r * d + c] = h[t * d + c];
    }
  zero_rows(x, used, F, d);
}

// gates NULL: all 1
template <typename T>
__global__ void __launch_bounds__(kThreads)
    sum_any_kernel(const T* __restrict__ y, const int32_t* __restrict__ inv,
                   const float* __restrict__ gates, int64_t Tn, int d, int k, T* __restrict__ out) {
  pdl_wait();
  pdl_trigger();
  const int64_t F = Tn * k;
  for (int64_t t = blockIdx.x; t < Tn; t += gridDim.x)
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
      float acc = 0.f;
      for (int s = 0; s < k; ++s) {
        const int64_t r = row_of(inv, t * k + s, F);
        if (r >= 0) acc = fmaf(gates != nullptr ? gates[t * k + s] : 1.f, to_f32<T>(y[r * d + c]), acc);
      }
      out[t * d + c] = from_f32<T>(acc);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    unsort_backward_any_kernel(const T* __restrict__ dout, const T* __restrict__ y,
                               const float* __restrict__ gates, const int32_t* __restrict__ inv,
                               const int32_t* __restrict__ offsets, int64_t Tn, int d, int N, int k,
                               T* __restrict__ dy, float* __restrict__ dgates) {
  __shared__ float part[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int64_t F = Tn * k;
  for (int64_t t = blockIdx.x; t < Tn; t += gridDim.x)
    for (int s = 0; s < k; ++s) {
      const int64_t r = row_of(inv, t * k + s, F);
      const float g = gates[t * k + s];
      float acc = 0.f;
      if (r >= 0)
        for (int c = threadIdx.x; c < d; c += blockDim.x) {
          const float v = to_f32<T>(dout[t * d + c]);
          acc = fmaf(v, to_f32<T>(y[r * d + c]), acc);
          dy[r * d + c] = from_f32<T>(g * v);
        }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = acc;
      __syncthreads();
      if (threadIdx.x == 0) {
        float all = part[0];
        for (int w = 1; w < kThreads / 32; ++w) all += part[w];
        dgates[t * k + s] = all;
      }
      __syncthreads();
    }
  zero_rows(dy, rows_used(offsets, N, F), F, d);
}

dim3 grid_for(int64_t T, int num_sms) {
  const int64_t cap = static_cast<int64_t>(num_sms) * 16;
  return dim3(static_cast<unsigned>(T < cap ? T : cap));
}

template <typename T>
cudaError_t sort_rows(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return launch_pdl(sort_any_kernel<T>, grid_for(a.T, num_sms), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.src), a.inv, a.offsets, a.T, a.d, a.N, a.k,
                    static_cast<T*>(a.dst), a.perm, a.status);
}
template <typename T>
cudaError_t sum_rows(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return launch_pdl(sum_any_kernel<T>, grid_for(a.T, num_sms), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.src), a.inv, a.gates, a.T, a.d, a.k,
                    static_cast<T*>(a.dst));
}
template <typename T>
cudaError_t unsort_backward(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return launch_pdl(unsort_backward_any_kernel<T>, grid_for(a.T, num_sms), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.src), static_cast<const T*>(a.y), a.gates, a.inv,
                    a.offsets, a.T, a.d, a.N, a.k, static_cast<T*>(a.dst), a.dgates);
}

}  // namespace

cudaError_t launch_token_sort(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? sort_rows<__nv_bfloat16>(a, num_sms, st) : sort_rows<float>(a, num_sms, st);
}
cudaError_t launch_token_sum(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? sum_rows<__nv_bfloat16>(a, num_sms, st) : sum_rows<float>(a, num_sms, st);
}
cudaError_t launch_token_unsort_backward(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return a.bf16 ? unsort_backward<__nv_bfloat16>(a, num_sms, st)
                : unsort_backward<float>(a, num_sms, st);
}

}  // namespace pr2
