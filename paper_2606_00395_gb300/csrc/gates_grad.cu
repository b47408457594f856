// Gradient of the replay gates w.r.t. the router logits (pr2_replay_gates_backward).
//
// gates_s = rho_{idx_s} of rho = Softmax(p), so with dr_j = sum of dgates over the slots that name
// expert j:  dp_j = rho_j (dr_j - G),  G = sum_s dgates_s rho_{idx_s}.
// Renormalised gates g_s = rho_{idx_s} / S:  d rho_{idx_s} = (dgates_s - sum_u dgates_u g_u) / S =: dr,
// and G = sum dr rho = 0 exactly, so only the selected experts get a gradient, g_s (dgates_s - G').
// 8, 16 or 32 lanes per token, lane s holding slot s, four experts a lane and step: every expert's -rho_j G is
// stored first, then the selected ones' values over it.  N not a multiple of 4: a warp per token with dr
// in shared memory.  Bound by HBM for large batches (rho read, dp written): 262144 x 256 with
// k = 8 91 us (90 % of the copy rate), 10^6 x 64 with k = 4 117 us (68 %); 4096 x 128 with k = 8
// is 4.5 MB and takes 4.4 us a call, the host's part.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;

// Sums over a token's kLanes lanes.
template <int kLanes>
__device__ __forceinline__ void token_sums(float& a, float& b) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
}

// N % 4 == 0, N <= 16 kLanes, k <= kLanes; rows on 16 bytes.
template <int kLanes>
__global__ void __launch_bounds__(kWarps * 32)
    gates_backward_kernel(const float* __restrict__ probs, const int32_t* __restrict__ idx,
                          const float* __restrict__ dgates, int64_t T, int N, int k, int norm,
                          float* __restrict__ dlogits, int32_t* __restrict__ status) {
  constexpr int kTokens = kWarps * 32 / kLanes, kSteps = 4;
  pdl_wait();
  pdl_trigger();
  const int sub = threadIdx.x % kLanes, vecs = N / 4;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kTokens;
  int64_t t = static_cast<int64_t>(blockIdx.x) * kTokens + threadIdx.x / kLanes;
  // a token's slots are loaded a token ahead: its selected probabilities wait for them
  auto slot = [&](int64_t at, int& e, float& dg) {
    const bool own = at < T && sub < k;
    e = own ? idx[at * k + sub] : -1;
    dg = own ? dgates[at * k + sub] : 0.f;
  };
  int next_e;
  float next_dg;
  slot(t, next_e, next_dg);
  for (; __any_sync(0xffffffffu, t < T); t += step) {  // (a warp's tokens go round together)
    const bool live = t < T;
    const int e = next_e;
    float dg = next_dg;
    bool ok = e >= 0 && e < N;
    float rho = ok ? probs[t * N + e] : 0.f;
    float4 r[kSteps];
    const float4* row = reinterpret_cast<const float4*>(probs + t * N);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (live && sub + i * kLanes < vecs) r[i] = __ldcs(row + sub + i * kLanes);
    slot(t + step, next_e, next_dg);
    for (int s = 0; s < k - 1; ++s) {
      const int other = __shfl_sync(0xffffffffu, e, s, kLanes);
      if (s < sub && other == e) ok = false;
    }
    if (live && sub < k && !ok && status != nullptr) atomicOr(status, PR2_STATUS_BAD_INDEX);
    if (!ok) dg = rho = 0.f;
    float G = dg * rho, S = rho;
    token_sums<kLanes>(G, S);
    if (norm) {
      dg = S > 0.f ? (dg - G / S) / S : 0.f;
      G = 0.f;
    }
    float4* out = reinterpret_cast<float4*>(dlogits + t * N);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (live && sub + i * kLanes < vecs)
        out[sub + i * kLanes] = make_float4(-G * r[i].x, -G * r[i].y, -G * r[i].z, -G * r[i].w);
    __syncwarp();  // (the selected ones' values come after)
    if (ok) dlogits[t * N + e] = rho * (dg - G);
  }
}

__global__ void __launch_bounds__(kWarps * 32)
    gates_backward_any_kernel(const float* __restrict__ probs, const int32_t* __restrict__ idx,
                          const float* __restrict__ dgates, int64_t T, int N, int k, int norm,
                          float* __restrict__ dlogits, int32_t* __restrict__ status) {
  __shared__ float dr_s[kWarps][kMaxExperts];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  float* dr = dr_s[threadIdx.x >> 5];
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); t < T;
       t += static_cast<int64_t>(gridDim.x) * kWarps) {
    const int e = lane < k ? idx[t * k + lane] : -1;
    float dg = lane < k ? dgates[t * k + lane] : 0.f;
    for (int j = lane; j < N; j += 32) dr[j] = 0.f;
    bool ok = lane < k && e >= 0 && e < N;
    for (int s = 0; s < k - 1; ++s) {
      const int other = __shfl_sync(0xffffffffu, e, s);
      if (s < lane && other == e) ok = false;
    }
    if (lane < k && !ok && status != nullptr) atomicOr(status, PR2_STATUS_BAD_INDEX);
    const float rho = ok ? probs[t * N + e] : 0.f;
    if (!ok) dg = 0.f;
    float G = dg * rho, S = rho;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      G += __shfl_xor_sync(0xffffffffu, G, o);
      S += __shfl_xor_sync(0xffffffffu, S, o);
    }
    if (norm) {
      dg = S > 0.f ? (dg - G / S) / S : 0.f;
      G = 0.f;
    }
    __syncwarp();
    if (ok) dr[e] = dg;
    __syncwarp();
    for (int j = lane; j < N; j += 32) dlogits[t * N + j] = probs[t * N + j] * (dr[j] - G);
    __syncwarp();
  }
}

}  // namespace

cudaError_t launch_gates_backward(const float* probs, const int32_t* idx, const float* dgates,
                                  int64_t T, int N, int k, bool norm, float* dlogits,
                                  int32_t* status, int num_sms, cudaStream_t st) {
  const bool vec =
      N % 4 == 0 && ((reinterpret_cast<uintptr_t>(probs) | reinterpret_cast<uintptr_t>(dlogits)) & 15u) == 0;
  const int lanes = !vec || N > 64 || k > 16 ? 32 : N > 32 || k > 8 ? 16 : 8;
  const int per_block = kWarps * 32 / lanes;
  int64_t blocks = (T + per_block - 1) / per_block;
  const int64_t cap = static_cast<int64_t>(num_sms) * 8;
  if (blocks > cap) blocks = cap;
  auto* kernel = !vec ? gates_backward_any_kernel
                 : lanes == 32 ? gates_backward_kernel<32>
                 : lanes == 16 ? gates_backward_kernel<16>
                               : gates_backward_kernel<8>;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kWarps * 32), 0, st, 1, probs, idx, dgates, T,
                    N, k, norm ? 1 : 0, dlogits, status);
}

}  // namespace pr2
