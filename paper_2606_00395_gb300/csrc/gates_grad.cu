// Gradient of the replay gates w.r.t. the router logits (pr2_replay_gates_backward).
//
// gates_s = rho_{idx_s} of rho = Softmax(p), so with dr_j = sum of dgates over the slots that name
// expert j:  dp_j = rho_j (dr_j - G),  G = sum_s dgates_s rho_{idx_s}.
// Renormalised gates g_s = rho_{idx_s} / S:  d rho_{idx_s} = (dgates_s - sum_u dgates_u g_u) / S =: dr,
// and G = sum dr rho = 0 exactly, so only the selected experts get a gradient, g_s (dgates_s - G').
// One warp per token, lane s holding slot s; dr lies in shared memory.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;

__global__ void __launch_bounds__(kWarps * 32)
    gates_backward_kernel(const float* __restrict__ probs, const int32_t* __restrict__ idx,
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
  int64_t blocks = (T + kWarps - 1) / kWarps;
  const int64_t cap = static_cast<int64_t>(num_sms) * 8;
  if (blocks > cap) blocks = cap;
  return launch_pdl(gates_backward_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kWarps * 32), 0,
                    st, 1, probs, idx, dgates, T, N, k, norm ? 1 : 0, dlogits, status);
}

}  // namespace pr2
