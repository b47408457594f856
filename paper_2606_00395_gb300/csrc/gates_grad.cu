// Gradient of the replay gates w.r.t. the router logits (pr2_replay_gates_backward).
//
// gates_s = rho_{idx_s} of rho = Softmax(p), so with dr_j = sum of dgates over the slots that name
// expert j:  dp_j = rho_j (dr_j - G),  G = sum_s dgates_s rho_{idx_s}.
// Renormalised gates g_s = rho_{idx_s} / S:  only the selected experts get a gradient,
// g_s (dgates_s - G'),  G' = sum_s dgates_s g_s:  the same form with g_s for rho.  (S may be a denormal number
// where the replayed experts have all but vanished; the gates are finite all the same.)
// 8, 16 or 32 lanes per token, lane s holding slot s, four experts a lane and step: every expert's -rho_j G is
// stored first, then the selected ones' values over it.  N not a multiple of 4: a warp per token, an expert
// a lane and step.  Bound by HBM for large batches of many experts (rho read, dp written): 262144 x 256 with
// k = 8 89 us (92 % of the copy rate); 10^6 x 64 with k = 4 113 us (71 %), where a group of lanes has one token's
// loads in flight; 4096 x 128 with k = 8 is 4.5 MB and takes 3.7 us a call, the host's part.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;

// Sum over a token's kLanes lanes.
template <int kLanes>
__device__ __forceinline__ float token_sum(float v) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A slot's probability (0: no slot) becomes its gate; returns G.  Renormalised, with S = 0 giving gates of 0 and
// a NaN going through: both sums go round together and take one reciprocal, of S 2^64 where S is small and 1 / S
// may overflow (10^6 x 64, k = 4 119 us; rho / S and G / S as two divisions 136).  There the products with
// dgates may be denormal numbers, and G is summed again from the gates.
constexpr float kSmallSum = 9.0949470e-13f, kUp = 18446744073709551616.f;  // 2^-40, 2^64
template <int kLanes>
__device__ __forceinline__ float gates_and_mean(float& rho, float dg, int norm) {
  float G = dg * rho;
  if (!norm) return token_sum<kLanes>(G);
  float S = rho;
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    G += __shfl_xor_sync(0xffffffffu, G, o);
    S += __shfl_xor_sync(0xffffffffu, S, o);
  }
  const float up = S < kSmallSum ? kUp : 1.f, inv = S == 0.f ? 0.f : 1.f / (S * up);
  rho = rho * up * inv;
  G *= inv;
  if (__any_sync(0xffffffffu, S < kSmallSum)) {
    const float again = token_sum<kLanes>(dg * rho);
    if (S < kSmallSum) G = again;
  }
  return G;
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
    float gate = ok ? probs[t * N + e] : 0.f;
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
    if (!ok) dg = gate = 0.f;
    const float G = gates_and_mean<kLanes>(gate, dg, norm), others = norm ? 0.f : -G;
    float4* out = reinterpret_cast<float4*>(dlogits + t * N);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (live && sub + i * kLanes < vecs)
        out[sub + i * kLanes] = make_float4(others * r[i].x, others * r[i].y, others * r[i].z, others * r[i].w);
    __syncwarp();  // (the selected ones' values come after)
    if (ok) dlogits[t * N + e] = gate * (dg - G);
  }
}

__global__ void __launch_bounds__(kWarps * 32)
    gates_backward_any_kernel(const float* __restrict__ probs, const int32_t* __restrict__ idx,
                          const float* __restrict__ dgates, int64_t T, int N, int k, int norm,
                          float* __restrict__ dlogits, int32_t* __restrict__ status) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); t < T;
       t += static_cast<int64_t>(gridDim.x) * kWarps) {
    const int e = lane < k ? idx[t * k + lane] : -1;
    float dg = lane < k ? dgates[t * k + lane] : 0.f;
    bool ok = lane < k && e >= 0 && e < N;
    for (int s = 0; s < k - 1; ++s) {
      const int other = __shfl_sync(0xffffffffu, e, s);
      if (s < lane && other == e) ok = false;
    }
    if (lane < k && !ok && status != nullptr) atomicOr(status, PR2_STATUS_BAD_INDEX);
    if (!ok) dg = 0.f;
    float gate = ok ? probs[t * N + e] : 0.f;
    const float G = gates_and_mean<32>(gate, dg, norm), others = norm ? 0.f : -G;
    for (int j = lane; j < N; j += 32) dlogits[t * N + j] = others * probs[t * N + j];
    __syncwarp();  // (the selected ones' values come after)
    if (ok) dlogits[t * N + e] = gate * (dg - G);
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
