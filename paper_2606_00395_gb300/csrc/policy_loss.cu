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
// Tokens are dealt to blocks by their number; a block sums its tokens' terms in double and
// policy_finish_kernel the blocks' in order, so the loss does not depend on timing.
// One block per row.
#include <math_constants.h>

#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kThreads = 256;

// Running softmax sums over the entries above -inf: maximum m, l = sum exp(z - m),
// e = sum exp(z - m) (z - m).  Nothing seen: m = -inf, l = 0.  A NaN or +inf makes l NaN.
struct RowSum {
  float m, l, e;
};

// The sums relative to a larger maximum.
__device__ __forceinline__ void raise(RowSum& s, float m) {
  if (s.m == m) return;
  const float gap = s.m - m;
  const float f = __expf(gap);  // 0 from m = -inf
  s.e = s.m == -CUDART_INF_F ? s.l * f : fmaf(gap, s.l, s.e) * f;
  s.l *= f;
  s.m = m;
}

__device__ __forceinline__ void add(RowSum& s, float z) {
  if (z == -CUDART_INF_F) return;
  if (z > s.m) raise(s, z);
  const float x = z - s.m, p = __expf(x);
  s.l += p;
  s.e = fmaf(p, x, s.e);
}

__device__ __forceinline__ RowSum join(RowSum a, RowSum b) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m);
  raise(b, m);
  return RowSum{m, a.l + b.l, a.e + b.e};
}

// A token's terms: policy part, KL part and clip flag, each times its weight, and the factor c of
// its gradient.
struct TokenTerms {
  float policy, kl, shut, c;
};

__device__ __forceinline__ TokenTerms token_terms(const PolicyArgs& a, int64_t t, float w,
                                                  float logp) {
  const float A = a.advantage[t];
  const float r = a.logp_old != nullptr ? expf(logp - a.logp_old[t]) : 1.f;
  const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
  // min(r A, clip(r) A) takes the clipped side exactly where the clip shuts the gradient off; a NaN
  // ratio goes through.  A token of advantage 0 has no policy part, however large its ratio.
  const bool shut = A > 0.f ? r > hi : A < 0.f && r < lo;
  const float part = A == 0.f ? 0.f : (shut ? (A > 0.f ? hi : lo) : r) * A;
  TokenTerms o;
  o.policy = -w * part;
  o.shut = shut ? w : 0.f;
  float c = shut || A == 0.f ? 0.f : -r * A;
  o.kl = 0.f;
  if (a.logp_ref != nullptr) {
    const float gap = a.logp_ref[t] - logp, x = expm1f(gap);
    o.kl = w * (isinf(x) ? x : x - gap);
    if (a.kl_coef > 0.f) c -= a.kl_coef * x;
  }
  o.c = w * c;
  return o;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_any_kernel(const PolicyArgs a) {
  __shared__ RowSum part[kThreads / 32];
  __shared__ float row_c[3];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31;
  double sums[3] = {0.0, 0.0, 0.0};
  const T* logits = static_cast<const T*>(a.logits);
  T* grad = static_cast<T*>(a.grad);
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const T* row = logits + t * a.ld_logits;
    const int target = a.target[t];
    float w = a.weight != nullptr ? a.weight[t] : 1.f / static_cast<float>(a.T);
    if (w != 0.f && (target < 0 || target >= a.V)) {
      w = 0.f;
      if (tid == 0 && a.status != nullptr) atomicOr(a.status, PR2_STATUS_BAD_INDEX);
    }
    float f = 0.f, fl = 0.f, m = 0.f;
    if (w != 0.f) {
      RowSum s{-CUDART_INF_F, 0.f, 0.f};
      for (int64_t v = tid; v < a.V; v += kThreads) add(s, to_f32<T>(row[v]) * a.inv_temp);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        s = join(s, RowSum{__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.l, o),
                           __shfl_xor_sync(0xffffffffu, s.e, o)});
      if (lane == 0) part[tid >> 5] = s;
      __syncthreads();
      if (tid == 0) {
        for (int i = 1; i < kThreads / 32; ++i) s = join(s, part[i]);
        if (s.m == -CUDART_INF_F && s.l == 0.f) {  // no entry above -inf
          if (a.logp != nullptr) a.logp[t] = -CUDART_INF_F;
          if (a.entropy != nullptr) a.entropy[t] = 0.f;
          row_c[0] = 0.f;
        } else {
          const float logl = logf(s.l);
          const float logp = (to_f32<T>(row[target]) * a.inv_temp - s.m) - logl;
          if (a.logp != nullptr) a.logp[t] = logp;
          if (a.entropy != nullptr) a.entropy[t] = logl - s.e / s.l;
          const TokenTerms k = token_terms(a, t, w, logp);
          sums[0] += k.policy;
          sums[1] += k.kl;
          sums[2] += k.shut;
          row_c[0] = k.c * a.inv_temp * a.grad_scale;
          row_c[1] = row_c[0] / s.l;
          row_c[2] = s.m;
        }
      }
      __syncthreads();
      f = row_c[0];
      fl = row_c[1];
      m = row_c[2];
    } else if (tid == 0) {
      if (a.logp != nullptr) a.logp[t] = 0.f;
      if (a.entropy != nullptr) a.entropy[t] = 0.f;
    }
    if (grad == nullptr) continue;
    T* out = grad + t * a.ld_grad;
    for (int64_t v = tid; v < a.V; v += kThreads) {
      float g = 0.f;
      if (f != 0.f) g = fmaf(-fl, __expf(to_f32<T>(row[v]) * a.inv_temp - m), v == target ? f : 0.f);
      out[v] = from_f32<T>(g);
    }
  }
  if (tid == 0) {
    double* p = a.partial + static_cast<int64_t>(blockIdx.x) * 4;
    p[0] = sums[0];
    p[1] = sums[1];
    p[2] = sums[2];
  }
}

__global__ void __launch_bounds__(256)
    policy_finish_kernel(const double* __restrict__ partial, int n, float kl_coef,
                         float* __restrict__ loss) {
  __shared__ double sh[3][256];
  pdl_wait();
  pdl_trigger();
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = threadIdx.x; i < n; i += 256)
    for (int j = 0; j < 3; ++j) s[j] += partial[i * 4 + j];
  for (int j = 0; j < 3; ++j) sh[j][threadIdx.x] = s[j];
  for (int o = 128; o > 0; o >>= 1) {
    __syncthreads();
    if (threadIdx.x < o)
      for (int j = 0; j < 3; ++j) sh[j][threadIdx.x] += sh[j][threadIdx.x + o];
  }
  if (threadIdx.x == 0) {
    loss[0] = static_cast<float>(kl_coef > 0.f ? sh[0][0] + kl_coef * sh[1][0] : sh[0][0]);
    for (int j = 0; j < 3; ++j) loss[1 + j] = static_cast<float>(sh[j][0]);
  }
}

}  // namespace

cudaError_t launch_policy_loss(const PolicyArgs& a, int num_sms, cudaStream_t st) {
  int64_t blocks = static_cast<int64_t>(num_sms) * 4;
  if (blocks > a.T) blocks = a.T;
  if (blocks > kPolicyParts) blocks = kPolicyParts;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  cudaError_t err = a.bf16 ? launch_pdl(policy_any_kernel<__nv_bfloat16>, grid, block, 0, st, 1, a)
                           : launch_pdl(policy_any_kernel<float>, grid, block, 0, st, 1, a);
  if (err != cudaSuccess) return err;
  return launch_pdl(policy_finish_kernel, dim3(1), dim3(256), 0, st, 1,
                    static_cast<const double*>(a.partial), static_cast<int>(blocks), a.kl_coef, a.loss);
}

}  // namespace pr2
