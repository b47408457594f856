// C ABI of the training-side operators (declared in include/pr2.h): argument validation, workspace
// layout and the launches of each entry point.
#include <cmath>
#include <initializer_list>

#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int64_t kMaxSlots = int64_t{1} << 30;
constexpr int kMaxWidth = 1 << 30;  // of a token's row: the kernels count columns, a step past it too, in 32 bits

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) % bytes) == 0; }
bool aligned4(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned(p, 4)) return false;
  return true;
}

pr2_status check_policy(const pr2_policy_dims* dm) {
  if (dm == nullptr || dm->T < 0 || dm->V < 1 || dm->ld_logits < dm->V || dm->ld_grad < dm->V)
    return PR2_ERR_INVALID_ARG;
  if (dm->dtype != PR2_FP32 && dm->dtype != PR2_BF16) return PR2_ERR_INVALID_ARG;
  if (dm->flags & ~PR2_F_SYNC_STATUS) return PR2_ERR_INVALID_ARG;
  const float all[] = {dm->inv_temp, dm->clip_low, dm->clip_high, dm->kl_coef, dm->grad_scale};
  for (float x : all)
    if (!std::isfinite(x)) return PR2_ERR_INVALID_ARG;
  if (dm->inv_temp <= 0.f || dm->clip_low < 0.f || dm->clip_low > 1.f || dm->clip_high < 0.f ||
      dm->kl_coef < 0.f)
    return PR2_ERR_INVALID_ARG;
  const int64_t widest = dm->ld_logits > dm->ld_grad ? dm->ld_logits : dm->ld_grad;
  if (dm->V > (int64_t{1} << 30) || dm->T > kMaxSlots ||
      (dm->T > 0 && widest > (int64_t{1} << 60) / dm->T))
    return PR2_ERR_UNSUPPORTED;
  return PR2_OK;
}

// The sizes that the token calls use: T, d, N, k, dtype.
pr2_status check_tokens(const pr2_dims* dm) {
  if (dm == nullptr || dm->T < 0 || dm->d <= 0 || dm->N <= 0 || dm->k <= 0 || dm->k > dm->N)
    return PR2_ERR_INVALID_ARG;
  if (dm->dtype != PR2_FP32 && dm->dtype != PR2_BF16) return PR2_ERR_INVALID_ARG;
  if (dm->flags & ~(PR2_F_SYNC_STATUS | PR2_F_DELTA_LOSS | PR2_F_NORMALIZE_TOPK))
    return PR2_ERR_INVALID_ARG;
  if (dm->N > kMaxExperts || dm->k > kMaxTopKSimt || dm->T > kMaxSlots / dm->k || dm->d > kMaxWidth)
    return PR2_ERR_UNSUPPORTED;
  return PR2_OK;
}

size_t esize(int32_t dtype) { return dtype == PR2_FP32 ? 4 : 2; }

struct PlanWorkspace {
  int32_t* status;
  int32_t* blk_hist;
  int32_t* counts;
  int32_t* num_tiles;
  unsigned int* sync_ctr;
  TileEntry* tiles;
  size_t total;
};

PlanWorkspace carve_plan(const pr2_dims& dm, uint8_t* base) {
  PlanWorkspace w{};
  size_t off = 0;
  auto take = [&](size_t bytes) -> uint8_t* {
    uint8_t* p = base ? base + off : nullptr;
    off += (bytes + 255) & ~size_t{255};
    return p;
  };
  const int64_t F = dm.T * dm.k;
  const int64_t nblk = (F + kDispatchChunk - 1) / kDispatchChunk;
  w.status = reinterpret_cast<int32_t*>(take(sizeof(int32_t)));
  w.blk_hist = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * (size_t)nblk * dm.N));
  w.counts = reinterpret_cast<int32_t*>(take(sizeof(int32_t) * dm.N));
  w.num_tiles = reinterpret_cast<int32_t*>(take(sizeof(int32_t)));
  w.sync_ctr = reinterpret_cast<unsigned int*>(take(sizeof(unsigned int)));
  w.tiles = reinterpret_cast<TileEntry*>(
      take(sizeof(TileEntry) * (size_t)(F / kMinTileRows + dm.N + 1)));
  w.total = off;
  return w;
}

pr2_status check_act(const pr2_act_dims* dm) {
  if (dm == nullptr || dm->rows < 0 || dm->m < 1 || dm->ld < dm->m) return PR2_ERR_INVALID_ARG;
  if (dm->dtype != PR2_FP32 && dm->dtype != PR2_BF16) return PR2_ERR_INVALID_ARG;
  if (dm->m > (1 << 24) || dm->rows > (int64_t{1} << 34) ||
      (dm->rows > 0 && dm->ld > (int64_t{1} << 60) / dm->rows))
    return PR2_ERR_UNSUPPORTED;
  return PR2_OK;
}

}  // namespace
}  // namespace pr2

using namespace pr2;

extern "C" {

size_t pr2_policy_loss_workspace_bytes(const pr2_policy_dims* dims) {
  if (check_policy(dims) != PR2_OK) return 0;
  const size_t order = dims->T <= kPolicyDealt ? sizeof(int) * static_cast<size_t>(dims->T + 1) : 0;
  return sizeof(double) * 4 * kPolicyParts + order;
}

pr2_status pr2_policy_loss(const pr2_policy_dims* dims, const void* logits, const int32_t* target,
                           const float* weight, const float* advantage, const float* logp_old,
                           const float* logp_ref, float* loss, float* logp, float* entropy,
                           void* grad, void* workspace, size_t ws_bytes, int32_t* status_dev,
                           void* stream) {
  pr2_status s = check_policy(dims);
  if (s != PR2_OK) return s;
  const pr2_policy_dims& dm = *dims;
  if (loss == nullptr) return PR2_ERR_INVALID_ARG;
  if ((dm.flags & PR2_F_SYNC_STATUS) && status_dev == nullptr) return PR2_ERR_INVALID_ARG;
  if (dm.T > 0 && (logits == nullptr || target == nullptr || advantage == nullptr ||
                   (dm.kl_coef > 0.f && logp_ref == nullptr)))
    return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(logits, es) || !aligned(grad, es) ||
      !aligned4({target, weight, advantage, logp_old, logp_ref, loss, logp, entropy, status_dev}))
    return PR2_ERR_INVALID_ARG;
  if (grad != nullptr && grad == logits && dm.ld_grad != dm.ld_logits) return PR2_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dm.T == 0) return finish(cudaMemsetAsync(loss, 0, 4 * sizeof(float), st), dm.flags, status_dev, st);
  if (workspace == nullptr || ws_bytes < pr2_policy_loss_workspace_bytes(dims) ||
      !aligned(workspace, 256))
    return PR2_ERR_WORKSPACE;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  PolicyArgs a{};
  a.T = dm.T;
  a.V = dm.V;
  a.ld_logits = dm.ld_logits;
  a.ld_grad = dm.ld_grad;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.inv_temp = dm.inv_temp;
  a.clip_low = dm.clip_low;
  a.clip_high = dm.clip_high;
  a.kl_coef = dm.kl_coef;
  a.grad_scale = dm.grad_scale;
  a.logits = logits;
  a.target = target;
  a.weight = weight;
  a.advantage = advantage;
  a.logp_old = logp_old;
  a.logp_ref = logp_ref;
  a.loss = loss;
  a.logp = logp;
  a.entropy = entropy;
  a.grad = grad;
  a.partial = static_cast<double*>(workspace);
  a.order = reinterpret_cast<int*>(a.partial + 4 * kPolicyParts);
  a.status = status_dev;
  return finish(launch_policy_loss(a, num_sms, st), dm.flags, status_dev, st);
}

size_t pr2_token_sort_workspace_bytes(const pr2_dims* dims) {
  if (check_tokens(dims) != PR2_OK) return 0;
  return carve_plan(*dims, nullptr).total;
}

pr2_status pr2_token_sort(const pr2_dims* dims, const void* h, const int32_t* idx, void* x,
                          int32_t* offsets, int32_t* perm, int32_t* inv, void* workspace,
                          size_t ws_bytes, int32_t* status_dev, void* stream) {
  pr2_status s = check_tokens(dims);
  if (s != PR2_OK) return s;
  const pr2_dims& dm = *dims;
  if ((dm.flags & PR2_F_SYNC_STATUS) && status_dev == nullptr) return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(h, es) || !aligned(x, es) || !aligned4({idx, offsets, perm, inv, status_dev}))
    return PR2_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dm.T == 0) {  // empty tensors may have NULL data
    if (offsets == nullptr) return PR2_ERR_INVALID_ARG;
    return finish(cudaMemsetAsync(offsets, 0, sizeof(int32_t) * (dm.N + 1), st), dm.flags, status_dev,
                  st);
  }
  if (offsets == nullptr || inv == nullptr || (h == nullptr) != (x == nullptr))
    return PR2_ERR_INVALID_ARG;
  if (idx == nullptr ? x == nullptr : perm == nullptr) return PR2_ERR_INVALID_ARG;
  if (idx != nullptr && (workspace == nullptr || ws_bytes < carve_plan(dm, nullptr).total ||
                         !aligned(workspace, 256)))
    return PR2_ERR_WORKSPACE;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  TokenArgs a{};
  a.T = dm.T;
  a.d = dm.d;
  a.N = dm.N;
  a.k = dm.k;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.inv = inv;
  a.offsets = offsets;
  a.src = h;
  a.dst = x;
  if (idx != nullptr && dm.T * dm.k <= kPlanSlots) {
    const PlanWorkspace w = carve_plan(dm, static_cast<uint8_t*>(workspace));
    const cudaError_t err = launch_token_plan(idx, static_cast<int>(dm.T * dm.k), dm.k, dm.N, w.blk_hist,
                                              offsets, perm, inv, status_dev, st);
    if (err != cudaSuccess || x == nullptr) return finish(err, dm.flags, status_dev, st);
  } else if (idx != nullptr) {
    const PlanWorkspace w = carve_plan(dm, static_cast<uint8_t*>(workspace));
    int32_t* status = status_dev != nullptr ? status_dev : w.status;
    if (status_dev == nullptr && cudaMemsetAsync(w.status, 0, sizeof(int32_t), st) != cudaSuccess)
      return PR2_ERR_CUDA;
    DispatchArgs p{};
    p.idx = idx;
    p.T = dm.T;
    p.k = dm.k;
    p.N = dm.N;
    p.blk_hist = w.blk_hist;
    p.counts = w.counts;
    p.offsets = offsets;
    p.perm = perm;
    p.inv = inv;
    p.tiles = w.tiles;
    p.num_tiles = w.num_tiles;
    p.status = status;
    p.sync_ctr = w.sync_ctr;
    p.tile_rows = kMinTileRows;
    if (launch_dispatch(p, num_sms, st) != cudaSuccess) return PR2_ERR_CUDA;
    a.perm = perm;
    a.status = status;
  }
  return finish(launch_token_sort(a, num_sms, st), dm.flags, status_dev, st);
}

pr2_status pr2_token_sort_backward(const pr2_dims* dims, const void* dx, const int32_t* inv,
                                   void* dh, void* stream) {
  pr2_status s = check_tokens(dims);
  if (s != PR2_OK) return s;
  const pr2_dims& dm = *dims;
  if (dm.T == 0) return PR2_OK;
  if (dx == nullptr || inv == nullptr || dh == nullptr) return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(dx, es) || !aligned(dh, es) || !aligned(inv, 4)) return PR2_ERR_INVALID_ARG;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TokenArgs a{};
  a.T = dm.T;
  a.d = dm.d;
  a.N = dm.N;
  a.k = dm.k;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.inv = inv;
  a.src = dx;
  a.dst = dh;
  return finish(launch_token_sum(a, num_sms, st), 0u, nullptr, st);
}

pr2_status pr2_token_unsort(const pr2_dims* dims, const void* y, const float* gates,
                            const int32_t* inv, void* out, void* stream) {
  pr2_status s = check_tokens(dims);
  if (s != PR2_OK) return s;
  const pr2_dims& dm = *dims;
  if (dm.T == 0) return PR2_OK;
  if (y == nullptr || gates == nullptr || inv == nullptr || out == nullptr) return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(y, es) || !aligned(out, es) || !aligned4({gates, inv})) return PR2_ERR_INVALID_ARG;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TokenArgs a{};
  a.T = dm.T;
  a.d = dm.d;
  a.N = dm.N;
  a.k = dm.k;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.inv = inv;
  a.gates = gates;
  a.src = y;
  a.dst = out;
  return finish(launch_token_sum(a, num_sms, st), 0u, nullptr, st);
}

pr2_status pr2_token_unsort_backward(const pr2_dims* dims, const void* dout, const void* y,
                                     const float* gates, const int32_t* inv,
                                     const int32_t* offsets, void* dy, float* dgates,
                                     void* stream) {
  pr2_status s = check_tokens(dims);
  if (s != PR2_OK) return s;
  const pr2_dims& dm = *dims;
  if (dm.T == 0) return PR2_OK;
  if (dout == nullptr || y == nullptr || gates == nullptr || inv == nullptr || offsets == nullptr ||
      dy == nullptr || dgates == nullptr)
    return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(dout, es) || !aligned(y, es) || !aligned(dy, es) ||
      !aligned4({gates, inv, offsets, dgates}))
    return PR2_ERR_INVALID_ARG;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TokenArgs a{};
  a.T = dm.T;
  a.d = dm.d;
  a.N = dm.N;
  a.k = dm.k;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.inv = inv;
  a.offsets = offsets;
  a.gates = gates;
  a.src = dout;
  a.y = y;
  a.dst = dy;
  a.dgates = dgates;
  return finish(launch_token_unsort_backward(a, num_sms, st), 0u, nullptr, st);
}

pr2_status pr2_replay_gates_backward(const pr2_dims* dims, const float* probs, const int32_t* idx,
                                     const float* dgates, float* dlogits, int32_t* status_dev,
                                     void* stream) {
  pr2_status s = check_tokens(dims);
  if (s != PR2_OK) return s;
  const pr2_dims& dm = *dims;
  if ((dm.flags & PR2_F_SYNC_STATUS) && status_dev == nullptr) return PR2_ERR_INVALID_ARG;
  if (dm.T == 0) return PR2_OK;
  if (probs == nullptr || idx == nullptr || dgates == nullptr || dlogits == nullptr ||
      !aligned4({probs, idx, dgates, dlogits, status_dev}))
    return PR2_ERR_INVALID_ARG;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return finish(launch_gates_backward(probs, idx, dgates, dm.T, dm.N, dm.k,
                                      (dm.flags & PR2_F_NORMALIZE_TOPK) != 0, dlogits, status_dev,
                                      num_sms, st),
                dm.flags, status_dev, st);
}

pr2_status pr2_swiglu_checkpoint(const pr2_act_dims* dims, const void* gate, const void* up,
                                 void* act, int8_t* q, float* scale, void* stream) {
  pr2_status s = check_act(dims);
  if (s != PR2_OK) return s;
  const pr2_act_dims& dm = *dims;
  if (dm.rows == 0) return PR2_OK;
  if (gate == nullptr || up == nullptr || act == nullptr || q == nullptr || scale == nullptr)
    return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(gate, es) || !aligned(up, es) || !aligned(act, es) || !aligned(scale, 4))
    return PR2_ERR_INVALID_ARG;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ActArgs a{};
  a.rows = dm.rows;
  a.ld = dm.ld;
  a.m = dm.m;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.gate = gate;
  a.up = up;
  a.act = act;
  a.q = q;
  a.scale = scale;
  return finish(launch_swiglu_checkpoint(a, num_sms, st), 0u, nullptr, st);
}

pr2_status pr2_swiglu_checkpoint_backward(const pr2_act_dims* dims, const void* dact,
                                          const int8_t* q, const float* scale, void* dgate,
                                          void* dup, void* act, void* stream) {
  pr2_status s = check_act(dims);
  if (s != PR2_OK) return s;
  const pr2_act_dims& dm = *dims;
  if (dm.rows == 0) return PR2_OK;
  if (dact == nullptr || q == nullptr || scale == nullptr || dgate == nullptr || dup == nullptr)
    return PR2_ERR_INVALID_ARG;
  const size_t es = esize(dm.dtype);
  if (!aligned(dact, es) || !aligned(dgate, es) || !aligned(dup, es) || !aligned(act, es) ||
      !aligned(scale, 4))
    return PR2_ERR_INVALID_ARG;
  const int num_sms = num_sms_of_current_device();
  if (num_sms <= 0) return PR2_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  ActArgs a{};
  a.rows = dm.rows;
  a.ld = dm.ld;
  a.m = dm.m;
  a.bf16 = dm.dtype == PR2_BF16 ? 1 : 0;
  a.dact = dact;
  a.q = const_cast<int8_t*>(q);
  a.scale = const_cast<float*>(scale);
  a.act = act;
  a.dgate = dgate;
  a.dup = dup;
  return finish(launch_swiglu_backward(a, num_sms, st), 0u, nullptr, st);
}

}  // extern "C"
