// Rows of tokens in expert order and back, with their gradients (pr2_token_*).
//
//   sort:            x[inv[t,s]] = h[t];            backward  dh[t] = sum_s dx[inv[t,s]]
//   unsort:          out[t] = sum_s g[t,s] y[inv[t,s]]
//   unsort_backward: dy[inv[t,s]] = g[t,s] dout[t],  dg[t,s] = <dout[t], y[inv[t,s]]>
// Every kernel walks tokens: a token's row is read or written once and its k rows in the other
// order are found through inv, so nothing is written twice and the sums do not depend on the launch
// but for the split of a row over warps.  Rows past offsets[N], which no slot names, are zeroed.
// A row number outside [0, T k) is taken as an invalid slot.
// The plan of up to 32768 slots is made by one cluster (plan_kernel), of up to 4 M slots by two launches
// (plan_count_kernel, plan_place_kernel), of more by the layer forward's dispatch.
//
// All of it is bound by HBM: the k expert rows, read or written once.  A warp takes a piece of a
// token's row, a lane V neighbouring columns: 16 bytes where d and the pointers allow it, else one
// fp32 element or a pair of bf16 ones (a row of odd width starts at any element, so a row's pairs
// start at its first column or at its second, whichever lies on 4 bytes).  bf16, k = 8, back to back:
// 32768 x 2048 sorted in 190 us (94 % of the copy rate), summed in 185 (96 %), unsort gradient 351 (96 %);
// 4096 x 2047 (pairs) 28, 57 and 82 us against 21, 23 and 48 for 2048 columns.
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kSlots = 8;  // slots handled at once; more go in further rounds

template <typename T, int V>
struct Lane;  // V elements: 16 bytes, or one
template <>
struct Lane<float, 1> {
  using Raw = float;
  using Held = float;  // a Raw on its way (in a register of its own)
  static __device__ __forceinline__ void unpack(Held r, float (&f)[1]) { f[0] = r; }
  static __device__ __forceinline__ Raw pack(const float (&f)[1]) { return f[0]; }
  static __device__ __forceinline__ Held load(const Raw* p) { return __ldg(p); }
  static __device__ __forceinline__ Raw raw(Held r) { return r; }
  static __device__ __forceinline__ Raw zero() { return 0.f; }
};
template <>
struct Lane<float, 4> {
  using Raw = uint4;
  using Held = uint4;
  static __device__ __forceinline__ Held load(const Raw* p) { return __ldcs(p); }
  static __device__ __forceinline__ Raw raw(const Held& r) { return r; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x);
    f[1] = __uint_as_float(r.y);
    f[2] = __uint_as_float(r.z);
    f[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ Raw pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
};
template <>
struct Lane<__nv_bfloat16, 8> {
  using Raw = uint4;
  using Held = uint4;
  static __device__ __forceinline__ Held load(const Raw* p) { return __ldcs(p); }
  static __device__ __forceinline__ Raw raw(const Held& r) { return r; }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&f)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw pack(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                      pack_bf16x2(f[6], f[7]));
  }
  static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
};
template <typename T, int V>
__device__ __forceinline__ const typename Lane<T, V>::Raw* lanes_of(const T* p) {
  return reinterpret_cast<const typename Lane<T, V>::Raw*>(p);
}
template <typename T, int V>
__device__ __forceinline__ typename Lane<T, V>::Raw* lanes_of(T* p) {
  return reinterpret_cast<typename Lane<T, V>::Raw*>(p);
}

// Row of the token's slot s0 + lane (lane < kSlots), -1 for none.
__device__ __forceinline__ int my_row(const int32_t* __restrict__ inv, int64_t t, int k, int s, int F) {
  if (s >= k) return -1;
  const int p = inv[t * k + s];
  return p < F ? p : -1;  // (negative: -1 or as bad)
}

// First row that no slot names.
__device__ __forceinline__ int rows_used(const int32_t* __restrict__ offsets, int N, int F) {
  const int n = offsets[N];
  return n < 0 ? 0 : n < F ? n : F;
}

// Rows from .. F - 1 of n Raws each.
template <typename Raw>
__device__ __forceinline__ void zero_rows(Raw* x, int from, int F, int n) {
  for (int r = from + blockIdx.x; r < F; r += gridDim.x)
    for (int c = threadIdx.x; c < n; c += kThreads) x[static_cast<int64_t>(r) * n + c] = Raw{};
}
__device__ __forceinline__ void fill_perm(int32_t* __restrict__ perm, int from, int F) {
  if (perm == nullptr) return;
  for (int64_t r = from + static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; r < F;
       r += static_cast<int64_t>(gridDim.x) * kThreads)
    perm[r] = -1;
}

// ---- the plan of a batch of up to kPlanSlots slots -----------------------------------------------------
// One cluster, S slots per thread (a thread's are 1024 apart): counts per 32 slots and expert by
// ballots, summed per block, the blocks' counts exchanged through distributed shared memory;
// then every block scans the experts' totals and places its slots in order.  No memory outside the
// cluster is waited for, so it is an ordinary launch.  Latency-bound: with k = 8 and 128 experts up to
// 8192 slots take 5.2 us a call, 16384 (two a thread) 5.9 and 32768 (four) 9.3, where the dispatch's
// cooperative launch and the clearing of its counters take 12 to 14 and the two launches below 12.0.
constexpr int kPlanThreads = 1024;
constexpr int kPlanBlocks = 8;

constexpr size_t plan_smem_bytes(int N, int S) {
  return sizeof(int) * static_cast<size_t>(N) * (32 * S + kPlanBlocks + 1);
}

// The lanes with the same e (-1 <= e < N) as this one: a ballot per bit, which takes less than a
// __match_any_sync (placing 4096 slots of a block 1 us less, counting them so 3 us).
__device__ __forceinline__ unsigned lanes_with(int e, int N) {
  unsigned same = __ballot_sync(0xffffffffu, e >= 0);
  if (e < 0) same = ~same;
  for (int bits = N - 1, b = 0; bits > 0; bits >>= 1, ++b) {
    const unsigned m = __ballot_sync(0xffffffffu, (e >> b) & 1);
    same &= (e >> b) & 1 ? m : ~m;
  }
  return same;
}

// Exclusive scan, from `sum` on, of column[0], column[stride], ... (kRows of them); returns the end.
// Sixteen are loaded before any is stored.
template <int kRows>
__device__ __forceinline__ int scan_column(int* column, int stride, int sum) {
#pragma unroll 1
  for (int w = 0; w < kRows; w += 16) {
    int c[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) c[j] = column[(w + j) * stride];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      column[(w + j) * stride] = sum;
      sum += c[j];
    }
  }
  return sum;
}

// The thread's slots f0 + i 1024: their expert, -1 if invalid.  A slot's earlier ones in its token are
// the lanes below it, or in the warp before.
template <int S>
__device__ __forceinline__ void slots_of(const int32_t* __restrict__ idx, int f0, int F, int k, int N, int (&e)[S],
                                         int32_t* __restrict__ status) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < S; ++i) e[i] = f0 + i * kPlanThreads < F ? idx[f0 + i * kPlanThreads] : -1;
#pragma unroll
  for (int i = 0; i < S; ++i) {
    const int f = f0 + i * kPlanThreads, slot = f % k, raw = e[i];
    bool bad = raw < 0 || raw >= N;
    for (int j = 1; j < k; ++j) {
      const int other = __shfl_up_sync(0xffffffffu, raw, j);
      bad |= j <= slot && j <= lane && other == raw;
    }
    if (f < F)
      for (int j = lane + 1; j <= slot; ++j) bad |= idx[f - j] == raw;
    if (f < F && bad && status != nullptr) atomicOr(status, PR2_STATUS_BAD_INDEX);
    e[i] = bad ? -1 : raw;
  }
}

template <int S>
__global__ void __launch_bounds__(kPlanThreads)
    plan_kernel(const int32_t* __restrict__ idx, int F, int k, int N, int blocks, int32_t* __restrict__ offsets,
                int32_t* __restrict__ perm, int32_t* __restrict__ inv, int32_t* __restrict__ status) {
  extern __shared__ int plan_smem[];
  int* before = plan_smem;                // [32 S][N] slots of the expert in earlier groups of 32
  int* counts = before + 32 * S * N;      // [kPlanBlocks][N]
  int* first = counts + kPlanBlocks * N;  // [N] row of the block's first slot of the expert
  __shared__ int warp_sum[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blocks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  for (int i = tid; i < 32 * S * N; i += kPlanThreads) before[i] = 0;
  if (blocks > 1) cluster_sync();  // peers write to counts
  pdl_wait();
  pdl_trigger();
  const int f0 = rank * kPlanThreads * S + tid;
  int e[S];
  unsigned same[S];
  slots_of(idx, f0, F, k, N, e, status);
#pragma unroll
  for (int i = 0; i < S; ++i) same[i] = lanes_with(e[i], N);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S; ++i)
    if (e[i] >= 0 && lane == __ffs(same[i]) - 1) before[(i * 32 + warp) * N + e[i]] = __popc(same[i]);
  __syncthreads();
  if (tid < N) {
    const int sum = scan_column<32 * S>(before + tid, N, 0);
    for (int b = 0; b < blocks; ++b) {
      const uint32_t at = smem_u32(&counts[rank * N + tid]);
      if (blocks > 1)
        asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(mapa_shared(at, b)), "r"(sum) : "memory");
      else
        counts[tid] = sum;
    }
  }
  if (blocks > 1)
    cluster_sync();
  else
    __syncthreads();
  int all = 0, mine = 0;
  if (tid < N)
    for (int b = 0; b < blocks; ++b) {
      const int c = counts[b * N + tid];
      mine += b < rank ? c : 0;
      all += c;
    }
  int scan = all;  // inclusive over the experts
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  int earlier = 0, used = 0;
  for (int w = 0; w < kMaxExperts / 32; ++w) {
    earlier += w < warp ? warp_sum[w] : 0;
    used += warp_sum[w];
  }
  if (tid < N) {
    const int off = earlier + scan - all;
    first[tid] = off + mine;
    if (rank == 0) offsets[tid] = off;
  }
  if (rank == 0 && tid == 0) offsets[N] = used;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S; ++i) {
    const int f = f0 + i * kPlanThreads;
    if (f >= F) break;
    int row = -1;
    if (e[i] >= 0) {
      row = first[e[i]] + before[(i * 32 + warp) * N + e[i]] + __popc(same[i] & lanemask_lt());
      perm[row] = f;
    }
    inv[f] = row;
    if (f >= used) perm[f] = -1;
  }
}

// ---- the plan of larger batches -------------------------------------------------------------------------
// Blocks of kLargeSlots slots: one launch counts each block's slots per expert, the next adds up all
// blocks' counts, and the earlier blocks' apart, and places its own.  T = 32768, k = 8, N = 128: 12.7 us a
// call, the dispatch's one cooperative launch with a grid barrier 21.
constexpr int kLargeMost = 4;  // slots per thread
constexpr int kLargeSlots = kPlanThreads * kLargeMost;

__global__ void __launch_bounds__(kPlanThreads)
    plan_count_kernel(const int32_t* __restrict__ idx, int F, int k, int N, int32_t* __restrict__ hist,
                      int32_t* __restrict__ status) {
  __shared__ int sum[kMaxExperts];
  if (threadIdx.x < kMaxExperts) sum[threadIdx.x] = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  int e[kLargeMost];
  slots_of(idx, static_cast<int>(blockIdx.x) * kLargeSlots + static_cast<int>(threadIdx.x), F, k, N, e, status);
#pragma unroll
  for (int i = 0; i < kLargeMost; ++i)
    if (e[i] >= 0) atomicAdd(&sum[e[i]], 1);
  __syncthreads();
  if (static_cast<int>(threadIdx.x) < N) hist[static_cast<int64_t>(blockIdx.x) * N + threadIdx.x] = sum[threadIdx.x];
}

__global__ void __launch_bounds__(kPlanThreads)
    plan_place_kernel(const int32_t* __restrict__ idx, int F, int k, int N, const int32_t* __restrict__ hist,
                      int32_t* __restrict__ offsets, int32_t* __restrict__ perm, int32_t* __restrict__ inv) {
  extern __shared__ int plan_smem[];
  int* before = plan_smem;                        // [32 kLargeMost][N]
  int* total = before + 32 * kLargeMost * N;      // [N] slots of the expert in all blocks
  int* earlier = total + N;                       // [N] in earlier blocks; then the row of the block's first
  __shared__ int warp_sum[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x, blocks = gridDim.x;
  for (int i = tid; i < (32 * kLargeMost + 2) * N; i += kPlanThreads) before[i] = 0;
  pdl_wait();
  pdl_trigger();
  const int f0 = rank * kLargeSlots + tid;
  int e[kLargeMost];
  unsigned same[kLargeMost];
  slots_of(idx, f0, F, k, N, e, nullptr);
#pragma unroll
  for (int i = 0; i < kLargeMost; ++i) same[i] = lanes_with(e[i], N);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kLargeMost; ++i)
    if (e[i] >= 0 && lane == __ffs(same[i]) - 1) before[(i * 32 + warp) * N + e[i]] = __popc(same[i]);
  // blocks' counts: thread (p, n) takes expert n of every parts-th block
  const int parts = kPlanThreads / N, p = tid / N, n = tid - p * N;
  if (p < parts) {
    int all = 0, mine = 0;
#pragma unroll 4
    for (int b = p; b < blocks; b += parts) {
      const int c = hist[static_cast<int64_t>(b) * N + n];
      all += c;
      mine += b < rank ? c : 0;
    }
    atomicAdd(&total[n], all);
    atomicAdd(&earlier[n], mine);
  }
  __syncthreads();
  const int all = tid < N ? total[tid] : 0;
  int scan = all;  // inclusive over the experts
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  int below = 0, used = 0;
  for (int w = 0; w < kMaxExperts / 32; ++w) {
    below += w < warp ? warp_sum[w] : 0;
    used += warp_sum[w];
  }
  if (tid < N) {
    const int off = below + scan - all;
    if (rank == 0) offsets[tid] = off;
    scan_column<32 * kLargeMost>(before + tid, N, off + earlier[tid]);
  }
  if (rank == 0 && tid == 0) offsets[N] = used;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kLargeMost; ++i) {
    const int f = f0 + i * kPlanThreads;
    if (f >= F) break;
    int row = -1;
    if (e[i] >= 0) {
      row = before[(i * 32 + warp) * N + e[i]] + __popc(same[i] & lanemask_lt());
      perm[row] = f;
    }
    inv[f] = row;
    if (f >= used) perm[f] = -1;
  }
}

template <int S>
cudaError_t run_plan(const int32_t* idx, int F, int k, int N, int32_t* offsets, int32_t* perm, int32_t* inv,
                     int32_t* status, cudaStream_t st) {
  int blocks = 1;
  while (blocks * kPlanThreads * S < F) blocks *= 2;
  constexpr size_t most = plan_smem_bytes(kMaxExperts, S);  // the kernel's limit, whatever N
  if (most + 1024 > 48 * 1024) {
    const cudaError_t err = cudaFuncSetAttribute(plan_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(most));
    if (err != cudaSuccess) return err;
  }
  return launch_pdl(plan_kernel<S>, dim3(blocks), dim3(kPlanThreads), plan_smem_bytes(N, S), st, blocks, idx, F, k, N,
                    blocks, offsets, perm, inv, status);
}

// ---- sort: a warp per (token, U lanes' worth of its columns) ---------------------------------------
template <typename T, int V, int U>
__global__ void __launch_bounds__(kThreads)
    sort_kernel(const T* __restrict__ h, const int32_t* __restrict__ inv,
                const int32_t* __restrict__ offsets, int Tn, int d, int N, int k, T* __restrict__ x,
                int32_t* __restrict__ perm, const int32_t* status) {
  using L = Lane<T, V>;
  pdl_wait();
  pdl_trigger();
  if (status_timed_out(status)) return;  // dispatch gave up: its tables may be unwritten
  const int F = Tn * k, lane = threadIdx.x & 31, n = d / V;
  const int used = rows_used(offsets, N, F);
  fill_perm(perm, used, F);
  if (x == nullptr) return;  // the plan alone
  const int pieces = (n + 32 * U - 1) / (32 * U);
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x) * kWarps,
             pieces);
  for (; at.row < Tn; at.next()) {
    const int64_t t = at.row;
    const int c0 = at.col * 32 * U + lane;
    typename L::Held v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * 32 < n) v[u] = L::load(lanes_of<T, V>(h + t * d) + c0 + u * 32);
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const int mine = lane < kSlots ? my_row(inv, t, k, s0 + lane, F) : -1;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
        if (r < 0) continue;
        auto* dst = lanes_of<T, V>(x + static_cast<int64_t>(r) * d);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u * 32 < n) __stcs(dst + c0 + u * 32, L::raw(v[u]));
      }
    }
  }
  zero_rows(lanes_of<T, V>(x), used, F, n);
}

// ---- sums of a token's rows (unsort; sort_backward: gates NULL, all 1) ------------------------------
template <typename T, int V, int U>
__global__ void __launch_bounds__(kThreads)
    sum_kernel(const T* __restrict__ y, const int32_t* __restrict__ inv, const float* __restrict__ gates,
               int Tn, int d, int k, T* __restrict__ out) {
  using L = Lane<T, V>;
  pdl_wait();
  pdl_trigger();
  const int F = Tn * k, lane = threadIdx.x & 31, n = d / V;
  const int pieces = (n + 32 * U - 1) / (32 * U);
  // (a division an item: its operands take fewer registers than a running row and column, and the loads
  // in flight need them)
  const int64_t items = static_cast<int64_t>(Tn) * pieces;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); i < items;
       i += static_cast<int64_t>(gridDim.x) * kWarps) {
    const int64_t t = i / pieces;
    const int c0 = static_cast<int>(i - t * pieces) * 32 * U + lane;
    float acc[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) acc[u][j] = 0.f;
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const int mine = lane < kSlots ? my_row(inv, t, k, s0 + lane, F) : -1;
      const float my_g = lane < kSlots && s0 + lane < k && gates != nullptr ? gates[t * k + s0 + lane] : 1.f;
      typename L::Held raw[kSlots][U];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
#pragma unroll
        for (int u = 0; u < U; ++u)
          raw[s][u] = r >= 0 && c0 + u * 32 < n ? L::load(lanes_of<T, V>(y + static_cast<int64_t>(r) * d) + c0 + u * 32)
                                                : L::zero();
      }
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
        const float g = __shfl_sync(0xffffffffu, my_g, s);
        if (r < 0) continue;  // (its gate may hold anything)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[V];
          L::unpack(raw[s][u], f);
#pragma unroll
          for (int j = 0; j < V; ++j) acc[u][j] = fmaf(g, f[j], acc[u][j]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * 32 < n) lanes_of<T, V>(out + t * d)[c0 + u * 32] = L::pack(acc[u]);
  }
}

// Gates' gradients of a token's slots s0 .. s0 + 7 from its G warps' partial sums (every thread of the
// block calls this if G > 1).
template <int G>
__device__ __forceinline__ void write_gate_grads(const float (&acc)[kSlots], int64_t t, bool valid, int s0, int k,
                                                 float (*part)[kSlots], float* __restrict__ dgates) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float sum = warp_sum8(acc);  // of slot s in the lanes whose bits 4, 3, 2 are s
  const int s = lane >> 2;
  if (G == 1) {
    if ((lane & 3) == 0 && s0 + s < k) dgates[t * k + s0 + s] = sum;
    return;
  }
  if ((lane & 3) == 0) part[warp][s] = sum;
  __syncthreads();
  if (warp % G == 0 && lane < kSlots && valid && s0 + lane < k) {
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < G; ++w) all += part[warp + w][lane];
    dgates[t * k + s0 + lane] = all;
  }
  __syncthreads();
}

// ---- unsort_backward: G warps a token -----------------------------------------------------------------
template <typename T, int V, int U, int G>
__global__ void __launch_bounds__(kThreads)
    unsort_backward_kernel(const T* __restrict__ dout, const T* __restrict__ y,
                           const float* __restrict__ gates, const int32_t* __restrict__ inv,
                           const int32_t* __restrict__ offsets, int Tn, int d, int N, int k,
                           T* __restrict__ dy, float* __restrict__ dgates) {
  using L = Lane<T, V>;
  __shared__ float part[kWarps][kSlots];
  pdl_wait();
  pdl_trigger();
  const int F = Tn * k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = d / V;
  constexpr int kTokens = kWarps / G;  // of a block at once
  const int g_warp = warp % G;
  // (whole blocks go round together: with G > 1 they meet at a barrier)
  const int64_t step = static_cast<int64_t>(gridDim.x) * kTokens;
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens; t0 < Tn; t0 += step) {
    const int64_t t = t0 + warp / G;
    if (G == 1 && t >= Tn) break;
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const bool own = lane < kSlots && t < Tn;
      const int mine = own ? my_row(inv, t, k, s0 + lane, F) : -1;
      const float my_g = own && s0 + lane < k ? gates[t * k + s0 + lane] : 0.f;
      float acc[kSlots];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) acc[s] = 0.f;
      if (t < Tn)
        for (int c0 = g_warp * 32 * U + lane; c0 - lane < n; c0 += G * 32 * U) {
          typename L::Held raw[kSlots][U], own_raw[U];
#pragma unroll
          for (int u = 0; u < U; ++u)
            own_raw[u] = c0 + u * 32 < n ? L::load(lanes_of<T, V>(dout + t * d) + c0 + u * 32) : L::zero();
#pragma unroll
          for (int s = 0; s < kSlots; ++s) {
            const int r = __shfl_sync(0xffffffffu, mine, s);
#pragma unroll
            for (int u = 0; u < U; ++u)
              raw[s][u] = r >= 0 && c0 + u * 32 < n
                              ? L::load(lanes_of<T, V>(y + static_cast<int64_t>(r) * d) + c0 + u * 32)
                              : L::zero();
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float a[V];
            L::unpack(own_raw[u], a);
#pragma unroll
            for (int s = 0; s < kSlots; ++s) {
              const int r = __shfl_sync(0xffffffffu, mine, s);
              const float g = __shfl_sync(0xffffffffu, my_g, s);
              if (r < 0) continue;
              float f[V];
              L::unpack(raw[s][u], f);
#pragma unroll
              for (int j = 0; j < V; ++j) {
                acc[s] = fmaf(a[j], f[j], acc[s]);
                f[j] = g * a[j];
              }
              if (c0 + u * 32 < n) __stcs(lanes_of<T, V>(dy + static_cast<int64_t>(r) * d) + c0 + u * 32, L::pack(f));
            }
          }
        }
      write_gate_grads<G>(acc, t, t < Tn, s0, k, part, dgates);
    }
  }
  zero_rows(lanes_of<T, V>(dy), rows_used(offsets, N, F), F, n);
}

// ---- bf16 rows of any alignment: pairs of columns ---------------------------------------------------
using bf16 = __nv_bfloat16;

// 1 if the row's pairs on 4 bytes are the columns (2 j - 1, 2 j), 0 if (2 j, 2 j + 1).
__device__ __forceinline__ int row_parity(const bf16* row) {
  return static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 1) & 1;
}
// Columns c and c + 1; those outside [0, d) read as 0 and are not written.
__device__ __forceinline__ uint32_t load_pair(const bf16* row, int c, int d) {
  const auto* p = reinterpret_cast<const uint16_t*>(row) + c;
  if (c >= 0 && c + 1 < d && (reinterpret_cast<uintptr_t>(p) & 3u) == 0)
    return __ldg(reinterpret_cast<const uint32_t*>(p));
  const uint32_t lo = c >= 0 && c < d ? __ldg(p) : 0u, hi = c + 1 >= 0 && c + 1 < d ? __ldg(p + 1) : 0u;
  return lo | hi << 16;
}
__device__ __forceinline__ void store_pair(bf16* row, int c, int d, uint32_t v) {
  auto* p = reinterpret_cast<uint16_t*>(row) + c;
  if (c >= 0 && c + 1 < d && (reinterpret_cast<uintptr_t>(p) & 3u) == 0) {
    __stcs(reinterpret_cast<uint32_t*>(p), v);
    return;
  }
  if (c >= 0 && c < d) p[0] = static_cast<uint16_t>(v);
  if (c + 1 >= 0 && c + 1 < d) p[1] = static_cast<uint16_t>(v >> 16);
}
__device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
// Pairs of a row, either way they start.
__host__ __device__ __forceinline__ int pairs_of(int d) { return d / 2 + 1; }
// A token's columns 2 j - 1 .. 2 j + 1, for pairs of either parity.
struct Three {
  uint32_t even, odd;  // (2 j, 2 j + 1), (2 j - 1, 2 j)
  __device__ __forceinline__ void load(const bf16* row, int j, int d) {
    even = load_pair(row, 2 * j, d);
    const auto* p = reinterpret_cast<const uint16_t*>(row);
    odd = (j > 0 && 2 * j - 1 < d ? __ldg(p + 2 * j - 1) : 0u) | even << 16;
  }
};

template <int U>
__global__ void __launch_bounds__(kThreads)
    sort_pairs_kernel(const bf16* __restrict__ h, const int32_t* __restrict__ inv,
                      const int32_t* __restrict__ offsets, int Tn, int d, int N, int k, bf16* __restrict__ x,
                      int32_t* __restrict__ perm, const int32_t* status) {
  pdl_wait();
  pdl_trigger();
  if (status_timed_out(status)) return;
  const int F = Tn * k, lane = threadIdx.x & 31;
  const int used = rows_used(offsets, N, F);
  fill_perm(perm, used, F);
  if (x == nullptr) return;  // the plan alone
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x) * kWarps,
             (pairs_of(d) + 32 * U - 1) / (32 * U));
  for (; at.row < Tn; at.next()) {
    const int64_t t = at.row;
    const int j0 = at.col * 32 * U + lane;
    Three v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].load(h + t * d, j0 + u * 32, d);
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const int mine = lane < kSlots ? my_row(inv, t, k, s0 + lane, F) : -1;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
        if (r < 0) continue;
        bf16* dst = x + static_cast<int64_t>(r) * d;
        const int p = row_parity(dst);
#pragma unroll
        for (int u = 0; u < U; ++u) store_pair(dst, 2 * (j0 + u * 32) - p, d, p != 0 ? v[u].odd : v[u].even);
      }
    }
  }
  zero_rows(reinterpret_cast<uint16_t*>(x), used, F, d);
}

template <int U>
__global__ void __launch_bounds__(kThreads)
    sum_pairs_kernel(const bf16* __restrict__ y, const int32_t* __restrict__ inv, const float* __restrict__ gates,
                     int Tn, int d, int k, bf16* __restrict__ out) {
  pdl_wait();
  pdl_trigger();
  const int F = Tn * k, lane = threadIdx.x & 31;
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x) * kWarps,
             (pairs_of(d) + 32 * U - 1) / (32 * U));
  for (; at.row < Tn; at.next()) {
    const int64_t t = at.row;
    bf16* dst = out + t * d;
    const int parity = row_parity(dst), c0 = 2 * (at.col * 32 * U + lane) - parity;
    float acc[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) acc[u][0] = acc[u][1] = 0.f;
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const int mine = lane < kSlots ? my_row(inv, t, k, s0 + lane, F) : -1;
      const float my_g = lane < kSlots && s0 + lane < k && gates != nullptr ? gates[t * k + s0 + lane] : 1.f;
      // A row whose pairs start one column off the output's is loaded from a column earlier, and a pair
      // put together from a lane's upper half and the next lane's lower one; the last lane loads one more.
      uint32_t raw[kSlots][U], more[kSlots];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
        const bf16* row = y + static_cast<int64_t>(r) * d;
        const int off = row_parity(row) ^ parity;
#pragma unroll
        for (int u = 0; u < U; ++u) raw[s][u] = r >= 0 ? load_pair(row, c0 + u * 64 - off, d) : 0u;
        more[s] = r >= 0 && off != 0 && lane == 31 ? load_pair(row, c0 + (U - 1) * 64 + 1, d) : 0u;
      }
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
        const float g = __shfl_sync(0xffffffffu, my_g, s);
        if (r < 0) continue;  // (its gate may hold anything)
        if ((row_parity(y + static_cast<int64_t>(r) * d) ^ parity) != 0) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const uint32_t first = u + 1 < U ? __shfl_sync(0xffffffffu, raw[s][u + 1 < U ? u + 1 : u], 0) : more[s];
            uint32_t next = __shfl_down_sync(0xffffffffu, raw[s][u], 1);
            if (lane == 31) next = first;
            raw[s][u] = __byte_perm(raw[s][u], next, 0x5432);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          acc[u][0] = fmaf(g, low(raw[s][u]), acc[u][0]);
          acc[u][1] = fmaf(g, high(raw[s][u]), acc[u][1]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) store_pair(dst, c0 + u * 64, d, pack_bf16x2(acc[u][0], acc[u][1]));
  }
}

template <int U, int G>
__global__ void __launch_bounds__(kThreads)
    unsort_backward_pairs_kernel(const bf16* __restrict__ dout, const bf16* __restrict__ y,
                                 const float* __restrict__ gates, const int32_t* __restrict__ inv,
                                 const int32_t* __restrict__ offsets, int Tn, int d, int N, int k,
                                 bf16* __restrict__ dy, float* __restrict__ dgates) {
  __shared__ float part[kWarps][kSlots];
  pdl_wait();
  pdl_trigger();
  const int F = Tn * k, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = pairs_of(d);
  constexpr int kTokens = kWarps / G;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kTokens;
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens; t0 < Tn; t0 += step) {
    const int64_t t = t0 + warp / G;
    if (G == 1 && t >= Tn) break;
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const bool own = lane < kSlots && t < Tn;
      const int mine = own ? my_row(inv, t, k, s0 + lane, F) : -1;
      const float my_g = own && s0 + lane < k ? gates[t * k + s0 + lane] : 0.f;
      float acc[kSlots];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) acc[s] = 0.f;
      if (t < Tn)
        for (int j0 = warp % G * 32 * U + lane; j0 - lane < n; j0 += G * 32 * U) {
          uint32_t raw[kSlots][U];
          Three v[U];
#pragma unroll
          for (int u = 0; u < U; ++u) v[u].load(dout + t * d, j0 + u * 32, d);
#pragma unroll
          for (int s = 0; s < kSlots; ++s) {
            const int r = __shfl_sync(0xffffffffu, mine, s);
            const bf16* row = y + static_cast<int64_t>(r) * d;
#pragma unroll
            for (int u = 0; u < U; ++u)
              raw[s][u] = r >= 0 ? load_pair(row, 2 * (j0 + u * 32) - row_parity(row), d) : 0u;
          }
#pragma unroll
          for (int s = 0; s < kSlots; ++s) {
            const int r = __shfl_sync(0xffffffffu, mine, s);
            const float g = __shfl_sync(0xffffffffu, my_g, s);
            if (r < 0) continue;
            const int p = row_parity(y + static_cast<int64_t>(r) * d);
            bf16* dst = dy + static_cast<int64_t>(r) * d;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const uint32_t a = p != 0 ? v[u].odd : v[u].even;
              acc[s] = fmaf(low(a), low(raw[s][u]), acc[s]);
              acc[s] = fmaf(high(a), high(raw[s][u]), acc[s]);
              store_pair(dst, 2 * (j0 + u * 32) - p, d, pack_bf16x2(g * low(a), g * high(a)));
            }
          }
        }
      write_gate_grads<G>(acc, t, t < Tn, s0, k, part, dgates);
    }
  }
  zero_rows(reinterpret_cast<uint16_t*>(dy), rows_used(offsets, N, F), F, d);
}

// ---- host ---------------------------------------------------------------------------------------------
unsigned blocks_for(int64_t items, int per_block, int num_sms, int per_sm) {
  const int64_t want = (items + per_block - 1) / per_block, cap = static_cast<int64_t>(num_sms) * per_sm;
  return static_cast<unsigned>(want < 1 ? 1 : want < cap ? want : cap);
}

bool vectors(const TokenArgs& a, int es) {
  const uintptr_t all = reinterpret_cast<uintptr_t>(a.src) | reinterpret_cast<uintptr_t>(a.y) |
                        reinterpret_cast<uintptr_t>(a.dst);
  return (all & 15u) == 0 && static_cast<int64_t>(a.d) * es % 16 == 0;
}

dim3 item_grid(int64_t rows, int units, int U, int num_sms) {
  return dim3(blocks_for(rows * ((units + 32 * U - 1) / (32 * U)), kWarps, num_sms, 16));
}

template <typename T, int V, int U>
cudaError_t sort_rows(const TokenArgs& a, int num_sms, cudaStream_t st) {
  const dim3 grid = a.dst != nullptr ? item_grid(a.T, a.d / V, U, num_sms)
                                     : dim3(blocks_for(a.T * a.k, kThreads, num_sms, 16));
  return launch_pdl(sort_kernel<T, V, U>, grid, dim3(kThreads), 0, st, 1, static_cast<const T*>(a.src), a.inv,
                    a.offsets, static_cast<int>(a.T), a.d, a.N, a.k, static_cast<T*>(a.dst), a.perm, a.status);
}
template <typename T, int V, int U>
cudaError_t sum_rows(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return launch_pdl(sum_kernel<T, V, U>, item_grid(a.T, a.d / V, U, num_sms), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.src), a.inv, a.gates, static_cast<int>(a.T), a.d, a.k,
                    static_cast<T*>(a.dst));
}

// unsort_backward: a block a token for few tokens, and for tokens of much work (eight pieces of a row for
// each warp) while a warp a token would leave the SMs unevenly filled; else a warp a token.  us with a warp / a
// block, "=" where the rule takes the slower one:
//   bf16, k = 8  2048 columns 4096 60.1 / 47.3, 9728 (the switch) 111 / 112, 12000 139 / 136 =, 32768 352 / 374;
//                7168 columns 8192 340 / 320, 9728 372 / 382, 12000 474 / 465 =, 32768 1219 / 1274;
//                512 columns 4096 14.0 / 26.1; 2047 columns 1000 38 / 18, 8192 154 / 159 =, 9728 170 / 187
//   bf16, k = 2  2048 columns 200 8.4 / 4.6, 304 (the switch) 8.3 / 4.5 =, 1000 8.4 / 6.8 =, 8192 40 / 45;
//                7168 columns 1000 32 / 17 =, 4096 81 / 64 =, 9728 136 / 154
//   fp32, k = 8  4096 columns 4096 208 / 169, 9728 409 / 408, 16384 685 / 681;
//                1023 columns 1000 26.6 / 13.8, 4096 69 / 76 =, 9728 155 / 170
//   fp32, k = 2  4096 columns 8192 139 / 113, 9728 148 / 132 =, 32768 463 / 434 =; 1024 columns 1000 8.8 / 5.7 =,
//                9728 41 / 44
template <typename T>
cudaError_t launch_unsort_backward(void (*warps)(const T*, const T*, const float*, const int32_t*, const int32_t*, int,
                                                 int, int, int, T*, float*),
                                   void (*blocks)(const T*, const T*, const float*, const int32_t*, const int32_t*, int,
                                                  int, int, int, T*, float*),
                                   int pieces, const TokenArgs& a, int num_sms, cudaStream_t st) {
  const bool many = a.T >= static_cast<int64_t>(num_sms) * (pieces * a.k >= kWarps * 8 ? 64 : 2);
  return launch_pdl(many ? warps : blocks, dim3(blocks_for(a.T, many ? kWarps : 1, num_sms, 16)), dim3(kThreads), 0, st,
                    1, static_cast<const T*>(a.src), static_cast<const T*>(a.y), a.gates, a.inv, a.offsets,
                    static_cast<int>(a.T), a.d, a.N, a.k, static_cast<T*>(a.dst), a.dgates);
}

}  // namespace

cudaError_t launch_token_plan(const int32_t* idx, int F, int k, int N, int32_t* hist, int32_t* offsets,
                              int32_t* perm, int32_t* inv, int32_t* status, cudaStream_t st) {
  if (F <= kPlanThreads * kPlanBlocks) return run_plan<1>(idx, F, k, N, offsets, perm, inv, status, st);
  if (F <= kPlanThreads * kPlanBlocks * 2) return run_plan<2>(idx, F, k, N, offsets, perm, inv, status, st);
  if (F <= kPlanThreads * kPlanBlocks * 4) return run_plan<4>(idx, F, k, N, offsets, perm, inv, status, st);
  const dim3 grid((F + kLargeSlots - 1) / kLargeSlots);
  auto smem = [](int experts) { return sizeof(int) * static_cast<size_t>(experts) * (32 * kLargeMost + 2); };
  cudaError_t err = cudaFuncSetAttribute(plan_place_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(smem(kMaxExperts)));
  if (err == cudaSuccess)
    err = launch_pdl(plan_count_kernel, grid, dim3(kPlanThreads), 0, st, 1, idx, F, k, N, hist, status);
  if (err != cudaSuccess) return err;
  return launch_pdl(plan_place_kernel, grid, dim3(kPlanThreads), smem(N), st, 1, idx, F, k, N,
                    static_cast<const int32_t*>(hist), offsets, perm, inv);
}

cudaError_t launch_token_sort(const TokenArgs& a, int num_sms, cudaStream_t st) {
  if (!a.bf16) return vectors(a, 4) ? sort_rows<float, 4, 2>(a, num_sms, st) : sort_rows<float, 1, 8>(a, num_sms, st);
  if (vectors(a, 2)) return sort_rows<bf16, 8, 2>(a, num_sms, st);
  constexpr int U = 4;
  const dim3 grid = a.dst != nullptr ? item_grid(a.T, pairs_of(a.d), U, num_sms)
                                     : dim3(blocks_for(a.T * a.k, kThreads, num_sms, 16));
  return launch_pdl(sort_pairs_kernel<U>, grid, dim3(kThreads), 0, st, 1, static_cast<const bf16*>(a.src), a.inv,
                    a.offsets, static_cast<int>(a.T), a.d, a.N, a.k, static_cast<bf16*>(a.dst), a.perm, a.status);
}
cudaError_t launch_token_sum(const TokenArgs& a, int num_sms, cudaStream_t st) {
  if (!a.bf16) return vectors(a, 4) ? sum_rows<float, 4, 1>(a, num_sms, st) : sum_rows<float, 1, 2>(a, num_sms, st);
  if (vectors(a, 2)) return sum_rows<bf16, 8, 1>(a, num_sms, st);
  // four pairs a lane unless that leaves most lanes of a narrow row without one (k = 8, d = 2047: 57 us
  // with four, 68 with two; k = 2, d = 65: 21 and 14)
  const bool wide = pairs_of(a.d) > 64;
  return launch_pdl(wide ? sum_pairs_kernel<4> : sum_pairs_kernel<2>,
                    item_grid(a.T, pairs_of(a.d), wide ? 4 : 2, num_sms), dim3(kThreads), 0, st, 1,
                    static_cast<const bf16*>(a.src), a.inv, a.gates, static_cast<int>(a.T), a.d, a.k,
                    static_cast<bf16*>(a.dst));
}
cudaError_t launch_token_unsort_backward(const TokenArgs& a, int num_sms, cudaStream_t st) {
  if (!a.bf16)
    return vectors(a, 4) ? launch_unsort_backward<float>(unsort_backward_kernel<float, 4, 1, 1>,
                                                         unsort_backward_kernel<float, 4, 1, kWarps>, a.d / 128, a,
                                                         num_sms, st)
                         : launch_unsort_backward<float>(unsort_backward_kernel<float, 1, 2, 1>,
                                                         unsort_backward_kernel<float, 1, 2, kWarps>, a.d / 64, a,
                                                         num_sms, st);
  return vectors(a, 2) ? launch_unsort_backward<bf16>(unsort_backward_kernel<bf16, 8, 1, 1>,
                                                      unsort_backward_kernel<bf16, 8, 1, kWarps>, a.d / 256, a,
                                                      num_sms, st)
                       : launch_unsort_backward<bf16>(unsort_backward_pairs_kernel<2, 1>,
                                                      unsort_backward_pairs_kernel<2, kWarps>, a.d / 128, a, num_sms,
                                                      st);
}

}  // namespace pr2
