// Rows of tokens in expert order and back, with their gradients (pr2_token_*).
//
//   sort:            x[inv[t,s]] = h[t];            backward  dh[t] = sum_s dx[inv[t,s]]
//   unsort:          out[t] = sum_s g[t,s] y[inv[t,s]]
//   unsort_backward: dy[inv[t,s]] = g[t,s] dout[t],  dg[t,s] = <dout[t], y[inv[t,s]]>
// Every kernel walks tokens: a token's row is read or written once and its k rows in the other
// order are found through inv, so nothing is written twice and the sums do not depend on the launch
// but for the split of a row over warps.  Rows past offsets[N], which no slot names, are zeroed.
// A row number outside [0, T k) is taken as an invalid slot.
//
// All of it is bound by HBM: the k expert rows, read or written once.  A warp takes a piece of a
// token's row, a lane V neighbouring columns: 16 bytes where d and the pointers allow it, else one
// element (a row of odd width starts at any element).
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kSlots = 8;  // slots handled at once; more go in further rounds

template <typename T, int V>
struct Lane;  // V elements: 16 bytes, or one
template <typename T>
struct Lane<T, 1> {
  using Raw = T;
  static __device__ __forceinline__ void unpack(const Raw& r, float (&f)[1]) { f[0] = to_f32<T>(r); }
  static __device__ __forceinline__ Raw pack(const float (&f)[1]) { return from_f32<T>(f[0]); }
  static __device__ __forceinline__ Raw zero() { return from_f32<T>(0.f); }
};
template <>
struct Lane<float, 4> {
  using Raw = uint4;
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

template <typename T, int V>
__device__ __forceinline__ void zero_rows(T* x, int from, int F, int d) {
  const int n = d / V;
  for (int r = from + blockIdx.x; r < F; r += gridDim.x)
    for (int c = threadIdx.x; c < n; c += kThreads) lanes_of<T, V>(x + static_cast<int64_t>(r) * d)[c] = Lane<T, V>::zero();
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
  if (perm != nullptr)
    for (int64_t r = used + static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; r < F;
         r += static_cast<int64_t>(gridDim.x) * kThreads)
      perm[r] = -1;
  if (x == nullptr) return;
  const int pieces = (n + 32 * U - 1) / (32 * U);
  RowWalk at(static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5), static_cast<int64_t>(gridDim.x) * kWarps,
             pieces);
  for (; at.row < Tn; at.next()) {
    const int64_t t = at.row;
    const int c0 = at.col * 32 * U + lane;
    typename L::Raw v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * 32 < n) v[u] = __ldg(lanes_of<T, V>(h + t * d) + c0 + u * 32);
    for (int s0 = 0; s0 < k; s0 += kSlots) {
      const int mine = lane < kSlots ? my_row(inv, t, k, s0 + lane, F) : -1;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
        if (r < 0) continue;
        auto* dst = lanes_of<T, V>(x + static_cast<int64_t>(r) * d);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u * 32 < n) __stcs(dst + c0 + u * 32, v[u]);
      }
    }
  }
  zero_rows<T, V>(x, used, F, d);
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
      typename L::Raw raw[kSlots][U];
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int r = __shfl_sync(0xffffffffu, mine, s);
#pragma unroll
        for (int u = 0; u < U; ++u)
          raw[s][u] = r >= 0 && c0 + u * 32 < n ? __ldcs(lanes_of<T, V>(y + static_cast<int64_t>(r) * d) + c0 + u * 32)
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
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens; t0 < Tn; t0 += static_cast<int64_t>(gridDim.x) * kTokens) {
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
          typename L::Raw raw[kSlots][U], own_raw[U];
#pragma unroll
          for (int u = 0; u < U; ++u)
            own_raw[u] = c0 + u * 32 < n ? __ldg(lanes_of<T, V>(dout + t * d) + c0 + u * 32) : L::zero();
#pragma unroll
          for (int s = 0; s < kSlots; ++s) {
            const int r = __shfl_sync(0xffffffffu, mine, s);
#pragma unroll
            for (int u = 0; u < U; ++u)
              raw[s][u] = r >= 0 && c0 + u * 32 < n
                              ? __ldcs(lanes_of<T, V>(y + static_cast<int64_t>(r) * d) + c0 + u * 32)
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
      // sum of slot s in the lanes whose bits 4, 3, 2 are s
      const float sum = warp_sum8(acc);
      const int s = (lane >> 2) & 7;
      const bool writes = (lane & 3) == 0;
      if (G == 1) {
        if (writes && s0 + s < k) dgates[t * k + s0 + s] = sum;
      } else {
        if (writes) part[warp][s] = sum;
        __syncthreads();
        if (g_warp == 0 && lane < kSlots && t < Tn && s0 + lane < k) {
          float all = 0.f;
#pragma unroll
          for (int w = 0; w < G; ++w) all += part[warp + w][lane];
          dgates[t * k + s0 + lane] = all;
        }
        __syncthreads();
      }
    }
  }
  zero_rows<T, V>(dy, rows_used(offsets, N, F), F, d);
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

template <typename T, int V, int U>
cudaError_t sort_rows(const TokenArgs& a, int num_sms, cudaStream_t st) {
  const int64_t items = a.dst != nullptr ? a.T * ((a.d / V + 32 * U - 1) / (32 * U)) : (a.T * a.k + 255) / 256;
  return launch_pdl(sort_kernel<T, V, U>, dim3(blocks_for(items, kWarps, num_sms, 16)), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.src), a.inv, a.offsets, static_cast<int>(a.T), a.d, a.N, a.k,
                    static_cast<T*>(a.dst), a.perm, a.status);
}
template <typename T, int V, int U>
cudaError_t sum_rows(const TokenArgs& a, int num_sms, cudaStream_t st) {
  const int64_t items = a.T * ((a.d / V + 32 * U - 1) / (32 * U));
  return launch_pdl(sum_kernel<T, V, U>, dim3(blocks_for(items, kWarps, num_sms, 16)), dim3(kThreads), 0, st, 1,
                    static_cast<const T*>(a.src), a.inv, a.gates, static_cast<int>(a.T), a.d, a.k,
                    static_cast<T*>(a.dst));
}
template <typename T, int V, int U, int G>
cudaError_t unsort_backward(const TokenArgs& a, int num_sms, cudaStream_t st) {
  return launch_pdl(unsort_backward_kernel<T, V, U, G>, dim3(blocks_for(a.T, kWarps / G, num_sms, 16)),
                    dim3(kThreads), 0, st, 1, static_cast<const T*>(a.src), static_cast<const T*>(a.y), a.gates,
                    a.inv, a.offsets, static_cast<int>(a.T), a.d, a.N, a.k, static_cast<T*>(a.dst), a.dgates);
}
template <typename T, int V, int U>
cudaError_t unsort_backward(const TokenArgs& a, int num_sms, cudaStream_t st) {
  // a warp a token while that fills the SMs, else a block a token
  return a.T >= static_cast<int64_t>(num_sms) * 16 ? unsort_backward<T, V, U, 1>(a, num_sms, st)
                                                   : unsort_backward<T, V, U, kWarps>(a, num_sms, st);
}

}  // namespace

cudaError_t launch_token_sort(const TokenArgs& a, int num_sms, cudaStream_t st) {
  if (a.bf16)
    return vectors(a, 2) ? sort_rows<__nv_bfloat16, 8, 2>(a, num_sms, st)
                         : sort_rows<__nv_bfloat16, 1, 8>(a, num_sms, st);
  return vectors(a, 4) ? sort_rows<float, 4, 2>(a, num_sms, st) : sort_rows<float, 1, 8>(a, num_sms, st);
}
cudaError_t launch_token_sum(const TokenArgs& a, int num_sms, cudaStream_t st) {
  if (a.bf16)
    return vectors(a, 2) ? sum_rows<__nv_bfloat16, 8, 1>(a, num_sms, st)
                         : sum_rows<__nv_bfloat16, 1, 4>(a, num_sms, st);
  return vectors(a, 4) ? sum_rows<float, 4, 1>(a, num_sms, st) : sum_rows<float, 1, 4>(a, num_sms, st);
}
cudaError_t launch_token_unsort_backward(const TokenArgs& a, int num_sms, cudaStream_t st) {
  if (a.bf16)
    return vectors(a, 2) ? unsort_backward<__nv_bfloat16, 8, 1>(a, num_sms, st)
                         : unsort_backward<__nv_bfloat16, 1, 4>(a, num_sms, st);
  return vectors(a, 4) ? unsort_backward<float, 4, 1>(a, num_sms, st) : unsort_backward<float, 1, 4>(a, num_sms, st);
}

}  // namespace pr2
