// Products of rows sorted by expert with the experts' matrices on the tcgen05 tensor cores: forward
// (bf16, or e4m3 with scales), gradient of the rows, gradient of the matrices.  fp32 accumulation.
//
//   forward  D[o, r] = sum_i W[o, i] x[r, i]       A = W,    both K-major
//   rows     D[i, r] = sum_o W[o, i] dy[r, o]      A = W^T,  MN-major; dy K-major
//   weight   D[o, i] = sum_r dy[r, o] x[r, i]      A = dy^T, B = x^T, both MN-major
// The operands stay as memory has them: which of a matrix's two orders the tensor core reads is a bit of
// its descriptor, so no transposed copy is made.
//
// A pair of CTAs computes 256 x 256 of D: each holds 128 rows of A and half of B in its shared memory
// and 128 x 256 of D in its tensor memory, 32 KB of operands for 512 clk of MMA where one CTA alone
// needs 48 KB (128 x 256) or has no room for a second accumulator (256 x 256).  The second accumulator
// lets the epilogue of a tile overlap the MMAs of the next one.  Tiles of rows are N, a multiple of 32, so an
// expert of few rows costs few MMAs and its matrix is read once a tile: of up to 256 rows, or of up to 384 in
// both accumulators without that overlap, where the expert has no more (see Plan).
//
// Warp roles: 0 TMA of A, 1 MMA (of the first CTA) and tensor memory, then (see Roles) TMA of B, epilogue, scheduler
// and loaders, where there is something that TMA cannot bring: operands that do not start on 16 bytes (sixteen
// warps); the zeros behind the last rows of an expert, which the gradient of the matrices must not mix with
// the next expert's (four).  Every wait is bounded (pr2_device.cuh).
//
// The tensor core adds to its fp32 accumulator by cutting bits off, so the error of a long sum grows with
// its length and to one side (terms of any sign, 8192 rows: 9e-6 of the norm, 512: 5e-7, fp32 FMAs in turn 3e-7; terms
// of one sign, 8192: 3.5e-5).  Results in fp32 therefore leave the accumulator every kMostMmas MMAs and are added up,
// rounded, where they are stored, by the thread or the copies of the warp that stored them before; results in 16
// bits every kLongMmas, in tensor memory.
//
// fp32 operands: each value is a sum of three bf16 values (24 bits), and eight of the nine products of their
// planes, the first in an accumulator of its own, give the product to 2^-32 (see split3).
//
// The launch has a pair for every job.  A pair that runs takes further jobs over from pairs that have not
// started (cluster launch control), so that the pairs end at about the same time whatever the experts'
// sizes, without a counter in memory.  The scheduler warps turn a pair's number into a job, once for all
// roles.  Gradient of the matrices: experts of most and of fewest rows in turn.  Forward and rows: as they are
// numbered, because jobs of one tile an expert wait for HBM and those of two for L2, and go better side by side (4096
// tokens, N = 128, k = 8: forward 226 us longest first, 214 as numbered).
#include <cudaTypedefs.h>

#include <type_traits>
#include <utility>

#include "group_plan.cuh"
#include "pr2_device.cuh"
#include "pr2_internal.h"

namespace pr2 {
namespace {

constexpr int kWarpMma = 1;
constexpr int kEpiWarps = 8;
constexpr int kAskAhead = 6;                    // K blocks before a job's end at which the next is taken
constexpr int kJobs = 8;                         // jobs between the scheduler and the last role
// What the loader warps do, and how many there are.
enum : int { kNoLoad = 0, kZeros = 1, kLoad = 2 };
enum : int { kBf16 = 0, kE4m3 = 1, kFp32 = 2 };  // types of rows and matrices; fp32: three bf16 planes each (split3)
template <int kLoaders>
constexpr int kLoadWarps = kLoaders == kLoad ? 16 : kLoaders == kZeros ? 4 : 0;
// Which warps do what.  Gradient of matrices whose operands TMA brings: the sums of an expert's rows stay in
// registers of the epilogue's two warpgroups (kKeep), which take them over from the other two.
template <int kOp, int kType, int kLoaders>
struct Roles {
  static constexpr bool kKeep = kOp == kGroupWeight && kLoaders == kZeros;
  static constexpr int kTmaB = kKeep ? 3 : 2;  // brings B, warp 0 A
  static constexpr int kEpi0 = kKeep ? 8 : 3, kSched = kKeep ? 2 : 11, kLoad0 = kKeep ? 4 : 12;
  static constexpr int kThreads = 32 * (kKeep ? 16 : kLoad0 + kLoadWarps<kLoaders>);
};
constexpr int kKeepThreads = 512, kKeepRegs = 128;        // at launch: all of an SM's registers
constexpr int kKeepEpiRegs = 200, kKeepOtherRegs = 56;    // then, in halves of the block
static_assert((kKeepEpiRegs + kKeepOtherRegs) * (kKeepThreads / 2) <= kKeepThreads * kKeepRegs, "registers");
constexpr int kHalf = 128 * 128;                // bytes of an operand's 128 rows of 128 bytes
constexpr uint32_t kTmemCols = 512, kAccCols = 256;
constexpr int kOutPitch = 128 * 2 + 16;         // forward, rows: 16 rows x 128 bf16, distinct banks
constexpr int kOutBuf = 16 * kOutPitch;
constexpr int kStoreBuf = 32 * 64;              // weight: 32 x 16 fp32 of a warp, two of them
constexpr int kMaxStages = 6;
constexpr int kRawPitch = 144;                  // 128 bytes from anywhere in a 16-byte word: nine such words
// MMAs in turn that a result in fp32 takes from one accumulator: of 16-bit operands 48 (relative error 7e-7; 32: 5e-7 and
// an eighth more time for gradients of matrices of many rows); of fp32 ones, whose results should be as close as those
// of fp32 FMAs, 16 (2.4e-7, FMAs 2.8e-7; 32: 4.8e-7 and 2 to 11 % less time); 16 where registers keep the sums.
constexpr int kMostMmas = 48, kExactMmas = 16, kKeepMmas = 16;
// And that a result in 16 bits takes (16384 bf16 or 32768 e4m3 columns): 8e-5 of a sum of terms of one sign, 4 % of half
// a step.  Longer sums (to one side 8e-4 at 131072 columns, 7e-3 at 2^20, where no value was rounded right) use one
// accumulator and add it every so many MMAs to their sums in the other, whose epilogue then overlaps nothing (8192
// rows, 8 matrices of 2048 x 32768: 681 us, without it 664; of 2048 x 16448 357, 343).
constexpr int kLongMmas = 1024;

// e4m3: K blocks (4096 columns) from which on up to 384 rows of an expert are one tile (see Plan)
constexpr int kWideBlocks = 32;

constexpr int kPlanBytes = 4;  // an expert: place in the order, or jobs before it

template <int kOp, int kType, int kLoaders>
struct Layout {
  static constexpr bool kSplit = kType == kFp32;
  static constexpr int kPlanes = kSplit ? 3 : 1;
  static constexpr int kEs = kSplit ? 4 : kType == kE4m3 ? 1 : 2;
  static constexpr int kCols = kSplit ? 128 : 256;  // columns of a tile of D
  static constexpr bool kW = kOp == kGroupWeight;
  // K block: 128 bytes of a K-major row (of a plane), 64 rows of an MN-major operand; gradient of fp32 matrices, both
  // of whose operands are MN-major: 32 rows, which leaves a stage more
  static constexpr int kBlock = kType == kE4m3 ? 128 : kSplit && kW ? 32 : 64;
  static constexpr int kUnits = kSplit ? kBlock / 32 : 1;  // parts of a K block that the loaders bring one by one
  static constexpr int kPlaneA = kSplit && kW ? kHalf / 2 : kHalf;  // bytes of a plane of A, and of a CTA's half of B
  // Most rows of a tile: 256, or 384 in two accumulators where TMA brings both operands (forward, rows)
  static constexpr int kTileRows = kSplit ? 128 : kW || kLoaders != kNoLoad ? 256 : 384;
  static constexpr int kPlaneB = kSplit ? kPlaneA / 2 : kTileRows / 2 * 128;
  static constexpr int kB = kPlanes * kPlaneA;                // offset of B in a stage
  static constexpr int kStage = kB + kPlanes * kPlaneB;
  static constexpr int kStages = kSplit ? (kW ? 3 : 2) : kLoaders == kLoad ? (kW ? 2 : 3) : 5;
  // What a loader warp keeps of a unit as memory has it, and of how many units
  static constexpr int kRawA = kSplit ? 1024 : 8 * kRawPitch, kRawB = kSplit ? 512 : 8 * kRawPitch;
  static constexpr int kRaw = kRawA + kRawB;
  static constexpr int kDepth = kLoaders != kLoad ? 0 : 3;
  static constexpr int kRawRing = kStages * kStage;
  static constexpr int kOut = kRawRing + kDepth * kRaw * kLoadWarps<kLoad>;
  static constexpr int kOutBytes = kW ? kEpiWarps * 2 * kStoreBuf : kSplit ? 0 : 4 * kOutBuf;
  static constexpr int kBar = kOut + kOutBytes;
  static constexpr int kJobRing = kBar + 512;
  static constexpr int kPlan = kJobRing + kJobs * 32;
  static constexpr int kBytes = 1024 + kPlan + 16;  // and kPlanBytes an expert, in fours
  static_assert((4 * kMaxStages + 2 * kJobs + 9) * 8 + 8 <= 512 - 16, "barriers");
  static_assert(kBytes + kPlanBytes * kMaxExpertsDispatch <= 232448, "shared memory");
  static_assert(kOut % 1024 == 0 && kBar % 32 == 0, "alignment");
};

struct TcMaps {
  CUtensorMap w[2];             // forward, rows: matrices; weight: results
  CUtensorMap wide[3], few[3];  // boxes of 64 and 16 rows: forward x (0); rows dy; weight dy (0, 1), x (2)
};

struct TcFlags {
  int tma_w, tma_r;  // forward, rows: matrices, rows by TMA; weight: x, dy
  int vec_out;       // results on 16 bytes
};

// ---- cluster forms of the building blocks -----------------------------------------------------
// Who wrote what a wait is for: threads of this CTA, copies and MMAs, whose completion is on the barrier itself
// (kHere), or threads of either CTA (kAnywhere: an acquire at cluster scope).
enum : int { kHere = 0, kAnywhere = 1 };
template <int kFrom>
__device__ __forceinline__ bool try_wait_pair(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  if constexpr (kFrom == kAnywhere) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
  }
  return ok != 0;
}
template <int kFrom>
__device__ __forceinline__ bool wait_until(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status,
                                           uint64_t limit_ns) {
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t it = 1;; ++it) {
    if (try_wait_pair<kFrom>(bar, parity)) return true;
    if ((it & 63u) == 0u) {
      if (abort_flag != nullptr && *abort_flag) return false;
      if (globaltimer_ns() - t0 > limit_ns) {
        if (abort_flag != nullptr) *abort_flag = 1;
        if (status != nullptr) atomicOr(status, PR2_STATUS_TIMEOUT);
        return false;
      }
    }
  }
}
template <int kFrom>
static __device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status,
                                              uint64_t limit_ns) {
  return wait_until<kFrom>(bar, parity, abort_flag, status, limit_ns);
}
// A whole warp waits; true if every lane saw the phase complete.  kInline: without a call, across which few
// registers could be kept.
template <int kFrom, bool kInline>
__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int32_t* status,
                                          uint64_t limit_ns = kWaitLimitNs) {
  bool in = try_wait_pair<kFrom>(bar, parity);
  if (!in) {
    in = kInline ? wait_until<kFrom>(bar, parity, abort_flag, status, limit_ns)
                 : wait_slow<kFrom>(bar, parity, abort_flag, status, limit_ns);
  }
  return __all_sync(0xffffffffu, in);
}
__device__ __forceinline__ void arrive_expect_at(uint32_t cluster_addr, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.release.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(cluster_addr),
               "r"(bytes)
               : "memory");
}
// An arrival that hands over no global memory: a release at cluster scope would wait for every store and
// copy that the thread has in flight (gradient of the matrices 366 -> 313 us without that).  Where shared
// memory is handed over, each writer goes through release_shared() first.
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// What this thread wrote into its CTA's shared memory is there for the async proxy and the whole cluster.
__device__ __forceinline__ void release_shared() {
  fence_proxy_async_smem();
  asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory");
}
// TMA loads of a pair's CTA, completing on a barrier of either CTA (a shared::cluster address).
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const void* map, uint32_t bar, int32_t x, int32_t y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_at(uint32_t dst, const void* map, uint32_t bar, int32_t x, int32_t y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const void* map, uint32_t bar, int32_t x, int32_t y,
                                             int32_t z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
// Adds to a value that this thread alone writes: no wait for what is there.
__device__ __forceinline__ void add_global(float* p, float v) {
  asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(p), "f"(v) : "memory");
}
template <int kOffset>
__device__ __forceinline__ float ld_shared_at(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1 + %2];" : "=f"(v) : "r"(addr), "n"(kOffset));
  return v;
}
// A value of each of eight rows 64 bytes apart.
template <size_t... kRow>
__device__ __forceinline__ void load_rows8(const uint32_t (&at)[4], float (&f)[8], std::index_sequence<kRow...>) {
  ((f[kRow] = ld_shared_at<static_cast<int>(kRow) * 64>(at[kRow / 2])), ...);
}
// `count` values to (or added to) addresses `step` apart.
template <int kMost, typename TC>
__device__ __forceinline__ void put_column(TC* p, int64_t step, const float (&f)[kMost], int count, bool add) {
  if (!add && count >= kMost) {  // (few instructions a value: they are what bounds these stores)
#pragma unroll
    for (int i = 0; i < kMost; ++i, p += step) *p = from_f32<TC>(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kMost; ++i, p += step)
      if (i < count) {
        if (sizeof(TC) == 4 && add) add_global(reinterpret_cast<float*>(p), f[i]);
        else *p = from_f32<TC>(f[i]);
      }
  }
}
__device__ __forceinline__ void store_3d(const void* map, uint32_t src, int32_t x, int32_t y, int32_t z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(src), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void add_3d(const void* map, uint32_t src, int32_t x, int32_t y, int32_t z) {
  asm volatile(
      "cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
          reinterpret_cast<uint64_t>(map)),
      "r"(src), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void bulk_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kPending) : "memory");
}
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ void pair_tmem_alloc(uint32_t* slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_free(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
// Arrive on the barrier at this place in both CTAs once the MMAs issued so far have completed.
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"(static_cast<uint16_t>(3))
      : "memory");
}
template <int kType>
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (kType == kE4m3) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
        "r"(accumulate)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
        "r"(accumulate)
        : "memory");
  }
}

// A warp's columns of an accumulator (16 of every 32, from c0 on) to, or onto, the sums.  Four at a time: more take
// registers that the rest of the epilogue needs (16: spills of 200 bytes, operands off 16 bytes 1 % slower).
__device__ __forceinline__ void add_chunk(uint32_t tacc, uint32_t tsum, int c0, int cols, bool add) {
  for (; c0 < cols; c0 += 32) {
#pragma unroll 1
    for (int c = c0; c < c0 + 16; c += 4) {
      uint32_t v[4], w[4] = {0u, 0u, 0u, 0u};
      auto load = [](uint32_t from, uint32_t (&r)[4]) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(from)
                     : "memory");
      };
      load(tacc + c, v);
      if (add) load(tsum + c, w);
      asm volatile("tcgen05.wait::ld.sync.aligned;"
                   : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])
                   :
                   : "memory");
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w[i]));
      asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(tsum + c), "r"(v[0]), "r"(v[1]),
                   "r"(v[2]), "r"(v[3])
                   : "memory");
    }
  }
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// ---- jobs -------------------------------------------------------------------------------------
struct alignas(32) Job {
  int e;     // expert; -1: no more jobs
  int pair;
  int m0;    // first column of A's 256 (two matrices in a forward pass: of each CTA's 128)
  int n0;    // weight: first column of B
  int row0;  // first row; forward, rows: of the tile
  int rows;  // rows of the tile; weight: of the expert
  int kb;    // K blocks
  int unused;
};

template <int kOp, typename L>
struct Plan {
  static constexpr int kBlock = L::kBlock;
  int total, m_blocks, n_blocks, each;  // each: jobs of an expert (weight)
  int kb;    // forward, rows: K blocks of every job
  int most;  // forward, rows: of an expert's rows that are one tile whatever kCols is
  int* order;   // [N], in shared memory; weight: experts, those of most rows and of fewest in turn
  int* prefix;  // [N + 1] forward, rows: jobs of the experts before
  // Tiles of n rows.  Up to 384 rows are one tile although it fills both accumulators, so that no epilogue
  // overlaps the next tile's MMAs: an expert's matrices then leave L2 once (128 experts of 320 rows, bf16, 2048 to 2 x
  // 768 columns: 197 us, in tiles of at most 256 rows 234; 512 to 2048 columns 95, 103).  More rows go in tiles of at
  // most 256 (bf16, 128 experts of 256 rows in the mean, 384 for all: 242 us against 238).  e4m3, whose K blocks of 128
  // columns cost as much, so that the epilogue weighs more, only from 4096 columns on (320 rows: 7168 to 2 x 2048 226 us
  // against 259 in tiles of 256, 4096 to 2 x 1024 156, 165; 3584 142, 146 and to 1024 93, 87; 2048 to 2 x 768 148, 134;
  // 768 to 2048 117, 97).
  __device__ __forceinline__ int tiles_of(int n) const {
    return L::kTileRows > L::kCols && n > 0 && n <= most ? 1 : (n + L::kCols - 1) / L::kCols;
  }
  // Job j, false if there is nothing to do.  A whole warp calls it.
  __device__ __forceinline__ bool job(const GroupArgs& g, int j, Job& b) const {
    b = Job{};
    if (j >= total) return false;
    if constexpr (kOp == kGroupWeight) {
      b.e = order[j / each];
      j %= each;
      b.n0 = j % n_blocks * L::kCols;
      j /= n_blocks;
      b.m0 = j % m_blocks * 256;
      b.pair = j / m_blocks;
      const ExpertRows r = expert_rows(g.offsets, b.e, static_cast<int>(g.rows));
      b.row0 = r.lo;
      b.rows = r.hi - r.lo;
      b.kb = (b.rows + kBlock - 1) / kBlock;
      return b.kb > 0 || !g.accumulate;
    } else {
      const int lane = threadIdx.x & 31;
      auto lowest = [&](auto holds) { return __ffs(__ballot_sync(0xffffffffu, holds(lane))) - 1; };
      b.e = expert_of_job(prefix, g.N, j, lowest);
      const ExpertRows all = expert_rows(g.offsets, b.e, static_cast<int>(g.rows));
      const int n = all.hi - all.lo;
      const RowTile t = row_tile(all.lo, n, tiles_of(n), j - prefix[b.e]);
      b.m0 = t.block * (kOp == kGroupForward && g.pairs == 2 ? 128 : 256);
      b.row0 = t.row0;
      b.rows = t.rows;
      b.kb = kb;
      return b.rows > 0;
    }
  }
};

// Waits that last as long as jobs do (all others wait for a step of the pipeline): for the loads of a job to come to
// their end, and what follows from that.  A job walks all rows of an expert, up to 2^30, so they run out after the usual
// limit and 20 us for each K block of the jobs that may be under way (one takes 0.3 to 1.6 us).
constexpr uint64_t kBlockLimitNs = 20000;
struct UnderWay {
  int64_t last = 0, before = 0;  // K blocks of the job before and of the one before that
  // The limit while a job of kb blocks and those two are under way; it is the last one then.
  __device__ __forceinline__ uint64_t limit(int kb) {
    const uint64_t blocks = static_cast<uint64_t>(kb + last + before);
    before = last;
    last = kb;
    return kWaitLimitNs + blocks * kBlockLimitNs;
  }
};

// A role's way through the scheduler's jobs: every warp of it reads each one and lets its place go.
struct JobReader {
  const Job* ring;
  uint64_t *full, *empty;
  int n = 0;
  template <bool kInline>
  __device__ __forceinline__ bool next(Job& b, volatile int* abort_flag, int32_t* status,
                                       uint64_t limit_ns = kWaitLimitNs) {
    const int slot = n % kJobs;
    if (!wait_pair<kHere, kInline>(&full[slot], (n / kJobs) & 1, abort_flag, status, limit_ns)) return false;
    ++n;
    const int4* p = reinterpret_cast<const int4*>(&ring[slot]);
    const int4 u = p[0], v = p[1];
    b.e = u.x, b.pair = u.y, b.m0 = u.z, b.n0 = u.w;
    b.row0 = v.x, b.rows = v.y, b.kb = v.z;
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(&empty[slot]);
    return b.e >= 0;
  }
};

// Cluster launch control: the number of a pair's first CTA, taken over from one that has not started, is
// written into both CTAs' `response`; false once there is none.
__device__ __forceinline__ void take_over(uint32_t response, uint64_t* bar) {
  asm volatile(
      "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.multicast::cluster::all.b128"
      " [%0], [%1];" ::"r"(response),
      "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ bool taken(uint32_t response, uint32_t& ctaid) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 h;\n\t"
      "mov.u32 %0, 0;\n\t"
      "ld.shared.b128 h, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
      "selp.u32 %1, 1, 0, p;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, h;\n\t}"
      : "=&r"(ctaid), "=&r"(ok)
      : "r"(response)
      : "memory");
  return ok != 0;
}

// ---- what TMA does not bring ------------------------------------------------------------------
// An operand's rows in a K block: byte b of row k of block c (kMn: blocks of 64 elements of the same rows,
// kBlockRows rows each; else one block) comes from base + k stride + c kRowBytes + b where k < rows and the byte
// lies before the end `bytes`, else it is 0.  A loader warp takes kRows of the rows: by cp.async into memory
// of its own as they are, and once they are there into the stage as the tensor core reads them.
struct RowSource {
  const uint8_t* base;
  int64_t stride, step;  // step: from one K block to the next
  int rows, bytes, step_rows, step_bytes;
};
// The part of a warp whose rows start at `first` of the tile's.
template <bool kMn, int kRowBytes, int kBlockRows>
__device__ __forceinline__ RowSource part_of(const RowSource& s, int first) {
  RowSource o = s;
  const int k = kMn ? first % kBlockRows : first, c = kMn ? first / kBlockRows : 0;
  o.base = s.base + k * s.stride + c * kRowBytes;
  o.rows = s.rows - k;
  o.bytes = s.bytes - c * kRowBytes;
  return o;
}

// 16-bit and 8-bit elements: 8 rows, each the nine 16-byte words that hold its 128 bytes wherever they
// start (copied as far as they count: what lies behind the end is zeros, what lies in front is never used
// and shares its 16 bytes with the row's first).  Where in its 16 bytes a row starts is the same in every K
// block, 128 bytes or 64 rows further.  Instructions bound it, not memory, so what a lane copies is worked
// out once a job (16 warps of that: 256 experts of 27 rows, two matrices of 601 x 608, forward 265 -> 190 us).
template <bool kMn>
struct RawRows {
  static constexpr int kRows = 8, kWords = 9 * kRows, kTurns = (kWords + 31) / 32;
  const uint8_t* word[kTurns];  // of this lane
  int upto[kTurns];             // bytes of the row there, beyond those of the block's (or all of them): kMn, else
  int64_t step;
  int left;  // rows (kMn) or bytes from this K block on
  __device__ __forceinline__ void start(const RowSource& s) {
    const int lane = threadIdx.x & 31;
    step = s.step;
    left = kMn ? s.rows : s.bytes;
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int v = 32 * t + lane, i = v / 9, c = 16 * (v - 9 * i);
      const uint8_t* p = s.base + i * s.stride;
      const int m = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15u);
      word[t] = p - m + c;
      upto[t] = kMn ? (s.bytes > 128 ? 128 : s.bytes) + m - c : i < s.rows ? m - c : -256;
    }
  }
  // `safe`: an address for copies of nothing.
  __device__ __forceinline__ void issue(uint32_t raw, const uint8_t* safe) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int v = 32 * t + lane;
      if (32 * t + 32 > kWords && v >= kWords) break;
      const int has = kMn ? (v / 9 < left ? upto[t] : 0) : (left > 128 ? 128 : left) + upto[t];
      const int n = has < 0 ? 0 : has > 16 ? 16 : has;
      cp_async_16(raw + 16 * v, n > 0 ? word[t] : safe, static_cast<uint32_t>(n));
      word[t] += step;
    }
    left -= kMn ? 64 : 128;
  }
  // `low`: where in its 16 bytes the first row starts.
  __device__ __forceinline__ static void put(uint32_t low, uint32_t stride, int first, int, uint32_t raw, uint32_t dst) {
    const int lane = threadIdx.x & 31;
    dst += first * 128 + (lane & 3) * 4;
    raw += 4 * lane;
    uint32_t lo[kRows], hi[kRows];  // (all rows' words first: one latency, not one a row)
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const uint32_t at = raw + i * kRawPitch + ((low + i * stride) & 12u);
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(lo[i]) : "r"(at));
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(hi[i]) : "r"(at + 4));  // (not used where it lies behind the row)
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + i * 128 + (((lane >> 2) ^ (i & 7)) << 4)),
                   "r"(__funnelshift_r(lo[i], hi[i], 8 * ((low + i * stride) & 3u)))
                   : "memory");
  }
};

// x = hi + mid + lo, each bf16, to the last bit of fp32: hi is x cut off after 8 bits (which cannot overflow and
// keeps infinities and, unlike its upper half word, any NaN), mid the rest to nearest, lo what that leaves, of
// either sign.  |mid| is below 2^-7 of x and |lo| below 2^-16, so the product left out (lo lo) is below 2^-32 of a
// product.  (Without mid lo and lo mid it is 2^-22, four units, for 1 to 4 % less time: 1001 tokens, 16 experts of
// 1000 x 515 51.6 us against 52.1, both gradients of 517 tokens, 60 experts of 192 x 250 35.2 against 36.7.)  An
// infinity leaves NaN in mid, but hi's products alone say what it comes to: see the epilogue.  Two values at once, in
// the halves of a word a plane.
__device__ __forceinline__ void split3(float x, float y, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const uint32_t bx = __float_as_uint(x), by = __float_as_uint(y);
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
  const float rx = x - __uint_as_float(bx & 0xffff0000u), ry = y - __uint_as_float(by & 0xffff0000u);
  mid = pack_bf16x2(rx, ry);
  lo = pack_bf16x2(rx - __uint_as_float(mid << 16), ry - __uint_as_float(mid & 0xffff0000u));
}

// fp32: a unit is 32 values of each K-major row, or 32 rows of 64 values of each block of an MN-major operand; in
// the stage, as three planes of bf16, half (unit 0 or 1 of the K block) of the rows' 128 bytes or of the blocks'
// rows.  kRowsK is of the K-major kind.  (K-major rows of 32 in planes with 64-byte swizzle made the MMAs three
// times as long.)
template <bool kMn, int kRowsK, int kPlane, int kBlockRows>
struct RawFloats {
  static constexpr int kRows = kMn ? kRowsK / 2 : kRowsK, kRowBytes = kMn ? 256 : 128;
  template <int kWord>
  __device__ __forceinline__ static void copy(const RowSource& s, uint32_t raw) {
    constexpr int kWords = kRowBytes / kWord, kAtOnce = kWords < 32 ? 32 / kWords : 1;
    const int lane = threadIdx.x & 31;
    const int i0 = kWords < 32 ? lane / kWords : 0;
#pragma unroll
    for (int i = 0; i < kRows; i += kAtOnce) {
      const uint8_t* p = s.base + (i + i0) * s.stride;
#pragma unroll
      for (int c0 = 0; c0 < kRowBytes; c0 += 32 * kWord) {
        const int c = c0 + (kWords < 32 ? lane % kWords : lane) * kWord;
        const bool in = i + i0 < s.rows && c < s.bytes;
        const uint32_t to = raw + (i + i0) * kRowBytes + c;
        if (kWord == 16) cp_async_16(to, in ? p + c : s.base, in ? 16u : 0u);
        else cp_async_4(to, in ? p + c : s.base, in ? 4u : 0u);
      }
    }
  }
  RowSource s;
  __device__ __forceinline__ void start(const RowSource& from) { s = from; }
  __device__ __forceinline__ void issue(uint32_t raw, const uint8_t*) {
    if ((reinterpret_cast<uintptr_t>(s.base) & 15u) == 0 && (s.stride & 15) == 0 && (s.bytes & 15) == 0)
      copy<16>(s, raw);
    else
      copy<4>(s, raw);
    s.base += s.step;
    s.rows -= s.step_rows;
    s.bytes -= s.step_bytes;
  }
  __device__ __forceinline__ static void put(uint32_t, uint32_t, int first, int unit, uint32_t raw, uint32_t dst) {
    const int lane = threadIdx.x & 31;
    const int row0 = kMn ? first / 32 * kBlockRows + first % 32 + unit * 32 : first;
    constexpr int kStep = kMn ? 2 : 4;  // rows at a time: four neighbouring values a lane
    const int c = kMn ? lane & 15 : lane & 7, i1 = kMn ? lane >> 4 : lane >> 3;
    raw += i1 * kRowBytes + c * 16;
    dst += (row0 + i1) * 128 + (c & 1) * 8;
    const int word = (c >> 1) + (kMn ? 0 : 4 * unit);  // of 16 bytes, before the swizzle
    constexpr int kIters = kRows / kStep;
    float f[kIters][4];
#pragma unroll
    for (int n = 0; n < kIters; ++n)
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(f[n][0]), "=f"(f[n][1]), "=f"(f[n][2]), "=f"(f[n][3])
                   : "r"(raw + n * kStep * kRowBytes));
#pragma unroll
    for (int n = 0; n < kIters; ++n) {
      uint32_t p[3], q[3];
      split3(f[n][0], f[n][1], p[0], p[1], p[2]);
      split3(f[n][2], f[n][3], q[0], q[1], q[2]);
      const int i0 = n * kStep;
      const uint32_t at = dst + i0 * 128 + ((word ^ ((row0 + i0 + i1) & 7)) << 4);
#pragma unroll
      for (int j = 0; j < 3; ++j)
        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + j * kPlane), "r"(p[j]), "r"(q[j]) : "memory");
    }
  }
};

// Zeros into rows left .. (the next multiple of 16) - 1 of a stage's four blocks of 64 rows; those of `which`.
__device__ __forceinline__ void zero_rows(uint32_t stage, int left, int which, int w, int warps) {
  const int n = ((left + 15) & ~15) - left;
  for (int v = w * 32 + (threadIdx.x & 31); v < n * 32; v += warps * 32) {
    const int c = (v >> 3) & 3;
    if ((which >> c) & 1)
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(stage + c * (kHalf / 2) + (left + (v >> 5)) * 128 +
                                                                    (v & 7) * 16),
                   "r"(0u)
                   : "memory");
  }
}

template <int kOp, int kType, typename TC, int kLoaders>
__global__ void __launch_bounds__(Roles<kOp, kType, kLoaders>::kThreads, 1)
    grouped_tc_kernel(const __grid_constant__ TcMaps maps, GroupArgs g, TcFlags fl) {
  using L = Layout<kOp, kType, kLoaders>;
  constexpr int kStages = L::kStages, kStage = L::kStage, kBlock = L::kBlock, kEs = L::kEs;
  constexpr bool k8 = kType == kE4m3, kSplit = kType == kFp32;
  using R = Roles<kOp, kType, kLoaders>;
  constexpr int kEpiWarp0 = R::kEpi0, kSchedWarp = R::kSched, kLoadWarp0 = R::kLoad0;
  constexpr int kMmas = kType == kE4m3 ? 4 : kBlock / 16;  // of a K block, in turn
  constexpr int kChunk = sizeof(TC) == 2 ? 1 << 30 : (R::kKeep ? kKeepMmas : kSplit ? kExactMmas : kMostMmas) / kMmas;
  // Results in 16 bits: longer sums leave the accumulator too, for its neighbour (see kLongMmas)
  constexpr bool kLong = sizeof(TC) == 2 && kOp != kGroupWeight;
  constexpr int kLongBlocks = kLongMmas / kMmas;
  static_assert((kLongBlocks & (kLongBlocks - 1)) == 0, "power of two");
  constexpr bool kAMn = kOp != kGroupForward, kBMn = kOp == kGroupWeight;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBar);  // the first CTA's counts
  uint64_t* empty = full + kMaxStages;
  uint64_t* tail = empty + kMaxStages;      // weight: an expert's last rows have landed in this CTA
  uint64_t* zeroed = tail + kMaxStages;     // and zeros stand behind them (the first CTA counts)
  uint64_t* job_full = zeroed + kMaxStages;  // [kJobs]
  uint64_t* job_empty = job_full + kJobs;    // [kJobs]
  uint64_t* acc_full = job_empty + kJobs;    // [2]
  uint64_t* acc_empty = acc_full + 2;       // [2], the first CTA's counts
  uint64_t* drain = acc_empty + 2;
  uint64_t* want = drain + 1;                // [2] the first CTA's TMA warp is near the end of a job
  uint64_t* answer = want + 2;               // cluster launch control has answered
  uint64_t* heard = answer + 1;              // and the second CTA has read that (the first CTA counts)
  uint4* response = reinterpret_cast<uint4*>(smem + L::kBar + 512 - 16);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(heard + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_ctarank());
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1 + (kLoaders == kLoad ? 2 * kLoadWarps<kLoaders> : 0));
      mbar_init(&empty[s], 1);
      mbar_init(&tail[s], 1);
      mbar_init(&zeroed[s], 2 * kLoadWarps<kZeros>);
    }
    for (int i = 0; i < kJobs; ++i) {  // TMA, epilogue, loaders, and of the first CTA the MMA warp
      mbar_init(&job_full[i], 1);
      mbar_init(&job_empty[i], 2 + kEpiWarps + kLoadWarps<kLoaders> + (rank == 0 ? 1 : 0));
    }
    mbar_init(&want[0], 1);
    mbar_init(&want[1], 1);
    mbar_init(answer, 1);
    mbar_init(heard, 1);
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], 2 * kEpiWarps);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kWarpMma) {
    pair_tmem_alloc(tmem_slot, kTmemCols);
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  cluster_sync();  // both CTAs' barriers stand before either arrives at the other's
  pdl_wait();
  pdl_trigger();

  // ---- the plan: weight: the experts' order by their rows; forward, rows: the jobs before each expert ----
  Plan<kOp, L> plan;
  {
    const int N = g.N, fours = (N + 3) & ~3, threads = static_cast<int>(blockDim.x);
    plan.order = plan.prefix = reinterpret_cast<int*>(smem + L::kPlan);
    int* cnt = reinterpret_cast<int*>(smem);  // (the stages' memory, until the plan stands)
    for (int e = threadIdx.x; e < fours; e += threads) {
      const ExpertRows r = e < N ? expert_rows(g.offsets, e, static_cast<int>(g.rows)) : ExpertRows{0, -1};
      cnt[e] = r.hi - r.lo;
    }
    const bool stop = status_timed_out(g.status);
    __syncthreads();
    if constexpr (kOp == kGroupWeight) {
      for (int e = threadIdx.x; e < N; e += threads) {
        const int own = cnt[e];
        int before = 0;
        for (int f = 0; f < fours; f += 4) {
          const int4 v = *reinterpret_cast<const int4*>(cnt + f);
          before += v.x > own || (v.x == own && f < e) ? 1 : 0;
          before += v.y > own || (v.y == own && f + 1 < e) ? 1 : 0;
          before += v.z > own || (v.z == own && f + 2 < e) ? 1 : 0;
          before += v.w > own || (v.w == own && f + 3 < e) ? 1 : 0;
        }
        // experts of many rows keep the tensor cores busy, those of few the HBM: in turn from both ends
        plan.order[before < (N + 1) / 2 ? 2 * before : 2 * (N - 1 - before) + 1] = e;
      }
      __syncthreads();
    }
    plan.kb = kOp == kGroupForward ? (g.d_in + kBlock - 1) / kBlock : g.pairs * ((g.d_out + kBlock - 1) / kBlock);
    plan.most = (kLong && plan.kb > kLongBlocks) || (k8 && plan.kb < kWideBlocks) ? 0 : L::kTileRows;
    plan.n_blocks = kOp == kGroupWeight ? (g.d_in + L::kCols - 1) / L::kCols : (g.d_in + 255) / 256;
    if constexpr (kOp == kGroupWeight) {
      plan.m_blocks = (g.d_out + 255) / 256;
      plan.each = g.pairs * plan.m_blocks * plan.n_blocks;
      plan.total = stop ? 0 : N * plan.each;
    } else {
      plan.m_blocks = kOp == kGroupForward ? (g.pairs == 2 ? (g.d_out + 127) / 128 : (g.d_out + 255) / 256)
                                           : plan.n_blocks;
      if (warp == 0) {
        const int per = (N + 31) / 32, e0 = lane * per, e1 = e0 + per < N ? e0 + per : N;  // a lane's experts
        int own = 0;
        for (int e = e0; e < e1; ++e) own += plan.tiles_of(cnt[e]) * plan.m_blocks;
        int upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        upto -= own;
        for (int e = e0; e < e1; ++e) {
          upto += plan.tiles_of(cnt[e]) * plan.m_blocks;
          plan.prefix[e + 1] = upto;
        }
        if (lane == 0) plan.prefix[0] = 0;
      }
      __syncthreads();
      plan.total = stop ? 0 : plan.prefix[N];
    }
  }
  fence_proxy_async_smem();  // the plan's use of the stages' memory is over before copies land there
  __syncthreads();
  // columns of D that a tile's MMAs cover
  auto columns = [&](const Job& b) {
    return kOp == kGroupWeight ? (L::kCols == 128 || g.d_in - b.n0 <= 128 ? 128 : 256) : round32(b.rows);
  };
  auto longer = [](const Job& b) { return kLong && b.kb > kLongBlocks; };
  // rows of a tile's first accumulator: all, or half of more than one holds
  auto first_rows = [&](const Job& b) {
    return kOp == kGroupWeight || b.rows <= L::kCols ? b.rows : round32((b.rows + 1) / 2);
  };

  const bool epilogue = warp >= kEpiWarp0 && warp < kEpiWarp0 + kEpiWarps;
  JobReader jobs{reinterpret_cast<const Job*>(smem + L::kJobRing), job_full, job_empty};
  Job b{};

  if (!epilogue) {  // (by whole warpgroups)
    if constexpr (R::kKeep) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kKeepOtherRegs));
  }
  if (epilogue) {
    if constexpr (R::kKeep) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kKeepEpiRegs));
    // ---------------- epilogue: TMEM lane 32 (warp % 4) + lane = row of D, column = column of D ----------------
    const int q = warp & 3;
    const int side = (warp - kEpiWarp0) >> 2;
    const uint32_t tq = tmem + (static_cast<uint32_t>(q * 32) << 16);
    const uint32_t freed = mapa_shared(smem_u32(acc_empty), 0);
    int used = 0;
    uint32_t sel = 0;
    bool in = true;
    // 16 columns of this lane from a column of the accumulator on; fp32: the large products' and the small ones' sums
    auto load16 = [&](uint32_t col, uint32_t (&v)[16], uint32_t (&small)[16]) {
      tmem_ld16(col, v);
      if constexpr (kSplit) tmem_ld16(col + kAccCols / 2, small);
    };
    auto ready16 = [&](uint32_t (&v)[16], uint32_t (&small)[16]) {
      tmem_wait_ld(v);
      if constexpr (kSplit) {
        reg_fence(small);
#pragma unroll
        for (int i = 0; i < 16; ++i) {  // (beside an infinity the small products are whatever its planes gave)
          const float large = __uint_as_float(v[i]);
          if (fabsf(large) < INFINITY) v[i] = __float_as_uint(large + __uint_as_float(small[i]));
        }
      }
    };
    // Gradient of the matrices: 32 x 16 blocks through two buffers of the warp (64-byte swizzle: the 16-byte
    // word c of row r sits at c ^ (r / 2 % 4)), each stored by one copy.  Results that do not lie on 16 bytes:
    // two neighbouring blocks, then runs of 32 values of a row (with an address and a branch a value, the
    // gradient of 128 experts of 17 rows, 1613 x 64, took 114 us; 64).
    const uint32_t sw = smem_u32(smem + L::kOut) + (warp - kEpiWarp0) * 2 * kStoreBuf;
    int o = 0, n = 0, cols = 0;  // the warp's first row of D, its rows and columns there
    auto place = [&]() {
      o = b.m0 + 128 * rank + 32 * q;
      n = g.d_out - o < 32 ? g.d_out - o : 32;
      cols = n <= 0 ? 0 : g.d_in - b.n0 > L::kCols ? L::kCols : g.d_in - b.n0;
    };
    const bool vec_out = R::kKeep || fl.vec_out;
    auto column = [&](int i) { return vec_out ? side * 16 + 32 * i : side * 32 + 64 * (i >> 1) + 16 * (i & 1); };
    auto inside = [&](int c) { return (vec_out ? c : c & ~16) < cols; };
    auto put_block = [&](const uint32_t (&v)[16], int step, bool add) {
      const int c0 = column(step);
      const uint32_t at = sw + sel * kStoreBuf;
      sel ^= 1u;
      if (vec_out && lane == 0) bulk_wait_read<1>();  // the copy before last has left this buffer
      __syncwarp();
#pragma unroll
      for (int c = 0; c < 4; ++c)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)),
                     "r"(v[4 * c]), "r"(v[4 * c + 1]), "r"(v[4 * c + 2]), "r"(v[4 * c + 3])
                     : "memory");
      if (vec_out) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (add) add_3d(&maps.w[b.pair], at, b.n0 + c0, o, b.e);
          else store_3d(&maps.w[b.pair], at, b.n0 + c0, o, b.e);
          bulk_commit();
        }
      } else if (step & 1) {
        __syncwarp();
        const int c = c0 - 16 + lane;
        float* p = static_cast<float*>(const_cast<void*>(g.W[b.pair])) +
                   (static_cast<int64_t>(b.e) * g.d_out + o) * g.d_in + b.n0 + c;
        const uint32_t from = sw + (lane >> 4) * kStoreBuf + (lane & 3) * 4;
        if (c < cols) {
#pragma unroll
          for (int r0 = 0; r0 < 32; r0 += 8) {
            float f[8];
            uint32_t at8[4];  // rows 2 i and 2 i + 1 of eight
#pragma unroll
            for (int i = 0; i < 4; ++i) at8[i] = from + r0 * 64 + ((((lane >> 2) ^ i) & 3) << 4);
            load_rows8(at8, f, std::make_index_sequence<8>{});
            if (r0 < n) put_column<8, float>(p, g.d_in, f, n - r0, add);
            p += 8 * static_cast<int64_t>(g.d_in);
          }
        }
      }
    };
    while (in && jobs.next<R::kKeep>(b, abort_flag, g.status)) {
      if constexpr (R::kKeep) {
        // the chunks' sums in registers, 8 blocks of 16 columns a lane, each accumulator free once it is read
        // (columns that no MMA has written are read too, but not stored)
        const int sums = (b.kb + kChunk - 1) / kChunk;
        place();
        uint32_t sum[8][16];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[i][j] = 0u;
        for (int chunk = 0; chunk < sums; ++chunk) {
          const int buf = used & 1;
          const uint32_t tacc = tq + buf * kAccCols;
          in = wait_pair<kHere, R::kKeep>(&acc_full[buf], (used >> 1) & 1, abort_flag, g.status);
          if (!in) break;
          tc_fence_after();
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint32_t v[16];
            tmem_ld16(tacc + column(i), v);
            tmem_wait_ld(v);
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[i][j] = __float_as_uint(__uint_as_float(sum[i][j]) + __uint_as_float(v[j]));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(freed + buf * 8);
          ++used;
        }
        if (!in) break;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (inside(column(i))) put_block(sum[i], i, g.accumulate);
        continue;
      }
      // each chunk of K (results in fp32), and of each the one or two accumulators of the tile's rows
      const int rows0 = first_rows(b), rows_all = b.rows, row_first = b.row0;
      // (a longer sum has both accumulators, of which the second takes no MMAs: it holds the chunks' sums)
      const int parts = rows0 < rows_all || longer(b) ? 2 : 1;
      const int per = longer(b) ? kLongBlocks : kChunk, sums = b.kb <= per ? 1 : (b.kb + per - 1) / per;
      for (int i = 0; i < parts * sums && in; ++i) {
        const int chunk = i / parts;
        if (parts == 2) {
          b.rows = i % 2 == 0 ? rows0 : rows_all - rows0;
          b.row0 = row_first + (i % 2 == 0 ? 0 : rows0);
        }
        const int buf = used & 1;
        uint32_t tacc = tq + buf * kAccCols;
        auto wait_acc = [&]() { return b.kb == 0 || wait_pair<kHere, R::kKeep>(&acc_full[buf], (used >> 1) & 1, abort_flag, g.status); };
        if constexpr (kOp == kGroupWeight) {
          in = wait_acc();
          if (!in) break;
          tc_fence_after();
          const bool add = g.accumulate || chunk > 0;
          place();
          if (chunk > 0 && fl.vec_out && lane == 0) bulk_wait_all();  // the chunk before has been added
          // (no block ahead of the one that is stored: that took more registers than there are)
          for (int step = 0; inside(column(step)); ++step) {
            uint32_t v[16], small[16];
            if (b.kb > 0) {
              load16(tacc + column(step), v, small);
              ready16(v, small);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) v[i] = 0u;
            }
            put_block(v, step, add);
          }
        } else {
          const int width = kOp == kGroupForward ? g.d_out : g.d_in;
          const int64_t ld = kOp == kGroupForward ? g.ld_out : g.ld_in;
          const int p = kOp == kGroupForward && g.pairs == 2 ? rank : 0;
          const int c128 = b.m0 + (kOp == kGroupForward && g.pairs == 2 ? 0 : 128 * rank);  // first column of the 128
          TC* out = static_cast<TC*>(const_cast<void*>(kOp == kGroupForward ? g.y[p] : g.x)) + b.row0 * ld + c128;
          const float* wscale = k8 ? g.wscale[p] + static_cast<int64_t>(b.e) * g.d_out : nullptr;
          float ws[4], row_scale = 0.f;
          if constexpr (k8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int o = c128 + 32 * q + (lane >> 2) + 8 * i;
              ws[i] = o < width ? wscale[o] : 0.f;
            }
            const int r = side * 16 + (lane & 15);
            row_scale = r < b.rows ? g.scale[b.row0 + r] : 0.f;
          }
          in = wait_acc();
          auto add_sums = [&]() {  // the results stand in the other accumulator then, once all chunks have been added
            if constexpr (kLong) {
              if (!longer(b) || i % 2 != 0) return;
              const uint32_t tsum = tq + (buf ^ 1) * kAccCols;
              add_chunk(tacc, tsum, side * 16, b.rows, chunk > 0);
              tacc = tsum;
              if (chunk + 1 < sums) b.rows = 0;  // nothing to store yet
            }
          };
          if (sizeof(TC) == 2 && fl.vec_out) {
            // fragments with the rows along registers, transposed by stmatrix into a [16][128] buffer of the
            // side, stored as 256 contiguous bytes a row
            in = named_bar_and(1 + side, 128, in);
            if (!in) break;
            tc_fence_after();
            add_sums();
            const int st_id = ((warp - kEpiWarp0) & 3) * 32 + lane;
            const uint32_t obuf = smem_u32(smem + L::kOut + side * 2 * kOutBuf);
            const uint32_t ost = static_cast<uint32_t>((lane & 7) * kOutPitch + q * 64 + (lane >> 3) * 16);
            const uint32_t old = static_cast<uint32_t>((st_id >> 4) * kOutPitch + (st_id & 15) * 16);
            const bool live = c128 + (st_id & 15) * 8 < width;  // (width % 8 == 0)
            uint32_t y0[8], y1[8];
            auto load_frags = [&](int c) {
              tmem_ld_frag(tacc + c, y0);
              tmem_ld_frag(tacc + c + (16u << 16), y1);
            };
            if (side * 16 < b.rows) load_frags(side * 16);
            for (int c0 = side * 16; c0 < b.rows; c0 += 32) {
              float rs[4];
              if constexpr (k8) {  // (lane's row of this chunk was loaded before; the next one's is now)
                const float now = row_scale;
                const int r = c0 + 32 + (lane & 15);
                row_scale = r < b.rows ? g.scale[b.row0 + r] : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  rs[i] = __shfl_sync(0xffffffffu, now, 8 * (i >> 1) + 2 * (lane & 3) + (i & 1));
              }
              uint32_t pk[2][4];
              tmem_wait_ld8(y0, y1);
#pragma unroll
              for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                  float a0 = __uint_as_float(y0[4 * i + 2 * jj]), a1 = __uint_as_float(y0[4 * i + 2 * jj + 1]);
                  float b0 = __uint_as_float(y1[4 * i + 2 * jj]), b1 = __uint_as_float(y1[4 * i + 2 * jj + 1]);
                  if constexpr (k8) {
                    a0 = a0 * rs[2 * i] * ws[jj];
                    a1 = a1 * rs[2 * i + 1] * ws[jj];
                    b0 = b0 * rs[2 * i] * ws[2 + jj];
                    b1 = b1 * rs[2 * i + 1] * ws[2 + jj];
                  }
                  pk[i][jj] = pack_bf16x2(a0, a1);
                  pk[i][2 + jj] = pack_bf16x2(b0, b1);
                }
              if (c0 + 32 < b.rows) load_frags(c0 + 32);  // on their way while this chunk is stored
              const uint32_t ob = obuf + sel * kOutBuf;
              sel ^= 1u;
              stmatrix_x4_trans(ob + ost, pk[0][0], pk[0][1], pk[0][2], pk[0][3]);
              stmatrix_x4_trans(ob + ost + 8 * kOutPitch, pk[1][0], pk[1][1], pk[1][2], pk[1][3]);
              named_bar_sync(1 + side, 128);  // (the other buffer's reads are behind it too)
              uint32_t v0[4], v1[4];
              ld_shared_v4(ob + old, v0);
              ld_shared_v4(ob + old + 8 * kOutPitch, v1);
              const int r = c0 + (st_id >> 4);
              TC* to = out + r * ld + (st_id & 15) * 8;
              if (live && r < b.rows) st_global_v4(to, v0);
              if (live && r + 8 < b.rows) st_global_v4(to + 8 * ld, v1);
            }
          } else {
            // a row's 32 neighbouring columns are a warp's lanes: single elements, 32 in a run
            if (!in) break;
            tc_fence_after();
            add_sums();
            const int o = 32 * q + lane;
            const bool live = c128 + o < width;
            const float own = k8 && live ? wscale[c128 + o] : 0.f;
            for (int c0 = side * 16; c0 < b.rows; c0 += 32) {
              uint32_t v[16], small[16];
              load16(tacc + c0, v, small);
              float now = row_scale;
              if constexpr (k8) {
                const int r = c0 + 32 + (lane & 15);
                row_scale = r < b.rows ? g.scale[b.row0 + r] : 0.f;
              }
              ready16(v, small);
              float f[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                f[i] = __uint_as_float(v[i]);
                if constexpr (k8) f[i] = f[i] * __shfl_sync(0xffffffffu, now, i) * own;
              }
              if (live) put_column<16, TC>(out + c0 * ld + o, ld, f, b.rows - c0, chunk > 0);
            }
          }
        }
        if (b.kb > 0) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_at(freed + buf * 8);
          ++used;
        }
      }
    }
  } else if (warp == 0 || warp == R::kTmaB) {
    // ---------------- TMA: one warp brings A, one B: issuing both bound a K block (0.42 us, now 0.29) ----------------
    const bool brings_a = warp == 0;
    const uint32_t sbase = smem_u32(smem);
    const uint32_t bars = mapa_shared(smem_u32(full), 0);
    int stage = 0;
    uint32_t phase = 1;
    bool ok = true;
    while (ok && jobs.next<R::kKeep>(b, abort_flag, g.status)) {
      const int near_end = b.kb > kAskAhead ? b.kb - kAskAhead : 0;
      uint64_t* ask = &want[(jobs.n - 1) & 1];
      if (brings_a && b.kb == 0 && rank == 0 && lane == 0) mbar_arrive(ask);
      const int half_cols = columns(b) / 2;
      const int first = first_rows(b), half_first = round32(first) / 2, half_rest = round32(b.rows - first) / 2;
      const int kb1 = kOp == kGroupRows ? b.kb / g.pairs : b.kb;
      for (int kb = 0; kb < b.kb; ++kb) {
        if (!wait_pair<kHere, R::kKeep>(&empty[stage], phase, abort_flag, g.status)) {
          ok = false;
          break;
        }
        if (elect_one()) {
          if (brings_a && rank == 0 && kb == near_end) mbar_arrive(ask);
          const uint32_t sa = sbase + stage * kStage, sb = sa + L::kB, bar = bars + stage * 8;
          if constexpr (kOp == kGroupWeight) {
            const int r0 = b.row0 + kb * kBlock, left = b.rows - kb * kBlock;
            const int o = b.m0 + 128 * rank, i = b.n0 + half_cols * rank;
            const uint32_t row_bytes = (fl.tma_r ? 256u : 0u) + (fl.tma_w ? half_cols * 2u : 0u);  // of this CTA
            if (left >= kBlock) {
              if (brings_a) {
                if (rank == 0) {
                  if (row_bytes != 0u) mbar_arrive_expect_tx(&full[stage], 2u * kBlock * row_bytes);
                  else mbar_arrive(&full[stage]);
                }
                if (fl.tma_r) {
                  pair_load_2d(sa, &maps.wide[b.pair], bar, o, r0);
                  pair_load_2d(sa + kHalf / 2, &maps.wide[b.pair], bar, o + 64, r0);
                }
              } else if (fl.tma_w) {
                pair_load_2d(sb, &maps.wide[2], bar, i, r0);
                if (half_cols == 128) pair_load_2d(sb + kHalf / 2, &maps.wide[2], bar, i + 64, r0);
              }
            } else {  // an expert's last rows: the loaders put zeros behind them before they count
              if (brings_a && rank == 0) mbar_arrive(&full[stage]);
              const int n = (left + 15) & ~15;
              if (row_bytes != 0u) {
                const uint32_t own = smem_u32(&tail[stage]);
                if (brings_a) mbar_arrive_expect_tx(&tail[stage], n * row_bytes);
                for (int r = 0; r < n; r += 16) {
                  if (brings_a && fl.tma_r) {
                    tma_load_at(sa + r * 128, &maps.few[b.pair], own, o, r0 + r);
                    tma_load_at(sa + kHalf / 2 + r * 128, &maps.few[b.pair], own, o + 64, r0 + r);
                  }
                  if (!brings_a && fl.tma_w) {
                    tma_load_at(sb + r * 128, &maps.few[2], own, i, r0 + r);
                    if (half_cols == 128) tma_load_at(sb + kHalf / 2 + r * 128, &maps.few[2], own, i + 64, r0 + r);
                  }
                }
              }
            }
          } else {
            int p = 0, k0 = kb * kBlock;
            if (kOp == kGroupRows && kb >= kb1) {
              p = 1;
              k0 = (kb - kb1) * kBlock;
            }
            if (brings_a) {
              if (rank == 0) {
                const uint32_t bytes =
                    (fl.tma_w ? 2u * kHalf : 0u) + (fl.tma_r ? 2u * (half_first + half_rest) * 128u : 0u);
                if (bytes != 0u) mbar_arrive_expect_tx(&full[stage], bytes);
                else mbar_arrive(&full[stage]);
              }
              if (fl.tma_w) {
                if constexpr (kOp == kGroupForward) {
                  if (g.pairs == 2) pair_load_3d(sa, &maps.w[rank], bar, k0, b.m0, b.e);
                  else pair_load_3d(sa, &maps.w[0], bar, k0, b.m0 + 128 * rank, b.e);
                } else {
                  const int i = b.m0 + 128 * rank;
                  pair_load_3d(sa, &maps.w[p], bar, i, k0, b.e);
                  pair_load_3d(sa + kHalf / 2, &maps.w[p], bar, i + 64, k0, b.e);
                }
              }
            } else if (fl.tma_r) {
              auto rows = [&](uint32_t dst, int r0, int n) {
                int r = 0;
                for (; r + 64 <= n; r += 64) pair_load_2d(dst + r * 128, &maps.wide[p], bar, k0, r0 + r);
                for (; r < n; r += 16) pair_load_2d(dst + r * 128, &maps.few[p], bar, k0, r0 + r);
              };
              rows(sb, b.row0 + half_first * rank, half_first);
              if (half_rest > 0) rows(sb + half_first * 128, b.row0 + first + half_rest * rank, half_rest);
            }
          }
        }
        __syncwarp();
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
  } else if (warp == kWarpMma) {
    // ---------------- MMA: the first CTA's warp in step, one elected lane issues ----------------
    if (rank == 0) {
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const uint32_t sbase = smem_u32(smem);
      constexpr uint32_t kLboA = kAMn ? L::kPlaneA / 2 / 16 : 1, kLboB = kBMn ? L::kPlaneB / 2 / 16 : 1;
      constexpr uint32_t kStepA = kAMn ? 128 : 2, kStepB = kBMn ? 128 : 2;  // of a descriptor, per MMA
      constexpr uint32_t kIdesc = (1u << 4) | (k8 ? 0u : (1u << 7) | (1u << 10)) | (kAMn ? 1u << 15 : 0u) |
                                  (kBMn ? 1u << 16 : 0u) | (16u << 24);
      int stage = 0;
      uint32_t phase = 0;
      int used = 0;
      uint32_t zero_phase = 0;  // a bit for each stage
      bool ok = true;
      while (ok && jobs.next<R::kKeep>(b, abort_flag, g.status)) {
        if (b.kb == 0) continue;
        const int rows0 = first_rows(b), rows1 = b.rows - rows0;
        const int cols0 = kOp == kGroupWeight ? columns(b) : round32(rows0);
        const bool two = L::kTileRows > L::kCols && kOp != kGroupWeight && rows1 > 0;
        const bool both = two || longer(b);
        // K blocks of an accumulator less one, as a mask
        const int in_turn = longer(b) ? kLongBlocks - 1 : 0x3fffffff;
        const uint32_t idesc = kIdesc | (static_cast<uint32_t>(cols0) >> 3 << 17);
        const uint32_t idesc1 = kIdesc | (static_cast<uint32_t>(round32(rows1)) >> 3 << 17);
        uint32_t d = 0;
        for (int kb = 0; kb < b.kb; ++kb) {
          const bool first = kLong ? (kb & in_turn) == 0 : kb % kChunk == 0;
          if (first) {
            const int buf = used & 1;
            if (!wait_pair<kAnywhere, R::kKeep>(&acc_empty[buf], ((used >> 1) & 1) ^ 1, abort_flag, g.status)) {
              ok = false;
              break;
            }
            if (both && !wait_pair<kAnywhere, R::kKeep>(&acc_empty[buf ^ 1], (((used + 1) >> 1) & 1) ^ 1, abort_flag, g.status)) {
              ok = false;
              break;
            }
            tc_fence_after();
            d = tm + buf * kAccCols;
          }
          if (!wait_pair<kLoaders == kLoad ? kAnywhere : kHere, R::kKeep>(&full[stage], phase, abort_flag, g.status)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sa = sbase + stage * kStage;
          const uint32_t la = ((sa & 0x3ffffu) >> 4) | (kLboA << 16);
          const uint32_t lb = (((sa + L::kB) & 0x3ffffu) >> 4) | (kLboB << 16);
          int steps = kMmas;
          if constexpr (kOp == kGroupWeight) {
            const int left = b.rows - kb * kBlock;
            if (left < kBlock) {
              steps = (left + 15) / 16;
              if constexpr (kLoaders == kZeros) {
                if (!wait_pair<kAnywhere, R::kKeep>(&zeroed[stage], (zero_phase >> stage) & 1u, abort_flag, g.status)) {
                  ok = false;
                  break;
                }
                zero_phase ^= 1u << stage;
                tc_fence_after();
              }
            }
          }
          const bool last = kb + 1 == b.kb || (kLong ? ((kb + 1) & in_turn) == 0 : (kb + 1) % kChunk == 0);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < kMmas; ++kk) {
              if (kOp == kGroupWeight && kk >= steps) break;
              const uint32_t more = !first || kk > 0 ? 1u : 0u;
              auto mma = [&](uint32_t acc, int pa, int pb, uint32_t add) {
                pair_mma<kType>(acc, umma_desc_lo(la + kStepA * kk + pa * (L::kPlaneA / 16)),
                                umma_desc_lo(lb + kStepB * kk + pb * (L::kPlaneB / 16)), idesc, add);
              };
              mma(d, 0, 0, more);
              if constexpr (kSplit) {  // the small products apart: they are added to the large ones at the end
                mma(d + kAccCols / 2, 1, 2, more);
                mma(d + kAccCols / 2, 2, 1, 1u);
                mma(d + kAccCols / 2, 0, 2, 1u);
                mma(d + kAccCols / 2, 2, 0, 1u);
                mma(d + kAccCols / 2, 1, 1, 1u);
                mma(d + kAccCols / 2, 0, 1, 1u);
                mma(d + kAccCols / 2, 1, 0, 1u);
              }
            }
            if (last) pair_commit(&acc_full[used & 1]);
            if (both && !two && last) pair_commit(&acc_full[(used & 1) ^ 1]);
            if (two) {  // the tile's other rows, against the same A
              const uint32_t lb1 = lb + cols0 / 2 * (128 / 16), d1 = tm + ((used & 1) ^ 1) * kAccCols;
#pragma unroll
              for (int kk = 0; kk < kMmas; ++kk)
                pair_mma<kType>(d1, umma_desc_lo(la + kStepA * kk), umma_desc_lo(lb1 + kStepB * kk), idesc1,
                                !first || kk > 0 ? 1u : 0u);
              if (last) pair_commit(&acc_full[(used & 1) ^ 1]);
            }
            pair_commit(&empty[stage]);
          }
          __syncwarp();
          if (last) used += both ? 2 : 1;
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (elect_one()) pair_commit(drain);
      __syncwarp();
    }
    // MMAs of the pair have read both CTAs' shared memory and written both tensor memories
    if (R::kKeep) wait_until<kHere>(drain, 0, nullptr, nullptr, kWaitLimitNs + kDrainLimitNs);
    else wait_slow<kHere>(drain, 0, nullptr, nullptr, kWaitLimitNs + kDrainLimitNs);
  } else if (warp == kSchedWarp) {
    // ---------------- scheduler ----------------
    const uint32_t answer_there = mapa_shared(smem_u32(answer), 1), heard_at = mapa_shared(smem_u32(heard), 0);
    int j = static_cast<int>(blockIdx.x >> 1), n = 0, asked = 0;
    UnderWay jobs_under_way;
    uint64_t limit = kWaitLimitNs;
    for (;;) {
      const bool work = plan.job(g, j, b);
      bool more = true;
      if (work) {
        limit = jobs_under_way.limit(b.kb);
        const int slot = n % kJobs;
        if (n >= kJobs && !wait_pair<kHere, R::kKeep>(&job_empty[slot], ((n / kJobs) & 1) ^ 1, abort_flag, g.status)) break;
        if (lane == 0) {
          int4* p = reinterpret_cast<int4*>(smem + L::kJobRing + slot * 32);
          p[0] = make_int4(b.e, b.pair, b.m0, b.n0);
          p[1] = make_int4(b.row0, b.rows, b.kb, 0);
          mbar_arrive(&job_full[slot]);
        }
        __syncwarp();
        ++n;
        // The next job is taken when the loads of this one are nearly issued, not sooner: others may be free
        // before.  Behind a short one (an answer takes about 1.4 us) two are kept in hand.
        const int of = b.kb > kAskAhead ? n - 1 : n - 2;
        if (rank == 0 && of >= 0)
          more = wait_pair<kHere, R::kKeep>(&want[of & 1], (of >> 1) & 1, abort_flag, g.status, limit);
      }
      if (rank == 0) {
        if (asked > 0) more = wait_pair<kAnywhere, R::kKeep>(heard, (asked - 1) & 1, abort_flag, g.status) && more;
        if (!more) break;  // (the second CTA's wait for an answer runs out)
        if (lane == 0) {
          mbar_arrive_expect_tx(answer, 16);
          arrive_expect_at(answer_there, 16);
          take_over(smem_u32(response), answer);
        }
        __syncwarp();
      }
      if (!wait_pair<kHere, R::kKeep>(answer, asked & 1, abort_flag, g.status, limit)) break;
      ++asked;
      uint32_t cta;
      more = taken(smem_u32(response), cta);
      release_shared();  // (the answer has been read)
      __syncwarp();
      if (rank == 1 && lane == 0) arrive_at(heard_at);
      if (!more) break;
      j = static_cast<int>(cta >> 1);
    }
    const int slot = n % kJobs;  // no more jobs
    if (n < kJobs || wait_pair<kHere, R::kKeep>(&job_empty[slot], ((n / kJobs) & 1) ^ 1, abort_flag, g.status)) {
      if (lane == 0) {
        *reinterpret_cast<int4*>(smem + L::kJobRing + slot * 32) = make_int4(-1, 0, 0, 0);
        mbar_arrive(&job_full[slot]);
      }
      __syncwarp();
    }
  } else if constexpr (kLoaders == kZeros) {
    // ---------------- zeros behind an expert's last rows, up to the end of the MMAs' 16 ----------------
    const int w = warp - kLoadWarp0;
    const uint32_t sbase = smem_u32(smem);
    const uint32_t done = mapa_shared(smem_u32(zeroed), 0);
    uint32_t tail_phase = 0;  // a bit for each stage
    int64_t blocks = 0;       // K blocks before this job
    UnderWay jobs_under_way;
    uint64_t limit = kWaitLimitNs;
    while (jobs.next<R::kKeep>(b, abort_flag, g.status, limit)) {
      blocks += b.kb;
      limit = jobs_under_way.limit(b.kb);
      const int left = b.rows % kBlock;
      if (left == 0) continue;
      const int stage = static_cast<int>((blocks - 1) % kStages);
      if (!wait_pair<kHere, R::kKeep>(&tail[stage], (tail_phase >> stage) & 1u, abort_flag, g.status, limit)) break;
      tail_phase ^= 1u << stage;
      zero_rows(sbase + stage * kStage, left, 15, w, kLoadWarps<kLoaders>);
      release_shared();
      __syncwarp();
      if (lane == 0) arrive_at(done + stage * 8);
    }
  } else if constexpr (kLoaders == kLoad) {
    // ---------------- loaders: rows of the next K blocks on their way while one is turned over ----------------
    const int w = warp - kLoadWarp0;
    const uint32_t sbase = smem_u32(smem);
    const uint32_t bars = mapa_shared(smem_u32(full), 0);
    const uint32_t raw0 = sbase + L::kRawRing + w * (L::kDepth * L::kRaw);
    using RawA = std::conditional_t<kSplit, RawFloats<kAMn, 128 / kLoadWarps<kLoaders>, L::kPlaneA, kBlock>, RawRows<kAMn>>;
    using RawB = std::conditional_t<kSplit, RawFloats<kBMn, 64 / kLoadWarps<kLoaders>, L::kPlaneB, kBlock>, RawRows<kBMn>>;
    constexpr int kPartBytes = kSplit ? 256 : 128, kPartRows = kSplit ? 32 : 64;  // of an MN-major block
    const uint8_t* safe = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(g.offsets) & ~uintptr_t{15});
    // bytes between rows of A and B, as far as they say where a row starts in its 16 bytes
    const uint32_t stride_a = static_cast<uint32_t>(kOp == kGroupWeight ? g.ld_out : g.d_in) * kEs;
    const uint32_t stride_b = static_cast<uint32_t>(kOp == kGroupRows ? g.ld_out : g.ld_in) * kEs;
    const int first_a = w * RawA::kRows, first_b = w * RawB::kRows;
    int stage = 0;
    uint32_t phase = 1, tail_phase = 0;  // tail_phase: a bit for each stage
    bool ok = true;
    while (ok && jobs.next<R::kKeep>(b, abort_flag, g.status)) {
      const int half_cols = columns(b) / 2;
      const int kb1 = kOp == kGroupRows ? b.kb / g.pairs : b.kb;
      const int64_t matrix = static_cast<int64_t>(b.e) * g.d_out * g.d_in;
      // Parts that only reach rows or columns of D behind its end are left as they are.
      bool load_a = kOp == kGroupWeight ? !fl.tma_r : !fl.tma_w;
      bool load_b = kOp == kGroupWeight ? !fl.tma_w : !fl.tma_r;
      RawA next_a;
      RawB next_b;
      uint32_t low_a[2], low_b[2];  // of the pairs
      // this warp's rows of both operands in the first K block (of pair p)
      auto start = [&](int p) {
        RowSource ra{}, rb{};
        constexpr int kUnit = kBlock / L::kUnits;
        ra.step_bytes = kAMn ? 0 : kUnit * kEs;
        ra.step_rows = kAMn ? kUnit : 0;
        rb.step_bytes = kBMn ? 0 : kUnit * kEs;
        rb.step_rows = kBMn ? kUnit : 0;
        if constexpr (kOp == kGroupWeight) {
          const int64_t r0 = b.row0;
          const int o = b.m0 + 128 * rank, i = b.n0 + half_cols * rank;
          ra.base = static_cast<const uint8_t*>(g.y[b.pair]) + (r0 * g.ld_out + o) * kEs;
          ra.stride = g.ld_out * kEs;
          rb.base = static_cast<const uint8_t*>(g.x) + (r0 * g.ld_in + i) * kEs;
          rb.stride = g.ld_in * kEs;
          ra.rows = rb.rows = b.rows;
          ra.bytes = (g.d_out - o) * kEs;
          rb.bytes = (g.d_in - i) * kEs;
        } else {
          ra.stride = static_cast<int64_t>(g.d_in) * kEs;
          if constexpr (kOp == kGroupForward) {
            const int o = b.m0 + (g.pairs == 2 ? 0 : 128 * rank);
            ra.base = static_cast<const uint8_t*>(g.W[g.pairs == 2 ? rank : 0]) +
                      (matrix + static_cast<int64_t>(o) * g.d_in) * kEs;
            ra.rows = g.d_out - o;
            ra.bytes = g.d_in * kEs;
          } else {
            const int i = b.m0 + 128 * rank;
            ra.base = static_cast<const uint8_t*>(g.W[p]) + (matrix + i) * kEs;
            ra.rows = g.d_out;
            ra.bytes = (g.d_in - i) * kEs;
          }
          const int r0 = half_cols * rank;
          rb.stride = (kOp == kGroupForward ? g.ld_in : g.ld_out) * kEs;
          rb.base = static_cast<const uint8_t*>(kOp == kGroupForward ? g.x : g.y[p]) + (b.row0 + r0) * rb.stride;
          rb.rows = b.rows - r0;
          rb.bytes = (kOp == kGroupForward ? g.d_in : g.d_out) * kEs;
        }
        ra.step = kAMn ? kUnit * ra.stride : kUnit * kEs;
        rb.step = kBMn ? kUnit * rb.stride : kUnit * kEs;
        ra = part_of<kAMn, kPartBytes, kPartRows>(ra, first_a);
        rb = part_of<kBMn, kPartBytes, kPartRows>(rb, first_b);
        load_a = load_a && (kAMn ? ra.bytes : ra.rows) > 0;
        load_b = load_b && (kBMn ? rb.bytes : rb.rows) > 0;
        if (load_a) next_a.start(ra);
        if (load_b) next_b.start(rb);
        low_a[p] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ra.base)) & 15u;
        low_b[p] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(rb.base)) & 15u;
      };
      start(0);
      const int units = b.kb * L::kUnits;
      auto issue = [&](int u) {
        if (u < units) {
          if (kOp == kGroupRows && u == kb1 * L::kUnits) start(1);
          const uint32_t raw = raw0 + u % L::kDepth * L::kRaw;
          if (load_a) next_a.issue(raw, safe);
          if (load_b) next_b.issue(raw + L::kRawA, safe);
        }
        cp_async_commit();
      };
#pragma unroll
      for (int u = 0; u < L::kDepth - 1; ++u) issue(u);
      for (int u = 0; u < units; ++u) {
        issue(u + L::kDepth - 1);
        cp_async_wait<L::kDepth - 1>();
        __syncwarp();  // every lane's copies of this unit have landed
        const int kb = u / L::kUnits, unit = u % L::kUnits;
        if (unit == 0 && !wait_pair<kHere, R::kKeep>(&empty[stage], phase, abort_flag, g.status)) {
          ok = false;
          break;
        }
        const int p = kOp == kGroupRows && u >= kb1 * L::kUnits ? 1 : 0;
        const uint32_t sa = sbase + stage * kStage, sb = sa + L::kB, raw = raw0 + u % L::kDepth * L::kRaw;
        if (load_a) RawA::put(low_a[p], stride_a, first_a, unit, raw, sa);
        if (load_b) RawB::put(low_b[p], stride_b, first_b, unit, raw + L::kRawA, sb);
        if constexpr (kOp == kGroupWeight && !kSplit) {
          const int left = b.rows - kb * kBlock;
          if (left < kBlock && (fl.tma_r || fl.tma_w)) {
            if (!wait_pair<kHere, R::kKeep>(&tail[stage], (tail_phase >> stage) & 1u, abort_flag, g.status)) {
              ok = false;
              break;
            }
            tail_phase ^= 1u << stage;
            zero_rows(sa, left, (fl.tma_r ? 3 : 0) | (fl.tma_w ? 12 : 0), w, kLoadWarps<kLoaders>);
          }
        }
        if (unit == L::kUnits - 1) release_shared();
        __syncwarp();  // (and every lane has read this unit's rows: the next copies may land there)
        if (unit == L::kUnits - 1) {
          if (lane == 0) arrive_at(bars + stage * 8);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      cp_async_wait<0>();
      __syncwarp();
    }
  }
  if (kOp == kGroupWeight && fl.vec_out && epilogue && lane == 0) bulk_wait_all();
  __syncthreads();
  // Once a role has given up, copies and launch control's answer may be in flight that nobody waits for: this CTA
  // stays until they have long landed.  (Without that each has been waited for where it was used.)
  if (*abort_flag) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < kDrainLimitNs) __nanosleep(1000);
    __syncthreads();
  }
  cluster_sync();  // neither CTA leaves while the other may still reach it
  if (warp == kWarpMma) {
    tc_fence_after();
    pair_tmem_free(tmem, kTmemCols);
  }
}

// ---- launch -----------------------------------------------------------------------------------
bool on16(const void* p, int64_t row_bytes) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && row_bytes % 16 == 0 && row_bytes < (int64_t{1} << 40);
}

template <int kOp, int kType, typename TC, int kLoaders>
cudaError_t launch_pairs(const TcMaps& m, const GroupArgs& g, const TcFlags& fl, int pairs, cudaStream_t st) {
  auto* kernel = grouped_tc_kernel<kOp, kType, TC, kLoaders>;
  constexpr int kBytes = Layout<kOp, kType, kLoaders>::kBytes;
  const int smem = kBytes + kPlanBytes * ((g.N + 3) & ~3);
  using R = Roles<kOp, kType, kLoaders>;
  static_assert(!R::kKeep || R::kThreads == kKeepThreads, "threads");
  // The limit is the kernel's, not the launch's: the same for every number of experts, so that a call with fewer
  // of them on another host thread cannot lower it between this and a launch.
  cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         kBytes + kPlanBytes * kMaxExpertsDispatch);
  if (err != cudaSuccess) return err;
  if constexpr (R::kKeep) {  // without the registers that the epilogue takes over it would wait forever
    static const int regs = [kernel] {
      cudaFuncAttributes attr{};
      return cudaFuncGetAttributes(&attr, kernel) == cudaSuccess ? attr.numRegs : 0;
    }();
    if (regs < kKeepRegs) return cudaErrorInvalidConfiguration;
  }
  return launch_pdl(kernel, dim3(2 * pairs), dim3(R::kThreads), smem, st, 2, m, g, fl);
}

template <int kOp, int kType, typename TC>
cudaError_t launch_tc(const GroupArgs& g, cudaStream_t st) {
  using L = Layout<kOp, kType, kLoad>;  // (sizes that do not depend on the loaders)
  constexpr int kEs = L::kEs;
  constexpr bool kTma = kType != kFp32;  // (fp32 operands pass through the loaders' registers)
  constexpr uint32_t kBox = 128 / kEs;
  const auto type = kType == kE4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  TcMaps m{};
  TcFlags fl{};
  const uint64_t N = g.N, d_in = g.d_in, d_out = g.d_out, rows = g.rows;
  bool ok = true;
  auto map_rows = [&](CUtensorMap* t, const void* p, uint64_t width, int64_t ld, uint32_t box_rows) {
    const uint64_t dims[2] = {width, rows}, strides[1] = {static_cast<uint64_t>(ld) * kEs};
    const uint32_t box[2] = {kBox, box_rows};
    ok = ok && make_tmap(t, type, 2, p, dims, strides, box);
  };
  int64_t jobs;
  if constexpr (kOp == kGroupWeight) {
    fl.tma_r = kTma && on16(g.y[0], g.ld_out * kEs) && (g.pairs == 1 || on16(g.y[1], 0));
    fl.tma_w = kTma && on16(g.x, g.ld_in * kEs);
    fl.vec_out = on16(g.W[0], static_cast<int64_t>(d_in) * 4) && (g.pairs == 1 || on16(g.W[1], 0)) &&
                 d_out * d_in * 4 < (uint64_t{1} << 40);
    for (int p = 0; p < g.pairs && fl.vec_out; ++p) {
      const uint64_t dims[3] = {d_in, d_out, N}, strides[2] = {d_in * 4, d_out * d_in * 4};
      const uint32_t box[3] = {16, 32, 1};
      ok = ok && make_tmap(&m.w[p], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, g.W[p], dims, strides, box,
                           CU_TENSOR_MAP_SWIZZLE_64B);
    }
    for (int p = 0; p < g.pairs && fl.tma_r; ++p) {
      map_rows(&m.wide[p], g.y[p], d_out, g.ld_out, 64);
      map_rows(&m.few[p], g.y[p], d_out, g.ld_out, 16);
    }
    if (fl.tma_w) {
      map_rows(&m.wide[2], g.x, d_in, g.ld_in, 64);
      map_rows(&m.few[2], g.x, d_in, g.ld_in, 16);
    }
    jobs = static_cast<int64_t>(g.N) * g.pairs * ((g.d_out + 255) / 256) * ((g.d_in + L::kCols - 1) / L::kCols);
  } else {
    const bool fwd = kOp == kGroupForward;
    const int64_t ld = fwd ? g.ld_in : g.ld_out;
    fl.tma_w = kTma && on16(g.W[0], static_cast<int64_t>(d_in) * kEs) && (g.pairs == 1 || on16(g.W[1], 0)) &&
               d_out * d_in * kEs < (uint64_t{1} << 40);
    fl.tma_r = !kTma ? false : fwd ? on16(g.x, ld * kEs) : on16(g.y[0], ld * kEs) && (g.pairs == 1 || on16(g.y[1], 0));
    fl.vec_out = fwd ? on16(g.y[0], g.ld_out * 2) && (g.pairs == 1 || on16(g.y[1], 0)) && g.d_out % 8 == 0
                     : on16(g.x, g.ld_in * 2) && g.d_in % 8 == 0;
    for (int p = 0; p < g.pairs; ++p) {
      if (fl.tma_w) {
        const uint64_t dims[3] = {d_in, d_out, N}, strides[2] = {d_in * kEs, d_out * d_in * kEs};
        const uint32_t box[3] = {kBox, fwd ? 128u : 64u, 1};
        ok = ok && make_tmap(&m.w[p], type, 3, g.W[p], dims, strides, box);
      }
      if (fl.tma_r && (!fwd || p == 0)) {
        map_rows(&m.wide[p], fwd ? g.x : g.y[p], fwd ? d_in : d_out, ld, 64);
        map_rows(&m.few[p], fwd ? g.x : g.y[p], fwd ? d_in : d_out, ld, 16);
      }
    }
    const int64_t tiles = g.rows / L::kCols + (g.rows < g.N ? g.rows : g.N);
    const int width = fwd ? g.d_out : g.d_in;
    jobs = tiles * (fwd && g.pairs == 2 ? (width + 127) / 128 : (width + 255) / 256);
  }
  if (!ok) return cudaErrorInvalidValue;
  if (jobs > INT32_MAX / 2) return cudaErrorNotSupported;
  const int pairs = static_cast<int>(jobs);  // one for each job that there may be
  if constexpr (kTma) {
    if (fl.tma_w && fl.tma_r && (kOp != kGroupWeight || fl.vec_out))
      return launch_pairs<kOp, kType, TC, kOp == kGroupWeight ? kZeros : kNoLoad>(m, g, fl, pairs, st);
  }
  return launch_pairs<kOp, kType, TC, kLoad>(m, g, fl, pairs, st);
}

}  // namespace

cudaError_t launch_grouped(const GroupArgs& g, cudaStream_t st) {
  if (g.bits8)
    return g.bf16 ? launch_tc<kGroupForward, kE4m3, __nv_bfloat16>(g, st)
                  : launch_tc<kGroupForward, kE4m3, float>(g, st);
  if (g.bf16) {
    if (g.op == kGroupForward) return launch_tc<kGroupForward, kBf16, __nv_bfloat16>(g, st);
    if (g.op == kGroupRows) return launch_tc<kGroupRows, kBf16, __nv_bfloat16>(g, st);
    return launch_tc<kGroupWeight, kBf16, float>(g, st);
  }
  if (g.op == kGroupForward) return launch_tc<kGroupForward, kFp32, float>(g, st);
  if (g.op == kGroupRows) return launch_tc<kGroupRows, kFp32, float>(g, st);
  return launch_tc<kGroupWeight, kFp32, float>(g, st);
}

}  // namespace pr2
