// Rows of an expert from the offsets of a token sort, and the tile that a job's number stands for.  Plain C++
// besides the functions' attributes, so that a host program can go through the jobs too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define PR2_PLAN __host__ __device__ __forceinline__
#else
#define PR2_PLAN inline
#endif

namespace pr2 {

// Rows [lo, hi) of expert e, whatever the offsets hold: inside [0, rows), lo <= hi.
struct ExpertRows {
  int lo, hi;
};
PR2_PLAN int clamp_row(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
PR2_PLAN ExpertRows expert_rows(const int32_t* offsets, int e, int rows) {
  const int lo = clamp_row(offsets[e], rows), hi = clamp_row(offsets[e + 1], rows);
  return ExpertRows{lo, hi < lo ? lo : hi};
}

// The expert of job j: prefix[e] <= j < prefix[e + 1], for 0 <= j < prefix[N], N <= 1024.  Jobs may come in any
// order: cluster launch control names the next one, and which that is is not specified.  `lowest(holds)`: the
// lowest lane of 0 .. 31 for which holds(lane).
template <typename Lowest>
PR2_PLAN int expert_of_job(const int* prefix, int N, int j, const Lowest& lowest) {
  const int per = (N + 31) / 32;  // experts of a lane, then a lane's experts
  const int first = per * lowest([&](int lane) {
    const int end = (lane + 1) * per;
    return j < prefix[end < N ? end : N];
  });
  return first + lowest([&](int lane) { return lane < per && first + lane < N && j < prefix[first + lane + 1]; });
}

constexpr int round32(int n) { return (n + 31) & ~31; }

// Job i of an expert's rows [lo, lo + n), cut into `tiles` tiles of the same size, for every block of columns.
struct RowTile {
  int block, row0, rows;  // rows <= 0: nothing to do
};
PR2_PLAN RowTile row_tile(int lo, int n, int tiles, int i) {
  const int size = round32((n + tiles - 1) / tiles), r = i % tiles * size;
  return RowTile{i / tiles, lo + r, n - r < size ? n - r : size};
}

}  // namespace pr2
