"""Jobs of the experts' products on the CPU (csrc/group_plan.cuh, compiled by the host's compiler): each stands
for one tile of one expert's rows and one block of columns, whatever the order in which they are asked for."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_00395_gb300", "csrc")
SOURCE = """
#include "group_plan.cuh"
// per job: expert, block, first row, rows
extern "C" void jobs(const int32_t* offsets, const int* prefix, const int* tiles, int N, int rows, const int* js, int n,
                     int* out) {
  auto lowest = [](auto holds) {
    for (int lane = 0; lane < 32; ++lane)
      if (holds(lane)) return lane;
    return -1;
  };
  for (int i = 0; i < n; ++i) {
    const int e = pr2::expert_of_job(prefix, N, js[i], lowest);
    const pr2::ExpertRows r = pr2::expert_rows(offsets, e, rows);
    const pr2::RowTile t = pr2::row_tile(r.lo, r.hi - r.lo, tiles[e], js[i] - prefix[e]);
    out[4 * i] = e, out[4 * i + 1] = t.block, out[4 * i + 2] = t.row0, out[4 * i + 3] = t.rows;
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    (where / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fPIC", "-shared", "-I", CSRC, "-o",
                    str(where / "plan.so"), str(where / "plan.cpp")], check=True)
    return ctypes.CDLL(str(where / "plan.so"))


def ints(a):
    return np.ascontiguousarray(a, dtype=np.int32).ctypes.data_as(ctypes.c_void_p)


@pytest.mark.parametrize("order", ["up", "down", "any"])
@pytest.mark.parametrize("N,most,columns", [(1, 5, 1), (1, 5000, 3), (3, 400, 7), (31, 40, 2), (32, 300, 1), (33, 900, 5),
                                            (256, 700, 3), (1000, 90, 2), (1024, 3, 4)])
def test_every_tile_once_in_any_order(plan, N, most, columns, order):
    rng = np.random.default_rng(N + most)
    counts = rng.integers(0, most + 1, N) * (rng.random(N) < 0.7)
    counts[rng.integers(N)] = most
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    tiles = -(-counts // 256)
    prefix = np.concatenate([[0], np.cumsum(tiles * columns)]).astype(np.int32)
    js = np.arange(prefix[-1], dtype=np.int32)
    js = {"up": js, "down": js[::-1], "any": rng.permutation(js)}[order].astype(np.int32)
    out = np.full((len(js), 4), -7, dtype=np.int32)
    plan.jobs(ints(offsets), ints(prefix), ints(np.maximum(tiles, 1)), N, int(offsets[-1]), ints(js), len(js),
              out.ctypes.data_as(ctypes.c_void_p))
    hits = np.zeros((offsets[-1], columns), dtype=int)
    for e, block, row0, rows in out:
        assert 0 <= block < columns and rows <= 256
        if rows > 0:
            assert offsets[e] <= row0 and row0 + rows <= offsets[e + 1]
            hits[row0:row0 + rows, block] += 1
    assert (hits == 1).all()


def test_a_range_of_offsets(plan):
    """Offsets outside the rows and descending ones give rows inside, or none."""
    for offsets in ([-9, 70, 20, 999, 60], [2 ** 31 - 1, -2 ** 31, 60, 5, 0]):
        at = np.clip(np.array(offsets, dtype=np.int64), 0, 60)
        counts = np.maximum(at[1:] - at[:-1], 0)
        tiles = -(-counts // 256)
        prefix = np.concatenate([[0], np.cumsum(tiles)])
        out = np.zeros((prefix[-1], 4), dtype=np.int32)
        plan.jobs(ints(offsets), ints(prefix), ints(np.maximum(tiles, 1)), 4, 60, ints(np.arange(prefix[-1])), int(prefix[-1]),
                  out.ctypes.data_as(ctypes.c_void_p))
        live = np.nonzero(counts)[0]
        assert out[:, 0].tolist() == live.tolist()
        assert out[:, 2].tolist() == at[live].tolist() and out[:, 3].tolist() == counts[live].tolist()
