"""8-bit products of experts of 257 to 384 rows, one tile or two by the length of the sums: both sides of that
border, with the tolerances of the shapes in test_gpu_grouped.py."""
import pytest

import test_gpu_grouped as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("pairs", [1, 2])
@pytest.mark.parametrize("d_in,pad,shift", [(3952, 0, 0), (3968, 0, 0), (3984, 0, 0), (4096, 16, 16), (4097, 0, 3)])
def test_8bit(d_in, pad, shift, pairs, whole, dtype):
    G.test_8bit(([257, 300, 0, 383, 384, 385, 40], d_in, 72, pad, 0, shift), pairs, whole, dtype)
