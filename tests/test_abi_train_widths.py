"""Token widths that the kernels' 32-bit column numbers cannot count are refused on the host (no GPU)."""
import ctypes

import pytest

from paper_2606_00395_gb300 import binding as B
from paper_2606_00395_gb300 import build

P = ctypes.c_void_p(256)
UNSUPPORTED = 2


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [(1 << 30) + 1, (1 << 31) - 200, (1 << 31) - 1])
def test_widths_past_the_limit(lib, d, dtype):
    dm = ctypes.byref(B.dims(1, d, 1, 1, 1, 0, dtype))
    assert lib.pr2_token_sort_workspace_bytes(dm) == 0
    assert lib.pr2_token_sort(dm, P, P, P, P, P, P, P, ctypes.c_size_t(1 << 30), None, None) == UNSUPPORTED
    assert lib.pr2_token_sort_backward(dm, P, P, P, None) == UNSUPPORTED
    assert lib.pr2_token_unsort(dm, P, P, P, P, None) == UNSUPPORTED
    assert lib.pr2_token_unsort_backward(dm, P, P, P, P, P, P, P, None) == UNSUPPORTED


def test_the_widest_row_is_taken(lib):
    assert B.pr2_token_sort_workspace_bytes(B.dims(1, 1 << 30, 1, 1, 1, 0, "fp32")) > 0
