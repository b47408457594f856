"""Long fp32 sums of terms of one sign in the experts' products: at most 16 MMAs in turn in one accumulator, then
rounded additions.

An accumulator that cuts off loses half a step in the mean: 2^-24 = U of what it holds, which after i of 16 MMAs is
i / 16 of its sum, so 8.5 U of it on average at most; the roundings have no mean and leave less than 1 U in the mean of
thousands of results.  A single result is off by at most 2 U for each of the 16 MMAs, U for each addition, and 1.25 U of
its terms.
"""
import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


def check(got, want, K):
    err = (got.double() - want) / want
    assert err.abs().max() <= (2 * 16 + K / 256 + 1 + 1.25) * R.U
    assert err.mean().abs() <= 9.5 * R.U


@pytest.mark.parametrize("K", [8192, 5001])
@pytest.mark.parametrize("d", [64, 75])
def test_sums_of_one_sign(K, d):
    g = torch.Generator(device="cuda").manual_seed(K)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    off = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    x, W, y = rand(64, K), rand(1, d, K), torch.empty(64, d, device="cuda")
    B.check(B.pr2_grouped_gemm(B.group_dims(64, 1, K, d, "fp32"), x, W, off, y))
    check(y, R.grouped(x, W, [0, 64])[0], K)
    dy, W, dx = [rand(64, K) for _ in range(2)], [rand(1, K, d) for _ in range(2)], torch.empty(64, d, device="cuda")
    B.check(B.pr2_grouped_gemm_backward(B.group_dims(64, 1, d, K, "fp32"), dy[0], W[0], off, dx, dy[1], W[1]))
    check(dx, R.grouped_backward(dy, W, [0, 64])[0], 2 * K)
    dy, x, dW = rand(K, 64), rand(K, d), torch.empty(1, 64, d, device="cuda")
    all_rows = torch.tensor([0, K], dtype=torch.int32, device="cuda")
    B.check(B.pr2_grouped_gemm_weight_grad(B.group_dims(K, 1, d, 64, "fp32"), dy, x, all_rows, dW))
    check(dW, R.grouped_weight_grad(dy, x, [0, K])[0], K)
