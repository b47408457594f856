"""Gradient of the renormalised gates where the selected experts' probabilities have all but vanished: the
gates are finite there, and so is the gradient g_s (dgates_s - sum_u dgates_u g_u).

Products of k gates (each below 1) with dgates, in 32 bits: (k + 8) 2^-24 of 2 max |dgates|."""
import pytest
import torch

import train_reference as R
from test_gpu_gates_grad import call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e-30, 1e-36, 1e-38, 1e-39, 1e-41, 1e-43])
@pytest.mark.parametrize("N,k", [(8, 2), (60, 4), (64, 16), (33, 5), (250, 7), (256, 32)])
def test_small_sums(N, k, size):
    T = 40
    g = torch.Generator().manual_seed(N + k)
    probs = torch.softmax(torch.randn(T, N, generator=g), 1)
    idx = torch.rand(T, N, generator=g).argsort(1)[:, :k].int().contiguous()
    small = size * (0.5 + torch.rand(T, k, generator=g, dtype=torch.float64))
    probs.scatter_(1, idx.long(), small.float())
    dg = 1000 * torch.randn(T, k, generator=g)
    got, status = call(probs, idx, dg, True)
    want = R.gates_backward(probs, idx, dg, True)
    assert status == 0 and torch.isfinite(got).all()
    bound = (k + 8) * 2.0 ** -24 * 2 * dg.abs().max(1, keepdim=True).values.double()
    assert ((got.double() - want).abs() <= bound).all(), float((got.double() - want).abs().max())


@pytest.mark.parametrize("N,k", [(8, 2), (33, 5)])
def test_sums_that_are_no_number_are_not_hidden(N, k):
    probs = torch.full((2, N), 1.0 / N)
    idx = torch.arange(k).int().repeat(2, 1).contiguous()
    probs[1, 0] = float("nan")
    got, _ = call(probs, idx, torch.ones(2, k), True)
    assert torch.isfinite(got[0]).all() and torch.isnan(got[1, 0])
