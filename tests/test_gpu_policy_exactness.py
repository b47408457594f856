"""Policy loss: what holds exactly, whatever 32 bits do, and confident targets.

Confident targets (a row's other entries add nothing to a 32-bit sum): the log-probability is
(y - n) log 2 - log part with one power of two (2^-22, as its documentation bounds it), one logarithm (1 unit,
2^-24 of at most 0.7) and one fused product (2^-25), the term's own exponent taken back out of the sum: 6e-7.
The entropy is the difference of log l and the mean exponent, of at most 40, which has three roundings of
2^-24: 8e-6.
"""
import math

import pytest
import torch

from test_gpu_policy_loss import DT, call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1, 8, 3000])
def test_a_row_of_one_entry_is_certain_at_any_height(V):
    """inv_temp log2 e is 1 in 32 bits, so integer logits are their own exponents and their powers exact: what
    is left is what the two constants' rounding does, which has to cancel in (y - n) log 2 - log part."""
    inv_temp = float(torch.tensor(math.log(2.0), dtype=torch.float32))
    heights = torch.arange(-60, 121).float()
    T = heights.numel()
    z = torch.full((T, V), -math.inf)
    target = torch.arange(T) % V
    z[torch.arange(T), target] = heights
    c = dict(buf=z.flatten(), shift=0, ld=V, V=V, logits=z, target=target.int(), advantage=torch.ones(T),
             weight=torch.full((T,), 1.0 / T), logp_old=None, logp_ref=None)
    got = call(c, "fp32", names=("weight",), inv_temp=inv_temp)
    assert not got["logp"].any(), float(got["logp"].abs().max())
    assert not got["entropy"].any(), float(got["entropy"].abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [64, 1000, 5001, 40001])
def test_confident_targets(V, dtype):
    tops = torch.cat([torch.arange(8.0, 27.5, 0.0625), torch.tensor([27.3125, 25.1875, 15.0])])
    T = tops.numel()
    g = torch.Generator().manual_seed(V)
    z = -20 + torch.randn(T, V, generator=g)
    target = torch.randint(0, V, (T,), generator=g).int()
    z[torch.arange(T), target.long()] = tops
    z = z.to(DT[dtype])
    c = dict(buf=z.flatten(), shift=0, ld=V, V=V, logits=z, target=target, advantage=torch.ones(T),
             weight=torch.full((T,), 1.0 / T), logp_old=None, logp_ref=None)
    got = call(c, dtype, names=("weight",))
    lp = torch.log_softmax(z.double(), 1)
    want = lp[torch.arange(T), target.long()]
    assert (got["logp"] <= 0).all(), float(got["logp"].max())
    assert ((got["logp"].double() - want).abs() <= 6e-7).all()
    entropy = -(lp.exp() * lp).sum(1)
    assert (got["entropy"] >= 0).all(), float(got["entropy"].min())
    assert ((got["entropy"].double() - entropy).abs() <= 8e-6).all()
