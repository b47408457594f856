"""Policy loss: what holds exactly, whatever 32 bits do."""
import math

import pytest
import torch

from test_gpu_policy_loss import call

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
