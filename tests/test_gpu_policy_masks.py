"""Policy loss of rows whose masked entries hold large finite numbers, against the plain 64-bit form
(tolerances as in test_gpu_policy_loss)."""
import math

import pytest
import torch

from test_gpu_policy_loss import DT, call, check, make

pytestmark = pytest.mark.gpu
VALUES = [-1e4, -3e5, -1e10, -1e15, -1e20, -1e30, -1e38]


def masked(T, V, dtype, seed, mask, value, shift=0, pad=0, inv_temp=1.0):
    """Entries of `mask` [T, V] but the targets hold `value`; the old and the reference policy's
    log-probabilities follow from that."""
    c = make(T, V, dtype, seed, pad=pad, shift=shift, std=1.0)
    at, a = torch.arange(T), c["target"].long()
    keep = c["logits"][at, a].clone()
    c["logits"][:, :V][mask] = value
    whole = mask.all(1)
    c["logits"][at, a] = torch.where(whole, c["logits"].new_full((T,), value), keep)
    lp = torch.log_softmax(c["logits"][:, :V].double() * inv_temp, 1)[at, a]
    c["weight"][:] = 1.0 / T
    c["logp_old"], c["logp_ref"] = (lp - 0.05).float(), (lp + 0.1).float()
    return c


def some_masks(T, V, seed):
    """A range of the vocabulary, each entry by chance, all but a few, whole rows."""
    g = torch.Generator().manual_seed(seed)
    v, t = torch.arange(V), torch.arange(T)[:, None]
    share = torch.rand(T, V, generator=g)
    kinds = [(v >= V // 3).expand(T, V), (v < V // 2).expand(T, V), share < 0.5, share < 0.97,
             torch.ones(T, V, dtype=torch.bool)]
    out = torch.zeros(T, V, dtype=torch.bool)
    for i, k in enumerate(kinds):
        out = torch.where(t % len(kinds) == i, k, out)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("value", VALUES)
@pytest.mark.parametrize("T,V,shift,inv_temp", [(10, 64, 0, 1.0), (10, 1000, 0, 1.0), (10, 1003, 1, 0.7),
                                                (10, 9000, 0, 1.3), (10, 40001, 1, 1.0)])
def test_entries_at_a_large_negative_number(T, V, shift, inv_temp, value, dtype):
    c = masked(T, V, dtype, V, some_masks(T, V, V), value, shift, inv_temp=inv_temp)
    kw = dict(clip_high=0.28, kl_coef=0.05, inv_temp=inv_temp)
    check(c, call(c, dtype, **kw), dtype, **kw)


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("value", [-1e10, -1e30])
def test_in_large_batches(value, grad):
    T, V = 500, 5003
    c = masked(T, V, "bf16", 3, some_masks(T, V, 4), value)
    kw = dict(clip_high=0.28, kl_coef=0.05)
    check(c, call(c, "bf16", grad=grad, **kw), "bf16", **kw)


@pytest.mark.parametrize("offset", [-3e7, -5e6, -726817.0, 1e4, 726600.0, 726817.0, 727000.0, 1e6, 3e7])
@pytest.mark.parametrize("V", [300, 9000])
def test_rows_far_from_zero(V, offset):
    """fp32 logits whose scaled values lie about 2^20 and far beyond: their differences are as exact as ever."""
    T = 8
    c = make(T, V, "fp32", 6, std=1.0)
    grid = 2.0 if abs(offset) > 1e7 else 0.5
    c["logits"][:] = (c["logits"] / grid * 4).round() * grid + offset
    lp = torch.log_softmax(c["logits"].double(), 1)[torch.arange(T), c["target"].long()]
    c["weight"][:] = 1.0 / T
    c["logp_old"], c["logp_ref"] = (lp - 0.05).float(), (lp + 0.1).float()
    kw = dict(kl_coef=0.05)
    check(c, call(c, "fp32", **kw), "fp32", **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("inv_temp", [0.7, 1.0, 1.3])
@pytest.mark.parametrize("T,V,shift", [(6, 21, 1), (6, 301, 3), (6, 999, 1), (6, 5003, 1), (6, 32001, 5), (500, 5003, 0)])
def test_first_and_last_entries_at_the_lowest_value(T, V, shift, inv_temp, dtype):
    """Only a few entries at either end, most of them outside the row's whole vectors."""
    v = torch.arange(V)
    mask = ((v < 3) | (v >= V - 3)).expand(T, V)
    value = torch.finfo(DT[dtype]).min
    c = masked(T, V, dtype, V, mask, value, shift, inv_temp=inv_temp)
    # (a target at either end keeps its logit, so the others of that end are the masked ones)
    kw = dict(clip_high=0.28, kl_coef=0.05, inv_temp=inv_temp)
    check(c, call(c, dtype, **kw), dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [300, 9001])
def test_a_target_at_the_lowest_value(V, dtype):
    """Its log-probability is that number, which is finite although its multiple by log2 e is not."""
    c = make(4, V, dtype, 9, std=1.0)
    c["weight"][:] = 0.25
    c["advantage"][:] = torch.tensor([1.0, -1.0, 2.0, 0.0])
    for t in (1, 2, 3):
        c["logits"][t, c["target"][t].long()] = torch.finfo(DT[dtype]).min
    got = call(c, dtype, names=("weight", "logp_old"))
    assert torch.isfinite(got["logp"]).all() and not got["grad"][1:].any()
    check(c, got, dtype, names=("weight", "logp_old"))
    assert math.isclose(float(got["logp"][1]), torch.finfo(DT[dtype]).min, rel_tol=1e-6)
