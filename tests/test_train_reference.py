"""The plain 64-bit forms that the GPU tests compare with, pinned on the CPU: gradients against
central differences, the loss against closed forms, the checkpoint against its error bound."""
import math

import pytest
import torch

import train_reference as R


def _policy_case(seed, T=5, V=11):
    g = torch.Generator().manual_seed(seed)
    logits = 2 * torch.randn(T, V, generator=g, dtype=torch.float64)
    target = torch.randint(0, V, (T,), generator=g)
    base = torch.log_softmax(logits * 0.8, 1)[torch.arange(T), target]
    kw = dict(target=target, advantage=torch.randn(T, generator=g),
              weight=torch.tensor([0.3, 0.0, 0.2, 0.4, 0.1]),
              logp_old=base - torch.tensor([0.05, 0.0, 0.5, -0.5, -0.1]),
              logp_ref=base + 0.3 * torch.randn(T, generator=g), inv_temp=0.8, clip_low=0.2,
              clip_high=0.28, kl_coef=0.1)
    return logits, kw


@pytest.mark.parametrize("seed", [0, 1, 2, 3])
def test_policy_gradient_is_the_difference_quotient(seed):
    logits, kw = _policy_case(seed)
    got = R.policy(logits, **kw)["grad"]
    h = 1e-5
    for t in range(logits.shape[0]):
        for v in range(logits.shape[1]):
            up, dn = logits.clone(), logits.clone()
            up[t, v] += h
            dn[t, v] -= h
            diff = (R.policy(up, **kw)["loss"][0] - R.policy(dn, **kw)["loss"][0]) / (2 * h)
            assert abs(float(diff - got[t, v])) < 1e-8  # h^2 times third derivatives, 1e-16 / h


def test_policy_closed_forms():
    # two equal logits: p = 1/2, entropy log 2; ratio 1 and advantage A give loss -A
    one = R.policy(torch.zeros(1, 2), torch.tensor([1]), torch.tensor([3.0]))
    assert math.isclose(float(one["loss"][0]), -3.0) and math.isclose(float(one["entropy"][0]), math.log(2))
    assert torch.allclose(one["grad"], torch.tensor([[1.5, -1.5]], dtype=torch.float64))
    # ratio e > 1 + clip_high with a positive advantage: clipped, no gradient
    cut = R.policy(torch.zeros(1, 2), torch.tensor([1]), torch.tensor([3.0]), clip_high=0.28,
                   logp_old=torch.tensor([math.log(0.5) - 1.0]))
    assert math.isclose(float(cut["loss"][0]), -3.84) and float(cut["loss"][3]) == 1.0
    assert not cut["grad"].any()
    # the KL term vanishes, with its gradient, where the policies agree
    same = R.policy(torch.zeros(1, 2), torch.tensor([1]), torch.tensor([0.0]), kl_coef=1.0,
                    logp_ref=torch.tensor([math.log(0.5)], dtype=torch.float64))
    assert abs(float(same["loss"][2])) < 1e-30 and same["grad"].abs().max() < 1e-15


@pytest.mark.parametrize("norm", [False, True])
def test_gate_gradient_is_the_difference_quotient(norm):
    g = torch.Generator().manual_seed(5)
    T, N = 4, 9
    p = torch.randn(T, N, generator=g, dtype=torch.float64)
    idx = torch.tensor([[0, 3, 8], [2, 2, 5], [-1, 9, 4], [-1, -1, 9]])
    dg = torch.randn(T, 3, generator=g, dtype=torch.float64)

    def value(p):
        rho, total = torch.softmax(p, 1), 0.0
        for t in range(T):
            row = idx[t].tolist()
            ok = [s for s in range(3) if 0 <= row[s] < N and row[s] not in row[:s]]
            gs = [rho[t, row[s]] for s in ok]
            S = sum(gs) if norm else 1.0
            total += sum(dg[t, s] * v / S for s, v in zip(ok, gs))
        return float(total)

    got = R.gates_backward(torch.softmax(p, 1), idx, dg, norm)
    h = 1e-5
    for t in range(T):
        for j in range(N):
            up, dn = p.clone(), p.clone()
            up[t, j] += h
            dn[t, j] -= h
            assert abs((value(up) - value(dn)) / (2 * h) - float(got[t, j])) < 1e-8


def test_swiglu_gradient_is_the_difference_quotient():
    gen = torch.Generator().manual_seed(1)
    g, u, d = (3 * torch.randn(64, generator=gen, dtype=torch.float64) for _ in range(3))
    dg, du, act = R.swiglu_backward(g, u, d)
    h = 1e-5
    assert torch.allclose(dg, d * (R.swiglu(g + h, u) - R.swiglu(g - h, u)) / (2 * h), atol=1e-7)
    assert torch.allclose(du, d * (R.swiglu(g, u + h) - R.swiglu(g, u - h)) / (2 * h), atol=1e-7)
    assert torch.equal(act, g * torch.sigmoid(g) * u)


def test_checkpoint_error_is_within_half_a_scale():
    x = torch.randn(7, 300, generator=torch.Generator().manual_seed(2)) * torch.logspace(-3, 3, 300)
    q, scale = R.hold(x)
    bound = 0.5 * scale.double()[:, torch.arange(300) // R.GROUP]
    # (1 + 2^-21): the 32-bit roundings of scale and reciprocal, at q = 127
    assert ((R.held(q, scale) - x.double()).abs() <= bound * (1 + 2 ** -21) + 127 * bound * 2 ** -22).all()
    assert int(q.abs().max()) == 127


def test_plan_is_a_stable_sort():
    offsets, perm, inv = R.plan([[1, 0], [1, 1], [5, 1]], 3)
    assert offsets == [0, 1, 4, 4] and perm == [1, 0, 2, 5, -1, -1] and inv == [1, 0, 2, -1, -1, 3]
