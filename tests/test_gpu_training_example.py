"""The example training step: its layer agrees with the library's own replay forward, its gradients
with automatic differentiation of the same network in 64 bits, and its loss goes down.

Tolerances (norm of the difference over the norm).  fp32: all but the 8-bit checkpoint is exact to
1e-5; a held value is off by at most half of max / 127 and, uniformly spread, by max / 127 / sqrt(12),
with a run's max about 3 times its root mean square 0.7 %, and gate and up enter the gradients of the
experts' weights together: 2e-2.  bf16 rounds about a dozen intermediate tensors by 2^-9 root mean
square on top: 3e-2; the gradient of the router is a difference of gates' gradients: 6e-2.
"""
import importlib.util
import os

import pytest
import torch

from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "replay_training_step.py")
spec = importlib.util.spec_from_file_location("replay_training_step", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def network(W, tokens, idx, rollout, clip=(0.2, 0.28), kl_coef=0.02):
    h = W["embed"][tokens]
    gates = torch.softmax(h @ W["router"].t(), 1).gather(1, idx)
    rows = []
    for s in range(idx.shape[1]):
        e = idx[:, s]
        g = torch.einsum("td,tmd->tm", h, W["gate"][e])
        u = torch.einsum("td,tmd->tm", h, W["up"][e])
        rows.append(torch.einsum("tm,tdm->td", g * torch.sigmoid(g) * u, W["down"][e]))
    out = (gates[..., None] * torch.stack(rows, 1)).sum(1)
    logp = torch.log_softmax((h + out) @ W["head"].t(), 1).gather(1, rollout["actions"].long()[:, None])[:, 0]
    r, A = (logp - rollout["logp"]).exp(), rollout["advantage"]
    part = torch.minimum(r * A, r.clamp(1 - clip[0], 1 + clip[1]) * A)
    gap = rollout["logp"] - logp
    return (-part + kl_coef * (gap.exp() - gap - 1)).mean(), out


@pytest.mark.parametrize("dtype,bound,router", [("fp32", 2e-2, 2e-2), ("bf16", 3e-2, 6e-2)])
def test_gradients_of_every_weight(dtype, bound, router):
    T, d, N, k, m, V = 96, 128, 16, 4, 192, 320
    W, tokens, g = example.init(T, d, N, k, m, V, dtype, seed=3)
    layer = example.ReplayedLayer(T, d, N, k, m, dtype)
    idx, rollout = example.roll_out(W, tokens, layer.dims, g)
    rollout["logp"] = rollout["logp"] + torch.tensor([0.05, -0.06, 0.1])[torch.arange(T) % 3].cuda()
    loss, grads, out = example.loss_and_grads(layer, W, tokens, idx, rollout)

    # the layer's output is that of the library's replay forward
    want = torch.empty_like(out)
    h = W["embed"][tokens]
    gates = torch.empty(T, k, device="cuda")
    B.check(B.pr2_moe_replay_forward(layer.dims, h, W["router"], idx, gates, None, W["gate"], W["up"], W["down"], None,
                                     None, None, want, workspace=B.alloc_workspace(layer.dims)))
    assert float((out.float() - want.float()).norm() / want.float().norm()) < (2e-2 if dtype == "bf16" else 1e-4)

    leaves = {n: v.cpu().double().requires_grad_() for n, v in W.items()}
    ref, _ = network(leaves, tokens.cpu(), idx.long().cpu(),
                     {n: v.cpu().double() if v.is_floating_point() else v.cpu() for n, v in rollout.items() if v is not None})
    ref.backward()
    assert abs(float(loss[0]) - float(ref.detach())) < (1e-5 if dtype == "fp32" else 1e-2)
    for n, got in grads.items():
        exact = leaves[n].grad
        err = float((got.cpu().double() - exact).norm() / exact.norm())
        assert err < (router if n == "router" else bound), (n, err)


def test_a_few_updates_lower_the_loss():
    lines = []
    losses = example.main(steps=6, log=lines.append)
    assert len(lines) == 6 and losses[-1][0] < losses[0][0] - 0.02
    assert all(x[2] >= 0 for x in losses)
