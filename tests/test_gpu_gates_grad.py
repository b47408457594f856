"""GPU gradient of the replay gates (pr2_replay_gates_backward) against the plain 64-bit form.

dlogits_j = rho_j (dr_j - G): dr and G are sums of at most k <= 32 products, so the error is below
(k + 8) 2^-24 of rho_j (|dr_j| + sum |dgates rho|); renormalised, dr and G carry 1/S.
"""
import pytest
import torch

import train_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


def case(T, N, k, seed):
    g = torch.Generator().manual_seed(seed)
    probs = torch.softmax(2 * torch.randn(T, N, generator=g), 1)
    idx = torch.rand(T, N, generator=g).argsort(1)[:, :k].int().contiguous()
    if T > 4:
        idx[1] = -1
        idx[2, 0] = N
        if k > 1:
            idx[3, 1] = idx[3, 0]
    return probs, idx, torch.randn(T, k, generator=g)


def call(probs, idx, dg, norm):
    T, N = probs.shape
    dm = B.dims(T, 1, N, idx.shape[1], 1, 0, "fp32", B.PR2_F_NORMALIZE_TOPK if norm else 0)
    out = torch.full((T, N), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.check(B.pr2_replay_gates_backward(dm, probs.cuda(), idx.cuda(), dg.cuda(), out, status=status))
    return out.cpu(), int(status.item())


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("T,N,k", [(1, 1, 1), (1, 8, 8), (7, 5, 3), (33, 60, 4), (130, 128, 8), (65, 256, 32),
                                   (9, 33, 32), (300, 129, 1), (12, 250, 7),
                                   (77, 32, 8), (50, 24, 9), (61, 64, 16), (40, 64, 17), (1000, 60, 8), (3, 4, 4), (2000, 256, 8)])
def test_matches_the_formula(T, N, k, norm):
    probs, idx, dg = case(T, N, k, T + N + k)
    got, status = call(probs, idx, dg, norm)
    want = R.gates_backward(probs, idx, dg, norm)
    ok = (idx >= 0) & (idx < N)
    S = torch.gather(probs, 1, idx.clamp(0, N - 1).long()).double()
    size = dg.double().abs().max(1, keepdim=True).values * (2 + k)
    if norm:
        size = size / torch.where(ok, S, 2.0).min(1, keepdim=True).values.clamp(max=1.0)
    assert ((got.double() - want).abs() <= (k + 8) * 2.0 ** -24 * probs.double() * size).all()
    assert status == (B.PR2_STATUS_BAD_INDEX if T > 4 else 0)
    if T > 4:
        assert not got[1].any()


def test_differences_through_the_replay_gates():
    """Against differences of the gates that pr2_route_replay computes (fp32: gates good to 1e-6, over
    a step of 2^-5: 1e-4; the step's own error is below 2^-10 / 6 of a gate's scale)."""
    T, d, N, k = 3, 8, 8, 2
    g = torch.Generator().manual_seed(3)
    for norm in (False, True):
        flags = B.PR2_F_NORMALIZE_TOPK if norm else 0
        dm = B.dims(T, d, N, k, 1, 0, "fp32", flags)
        W = torch.eye(N, d).cuda()  # logits are h itself
        h, dg = torch.randn(T, d, generator=g), torch.randn(T, k, generator=g)
        idx = torch.rand(T, N, generator=g).argsort(1)[:, :k].int().contiguous().cuda()

        def gates(h):
            out, probs = torch.empty(T, k, device="cuda"), torch.empty(T, N, device="cuda")
            B.check(B.pr2_route_replay(dm, h.cuda(), W, idx, out, probs))
            return out.cpu().double(), probs

        got, _ = call(gates(h)[1].cpu(), idx.cpu(), dg, norm)
        step = 2.0 ** -5
        for j in range(N):
            up, dn = h.clone(), h.clone()
            up[:, j] += step
            dn[:, j] -= step
            diff = ((gates(up)[0] - gates(dn)[0]) * dg.double()).sum(1) / (2 * step)
            assert ((diff - got[:, j].double()).abs() <= 2e-3).all()


def test_in_a_row_whose_selected_probabilities_vanish():
    probs = torch.zeros(2, 8)
    probs[:, 0] = 1.0
    idx = torch.tensor([[3, 4], [0, 5]], dtype=torch.int32)
    for norm in (False, True):
        got, status = call(probs, idx, torch.ones(2, 2), norm)
        assert status == 0 and torch.equal(got, R.gates_backward(probs, idx, torch.ones(2, 2), norm).float())


def test_an_invalid_slot_may_carry_anything():
    probs, idx, dg = case(6, 16, 4, 1)
    a, _ = call(probs, idx, dg, False)
    dg[1] = float("nan")
    dg[2, 0] = float("inf")
    dg[3, 1] = float("nan")
    b, _ = call(probs, idx, dg, False)
    assert torch.equal(a, b)
