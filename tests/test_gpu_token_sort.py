"""GPU token sort and its gradients (pr2_token_*) against the plain form.

The plan and the sorted rows are compared bit for bit.  Sums over k slots run in 32 bits in slot
order: at most k roundings of partial sums, k 2^-24 sum |g y|, and one rounding of the stored type.
A gate's gradient is a dot product of d terms whose partial sums are at most d / 32 + 40 deep:
(d / 32 + 40) 2^-24 sum |dout y|.
"""
import pytest
import torch

import train_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}  # half a unit in the last place
SHAPES = [  # T, d, N, k
    (1, 1, 1, 1), (1, 7168, 256, 8), (2, 9, 3, 2), (5, 64, 8, 8), (33, 130, 60, 4), (128, 1024, 128, 8),
    (129, 1023, 6, 6), (300, 257, 40, 32), (700, 2048, 128, 8), (1500, 40, 256, 3), (40, 8200, 16, 2), (1500, 9, 250, 8), (4000, 16, 256, 8), (4097, 8, 64, 8), (9000, 4, 7, 3), (7000, 4, 40, 3), (4097, 3, 250, 5),
    (17, 1028, 16, 5), (9, 20001, 16, 5)]


def route(T, N, k, seed, spoil=True):
    g = torch.Generator().manual_seed(seed)
    idx = torch.rand(T, N, generator=g).argsort(1)[:, :k].int().contiguous()
    if spoil and T > 3:
        idx[1] = -1                # a padding token
        idx[2, 0] = N              # out of range
        if k > 1:
            idx[3, k - 1] = idx[3, 0]  # repeated
    return idx


def rows(n, d, dtype, g, shift=0):
    """[n, d] on the GPU that starts `shift` elements into its buffer, with its CPU copy."""
    x = torch.randn(n, d, generator=g).to(DT[dtype])
    buf = torch.empty(n * d + shift, dtype=DT[dtype], device="cuda")
    buf[shift:].view(n, d).copy_(x)
    return buf[shift:].view(n, d), x


def sort(dm, idx, h, x):
    F = dm.T * dm.k
    ints = lambda n: torch.full((n,), -7, dtype=torch.int32, device="cuda")  # noqa: E731
    offsets, perm, inv, status = ints(dm.N + 1), ints(F), ints(F), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.check(B.pr2_token_sort(dm, h, idx, x, offsets, perm, inv, B.alloc_token_workspace(dm), status=status),
            "pr2_token_sort")
    torch.cuda.synchronize()
    return offsets, perm, inv, int(status.item())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("T,d,N,k", SHAPES)
def test_sort_and_back(T, d, N, k, shift, dtype):
    g = torch.Generator().manual_seed(T + d + N + k)
    idx = route(T, N, k, T + N)
    want = R.plan(idx.tolist(), N)
    dm, F = B.dims(T, d, N, k, 1, 0, dtype), T * k
    h, h_cpu = rows(T, d, dtype, g, shift)
    x, _ = rows(F, d, dtype, g, shift)
    offsets, perm, inv, status = sort(dm, idx.cuda(), h, x)
    assert offsets.tolist() == want[0] and perm.tolist() == want[1] and inv.tolist() == want[2]
    assert status == (B.PR2_STATUS_BAD_INDEX if want[0][N] < F else 0)
    used, slot = want[0][N], torch.tensor(want[1])
    assert torch.equal(x[:used].cpu(), h_cpu[slot[:used] // k]) and not x[used:].cpu().any()

    # sort_backward and unsort; rows that no slot names hold NaN
    y, y_cpu = rows(F, d, dtype, g, shift)
    y[used:] = float("nan")
    y_cpu[used:] = float("nan")
    gates = torch.rand(T, k, generator=g)
    picked = R.rows_of(y_cpu, torch.tensor(want[2]), T, k)
    for weights, name in ((None, "backward"), (gates, "unsort")):
        out, _ = rows(T, d, dtype, g, shift)
        if weights is None:
            B.check(B.pr2_token_sort_backward(dm, y, inv, out))
        else:
            B.check(B.pr2_token_unsort(dm, y, gates.cuda(), inv, out))
        terms = picked * (1.0 if weights is None else gates.double()[..., None])
        exact = terms.sum(1)
        err = (out.cpu().double() - exact).abs()
        assert (err <= EPS[dtype] * exact.abs() * (1 + 2 ** -6) + k * 2.0 ** -24 * terms.abs().sum(1)).all(), name

    # unsort_backward
    dout, dout_cpu = rows(T, d, dtype, g, shift)
    dy, _ = rows(F, d, dtype, g, shift)
    dgates = torch.full((T, k), 7.0, device="cuda")
    B.check(B.pr2_token_unsort_backward(dm, dout, y, gates.cuda(), inv, offsets, dy, dgates))
    grow = gates.reshape(-1)[slot[:used]].double()[:, None] * dout_cpu[slot[:used] // k].double()
    assert ((dy[:used].cpu().double() - grow).abs() <= EPS[dtype] * (1 + 2 ** -6) * grow.abs()).all()
    assert not dy[used:].cpu().any()
    prod = picked * dout_cpu.double()[:, None]
    assert ((dgates.cpu().double() - prod.sum(2)).abs() <= (d / 32 + 40) * 2.0 ** -24 * prod.abs().sum(2)).all()
    assert not dgates.cpu().reshape(-1)[torch.tensor(want[2]) < 0].any()


def test_plan_alone_and_rows_by_a_plan_given():
    T, d, N, k = 90, 96, 16, 4
    idx = route(T, N, k, 3)
    dm = B.dims(T, d, N, k, 1, 0, "bf16")
    h, h_cpu = rows(T, d, "bf16", torch.Generator().manual_seed(0))
    offsets, perm, inv, _ = sort(dm, idx.cuda(), None, None)
    want = R.plan(idx.tolist(), N)
    assert (offsets.tolist(), perm.tolist(), inv.tolist()) == want
    x = torch.full((T * k, d), 7.0, dtype=torch.bfloat16, device="cuda")
    B.check(B.pr2_token_sort(dm, h, None, x, offsets, None, inv))
    used = want[0][N]
    assert torch.equal(x[:used].cpu(), h_cpu[torch.tensor(want[1])[:used] // k]) and not x[used:].cpu().any()


@pytest.mark.parametrize("d", [64, 65])
def test_a_plan_with_rows_out_of_range_is_not_followed(d):
    T, N, k = 20, 8, 4
    dm = B.dims(T, d, N, k, 1, 0, "bf16")
    idx = route(T, N, k, 5, spoil=False)
    offsets, perm, inv, _ = sort(dm, idx.cuda(), None, None)
    bad = inv.clone()
    bad[5], bad[17], bad[60] = T * k, -3, 2 ** 31 - 1
    clean = torch.where((bad < 0) | (bad >= T * k), -1, bad)
    g = torch.Generator().manual_seed(1)
    h, y, dout = rows(T, d, "bf16", g)[0], rows(T * k, d, "bf16", g)[0], rows(T, d, "bf16", g)[0]
    gates = torch.rand(T, k, generator=g).cuda()
    got = []
    for plan in (bad, clean):
        x, dy = (torch.zeros(T * k, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dh, out = torch.empty_like(h), torch.empty_like(h)
        dg = torch.empty_like(gates)
        B.check(B.pr2_token_sort(dm, h, None, x, offsets, None, plan))
        B.check(B.pr2_token_sort_backward(dm, y, plan, dh))
        B.check(B.pr2_token_unsort(dm, y, gates, plan, out))
        B.check(B.pr2_token_unsort_backward(dm, dout, y, gates, plan, offsets, dy, dg))
        got.append([v.cpu() for v in (x, dh, out, dy, dg)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_every_slot_invalid():
    T, d, N, k = 50, 128, 8, 2
    dm = B.dims(T, d, N, k, 1, 0, "bf16")
    g = torch.Generator().manual_seed(2)
    x, _ = rows(T * k, d, "bf16", g)
    offsets, perm, inv, status = sort(dm, torch.full((T, k), -1, dtype=torch.int32, device="cuda"), rows(T, d, "bf16", g)[0], x)
    assert status == B.PR2_STATUS_BAD_INDEX and not offsets.cpu().any() and not x.cpu().any()
    assert (perm == -1).all() and (inv == -1).all()
    y = torch.full((T * k, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, dy = torch.ones(T, d, dtype=torch.bfloat16, device="cuda"), torch.ones_like(y)
    dg, gates = torch.ones(T, k, device="cuda"), torch.ones(T, k, device="cuda")
    B.check(B.pr2_token_unsort(dm, y, gates, inv, out))
    B.check(B.pr2_token_unsort_backward(dm, out, y, gates, inv, offsets, dy, dg))
    assert not out.cpu().any() and not dy.cpu().any() and not dg.cpu().any()


def test_agrees_with_the_layer_forward():
    """The plan is pr2_moe_forward's: counts are the offsets' steps, perm the same."""
    T, d, N, k, m = 200, 256, 16, 4, 192
    g = torch.Generator().manual_seed(6)
    idx = route(T, N, k, 6, spoil=False).cuda()
    dm = B.dims(T, d, N, k, m, 0, "bf16")
    h = torch.randn(T, d, generator=g).bfloat16().cuda()
    W = [(0.05 * torch.randn(N, a, b, generator=g)).bfloat16().cuda() for a, b in ((m, d), (m, d), (d, m))]
    counts = torch.empty(N, dtype=torch.int32, device="cuda")
    perm = torch.empty(T * k, dtype=torch.int32, device="cuda")
    out = torch.empty_like(h)
    gates = torch.rand(T, k, generator=g).cuda()
    B.check(B.pr2_moe_forward(dm, h, idx, gates, *W, None, None, None, out, counts, perm, B.alloc_workspace(dm)))
    offsets, perm2, inv, _ = sort(dm, idx, None, None)
    assert torch.equal(perm, perm2) and torch.equal(counts, offsets.diff())


@pytest.mark.parametrize("T,N,k", [(200000, 128, 8), (600000, 60, 8), (1100000, 5, 4)])
def test_plans_of_many_slots(T, N, k):
    """Sizes where the plan is made by blocks, and (over 4 M slots) by the layer's dispatch."""
    g = torch.Generator(device="cuda").manual_seed(T)
    idx = torch.rand(T, N, generator=g, device="cuda").topk(k, 1).indices.int().contiguous()
    idx[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    flat = idx.reshape(-1).long()
    ranked, order = torch.sort(torch.where(flat >= 0, flat, N), stable=True)
    offsets, perm, inv, status = sort(B.dims(T, 8, N, k, 1, 0, "bf16"), idx, None, None)
    want = torch.searchsorted(ranked, torch.arange(N + 1, device="cuda"))
    assert torch.equal(offsets.long(), want) and status == B.PR2_STATUS_BAD_INDEX
    used = int(want[N])
    assert torch.equal(perm[:used].long(), order[:used]) and (perm[used:] == -1).all()
    place = torch.full_like(flat, -1)
    place[order[:used]] = torch.arange(used, device="cuda")
    assert torch.equal(inv.long(), place)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_batches_and_another_stream(dtype):
    """Row offsets past 2^31 elements, twice and on a side stream with the same bits."""
    T, d, N, k = 40000, 7168, 64, 8
    if dtype == "fp32":
        T = 10000
    dm = B.dims(T, d, N, k, 1, 0, dtype)
    idx = torch.rand(T, N, device="cuda").argsort(1)[:, :k].int().contiguous()
    h = torch.randn(T, d, device="cuda").bfloat16().to(DT[dtype])  # 8 bits: sums of 8 equal rows are exact
    x = torch.empty(T * k, d, dtype=DT[dtype], device="cuda")
    offsets, perm, inv, _ = sort(dm, idx, h, x)
    assert torch.equal(perm[inv.long()], torch.arange(T * k, dtype=torch.int32, device="cuda"))
    for part in torch.arange(T * k, device="cuda").split(40000):
        assert torch.equal(x[part], h[perm[part].long() // k])
    one, two = torch.empty_like(h), torch.empty_like(h)
    gates = torch.full((T, k), 0.125, device="cuda")
    B.check(B.pr2_token_unsort(dm, x, gates, inv, one))  # eight equal rows: exact
    assert torch.equal(one, h)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.check(B.pr2_token_sort_backward(dm, x, inv, two))
    torch.cuda.synchronize()
    assert torch.equal(two, (8 * h.float()).to(DT[dtype]))
    dy, dg = x, torch.empty_like(gates)
    y = torch.ones_like(x)
    B.check(B.pr2_token_unsort_backward(dm, h, y, gates, inv, offsets, dy, dg))
    for part in torch.arange(T * k, device="cuda").split(40000):
        assert torch.equal(dy[part], (0.125 * h[perm[part].long() // k].float()).to(DT[dtype]))
    want = h.double().sum(1)
    assert ((dg.double() - want[:, None]).abs() <= (d / 32 + 40) * 2.0 ** -24 * h.double().abs().sum(1)[:, None]).all()


def test_gate_and_row_gradients_against_differences():
    """The weighted sum is linear in the gates and in the rows, so a difference quotient over a step
    of 1 is exact but for 32-bit rounding (tolerances as above)."""
    T, d, N, k = 6, 40, 8, 3
    dm = B.dims(T, d, N, k, 1, 0, "fp32")
    g = torch.Generator().manual_seed(9)
    offsets, perm, inv, _ = sort(dm, route(T, N, k, 9).cuda(), None, None)
    y, dout, gates = (torch.randn(*s, generator=g).cuda() for s in ((T * k, d), (T, d), (T, k)))
    dy, dg = torch.empty_like(y), torch.empty_like(gates)
    B.check(B.pr2_token_unsort_backward(dm, dout, y, gates, inv, offsets, dy, dg))

    def value(y, gates):
        out = torch.empty(T, d, device="cuda")
        B.check(B.pr2_token_unsort(dm, y, gates, inv, out))
        return float((out.double() * dout.double()).sum())

    base = value(y, gates)
    for t in range(T):
        for s in range(k):
            moved = gates.clone()
            moved[t, s] += 1.0
            assert abs(value(y, moved) - base - float(dg[t, s])) < 1e-4
    for r in (0, 7, T * k - 1):
        for c in (0, 39):
            moved = y.clone()
            moved[r, c] += 1.0
            assert abs(value(moved, gates) - base - float(dy[r, c])) < 1e-4


def test_captured_in_a_graph():
    T, d, N, k = 100, 64, 8, 2
    dm = B.dims(T, d, N, k, 1, 0, "bf16")
    g = torch.Generator().manual_seed(4)
    idx, h = route(T, N, k, 4, spoil=False).cuda(), rows(T, d, "bf16", g)[0]
    x = torch.empty(T * k, d, dtype=torch.bfloat16, device="cuda")
    want = sort(dm, idx, h, x)
    keep, dh = x.clone(), torch.empty_like(h)
    offsets, perm, inv = (torch.zeros_like(v) for v in want[:3])
    ws = B.alloc_token_workspace(dm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.check(B.pr2_token_sort(dm, h, idx, x, offsets, perm, inv, ws))
        B.check(B.pr2_token_sort_backward(dm, x, inv, dh))
    x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x, keep) and torch.equal(perm, want[1]) and torch.equal(dh, (2 * h.float()).bfloat16())
