"""GPU SwiGLU with an 8-bit checkpoint, and its backward pass, against the plain form.

q and scale are compared bit for bit with the format's own 32-bit roundings.  The sigmoid's exponential
is good to a few 2^-22 plus the rounding of its argument (2^-24 |g|, |g| < 80 where it matters): 1e-5
relative; then one rounding of the stored type.  dgate's factor 1 + g (1 - s) cancels near g = -1.28,
so its error is relative to |dact u s| (1 + |g|).
"""
import math

import pytest
import torch

import train_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -23}


def place(x, ld, shift):
    """x [R, m] with row stride ld, `shift` elements into a GPU buffer."""
    Rn, m = x.shape
    buf = torch.full((Rn * ld + shift + 8,), 7.0, dtype=x.dtype, device="cuda")
    v = buf[shift:shift + Rn * ld].view(Rn, ld)[:, :m]
    v.copy_(x)
    return v


def inputs(Rn, m, dtype, seed, std=3.0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.where(torch.rand(2 * m, generator=g) < 0.02, 20.0, 1.0)
    both = (std * torch.randn(Rn, 2 * m, generator=g) * wide).to(DT[dtype])
    return both[:, :m].contiguous(), both[:, m:].contiguous(), torch.randn(Rn, m, generator=g).to(DT[dtype])


def forward(gate, up, dtype, ld, shift):
    Rn, m = gate.shape
    dm = B.act_dims(Rn, m, dtype, ld)
    act = torch.full((Rn, m), 7.0, dtype=DT[dtype], device="cuda")
    q = torch.full((Rn, 2, m), 7, dtype=torch.int8, device="cuda")
    scale = torch.full((Rn, 2, -(-m // 128)), 7.0, device="cuda")
    B.check(B.pr2_swiglu_checkpoint(dm, place(gate, ld, shift), place(up, ld, shift), act, q, scale))
    return act, q, scale


def backward(dact, q, scale, dtype, ld, shift, with_act=True):
    Rn, m = dact.shape
    dm = B.act_dims(Rn, m, dtype, ld)
    dg, du = (place(torch.zeros(Rn, m, dtype=DT[dtype]), ld, shift) for _ in range(2))
    act = torch.full((Rn, m), 7.0, dtype=DT[dtype], device="cuda") if with_act else None
    B.check(B.pr2_swiglu_checkpoint_backward(dm, place(dact, m, shift), q, scale, dg, du, act))
    return dg.cpu().double(), du.cpu().double(), None if act is None else act.cpu().double()


def check_backward(got, q, scale, dact, dtype):
    g, u = (R.held(q[:, i].cpu(), scale[:, i].cpu()) for i in (0, 1))
    d = dact.double()
    want = R.swiglu_backward(g, u, d)
    size = (d * u * torch.sigmoid(g)).abs() * (1 + g.abs()), want[1].abs(), want[2].abs()
    for a, b, s in zip(got, want, size):
        if a is not None:
            assert ((a - b).abs() <= EPS[dtype] * b.abs() + 1e-5 * s + 1e-38).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Rn,m,extra,shift", [
    (1, 1, 0, 0), (1, 127, 0, 0), (3, 128, 0, 0), (5, 129, 1, 1), (2, 768, 768, 0), (700, 768, 0, 0), (33, 1000, 0, 0),
    (33, 1000, 1000, 4), (9, 1001, 0, 0), (4, 4096, 8, 8), (3000, 72, 0, 0), (257, 16, 16, 0), (2, 20000, 0, 0),
    (7, 136, 0, 0), (31, 8, 0, 0), (400, 264, 8, 0)])
def test_checkpoint_and_backward(Rn, m, extra, shift, dtype):
    gate, up, dact = inputs(Rn, m, dtype, Rn + m)
    ld = m + extra
    act, q, scale = forward(gate, up, dtype, ld, shift)
    for i, x in enumerate((gate, up)):
        wq, ws = R.hold(x)
        assert torch.equal(scale[:, i].cpu(), ws) and torch.equal(q[:, i].cpu(), wq)
    want = R.swiglu(gate.double(), up.double())
    assert ((act.cpu().double() - want).abs() <= EPS[dtype] * want.abs() + 1e-5 * want.abs() + 1e-38).all()
    check_backward(backward(dact, q, scale, dtype, ld, shift), q, scale, dact, dtype)
    check_backward(backward(dact, q, scale, dtype, ld, shift, with_act=False), q, scale, dact, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_zeros_tiny_and_non_finite_runs(dtype):
    m = 128 * 8
    gate, up, dact = inputs(4, m, dtype, 1)
    gate[0, :128] = 0.0
    up[0, 128:256] = 1e-35              # below the least held magnitude
    gate[1, 256:384] = torch.finfo(DT[dtype]).max / 4
    up[2, 400], gate[2, 700], up[3, 1023] = math.inf, math.nan, -math.inf
    gate[3, 0:128] = 1.5e-30
    act, q, scale = forward(gate, up, dtype, m, 0)
    for i, x in enumerate((gate, up)):
        wq, ws = R.hold(x)
        assert torch.equal(torch.isnan(scale[:, i].cpu()), torch.isnan(ws))
        assert torch.equal(torch.nan_to_num(scale[:, i].cpu(), 9.0), torch.nan_to_num(ws, 9.0))
        assert torch.equal(q[:, i].cpu(), wq)
    assert float(scale[0, 0, 0]) == 0.0 and float(scale[0, 1, 1]) == 0.0
    dg, du, again = backward(dact, q, scale, dtype, m, 0)
    for r, run in ((2, 3), (2, 5), (3, 7)):  # the runs that held an infinity or a NaN
        assert torch.isnan(dg[r, run * 128:(run + 1) * 128]).all() and torch.isnan(again[r, run * 128:(run + 1) * 128]).all()
    assert torch.isfinite(dg[0]).all() and torch.isfinite(du[0]).all()
    assert not again[0, :256].any()


def test_all_halfway_cases_round_to_even():
    # top 127 makes the factor 1: the values are the integers and halves themselves
    x = torch.arange(-127, 127.5, 0.5)
    x = torch.nn.functional.pad(x, (0, 512 - x.numel()), value=127.0)
    x.view(4, 128)[:, 0] = 127.0
    _, q, scale = forward(x[None], x[None], "fp32", 512, 0)
    assert torch.equal(q[0, 0].cpu().float(), torch.round(x)) and torch.equal(q[0, 0], q[0, 1])


def test_large_arguments_saturate():
    gate = torch.tensor([[-1e4, -200.0, -100.0, 100.0, 200.0, 1e4, 3e38, -3e38]])
    up = torch.ones(1, 8)
    act, q, scale = forward(gate, up, "fp32", 8, 0)
    assert torch.isfinite(act).all()
    want = R.swiglu(gate.double(), up.double())
    assert ((act.cpu().double() - want).abs() <= 2e-5 * want.abs() + 1e-38).all()
    gate = torch.tensor([[-100.0, 100.0, 50.0, -50.0, 0.0, 1.0, -1.0, 90.0]])
    _, q, scale = forward(gate, up, "fp32", 8, 0)
    dact = torch.ones(1, 8)
    got = backward(dact, q, scale, "fp32", 8, 0)
    assert all(torch.isfinite(v).all() for v in got)
    check_backward(got, q, scale, dact, "fp32")


def test_gradient_against_differences_of_the_held_activation():
    """Held values are on a grid: with q moved by one, the activation (64 bits, from the checkpoint) moves
    by scale times the gradient up to the second derivative (below 0.5 scale, with central steps a third
    of scale^2), and 1e-5 of 32-bit arithmetic."""
    gate, up, _ = inputs(2, 64, "fp32", 5, std=1.0)
    _, q, scale = forward(gate, up, "fp32", 64, 0)
    q = q.clamp(-126, 126)
    dact = torch.ones(2, 64)
    dg, du, _ = backward(dact, q, scale, "fp32", 64, 0)
    for i, got in ((0, dg), (1, du)):
        two = []
        for sign in (1, -1):
            moved = q.clone().cpu()
            moved[:, i] += sign
            two.append(R.swiglu(*(R.held(moved[:, j], scale[:, j].cpu()) for j in (0, 1))))
        sc = scale[:, i, 0].cpu().double()[:, None]
        other = R.held(q[:, 1 - i].cpu(), scale[:, 1 - i].cpu()).abs()
        assert (((two[0] - two[1]) / (2 * sc) - got).abs() <= (sc ** 2 + 2e-5) * (1 + other)).all()


def test_rows_past_32_bit_offsets_and_another_stream():
    Rn, m = 300000, 7200  # 2.16e9 elements a matrix
    gate = torch.full((Rn, m), 2.0, dtype=torch.bfloat16, device="cuda")
    dm = B.act_dims(Rn, m, "bf16")
    act = torch.empty_like(gate)
    q = torch.empty(Rn, 2, m, dtype=torch.int8, device="cuda")
    scale = torch.empty(Rn, 2, -(-m // 128), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.check(B.pr2_swiglu_checkpoint(dm, gate, gate, act, q, scale))
        assert bool((q == 127).all()) and bool((act == act[0, 0]).all())
        dg, du = torch.empty_like(gate), torch.empty_like(gate)
        B.check(B.pr2_swiglu_checkpoint_backward(dm, gate, q, scale, dg, du, act))
        assert bool((dg == dg[0, 0]).all()) and bool((du == du[0, 0]).all()) and bool((act == act[0, 0]).all())
    torch.cuda.synchronize()
    s = 1 / (1 + math.exp(-2))
    assert math.isclose(float(du[-1, -1]), 4 * s, rel_tol=2 ** -8)
    assert math.isclose(float(dg[-1, -1]), 4 * s * (1 + 2 * (1 - s)), rel_tol=2 ** -8)


def test_activation_again_in_place_of_its_gradient():
    gate, up, dact = inputs(40, 384, "bf16", 8)
    _, q, scale = forward(gate, up, "bf16", 384, 0)
    want = backward(dact, q, scale, "bf16", 384, 0)
    dm = B.act_dims(40, 384, "bf16")
    buf = dact.cuda()
    dg, du = torch.empty_like(buf), torch.empty_like(buf)
    B.check(B.pr2_swiglu_checkpoint_backward(dm, buf, q, scale, dg, du, buf))
    for a, b in zip((dg, du, buf), want):
        assert torch.equal(a.cpu().double(), b)
