"""Infinities and NaN in the experts' products: the results of the plain form, infinities with their sign, NaN where
an infinity meets 0 or one of the other sign.  The other values are small whole numbers, so the rest is exact."""
import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def bits(dtype, patterns):
    """NaN of any payload."""
    kind = {"fp32": torch.int32, "bf16": torch.int16}[dtype]
    return torch.tensor(patterns, dtype=torch.int64).to(kind).view(R.DT[dtype])


NANS = {"fp32": [0x7f800001, 0x7fc00000, 0x7f80ffff, 0xff800001 - 2 ** 32, 0x7fffffff],
        "bf16": [0x7f81, 0x7fc0, 0xff81 - 2 ** 16, 0x7fff, 0xffff - 2 ** 16]}


def special(t, dtype, g, most):
    """Some values of t infinite, fewer NaN."""
    flat = t.view(-1)
    n = flat.numel()
    at = torch.randperm(n, generator=g)[:most + 5]
    flat[at[:most]] = torch.where(torch.rand(most, generator=g) < 0.5, INF, -INF).to(t.dtype)
    flat[at[most:]] = bits(dtype, NANS[dtype])
    return t


def same(got, want):
    want = want.to(got.dtype)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(0, 3e38, -3e38), want.nan_to_num(0, 3e38, -3e38))


def plain(a, b):
    """a @ b in 64 bits, term by term, without a library's order or padding."""
    return (a.double()[:, :, None] * b.double()[None]).sum(1)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("which", ["rows", "matrices", "both"])
@pytest.mark.parametrize("d_in,d_out", [(72, 48), (65, 33), (600, 40)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_products(dtype, d_in, d_out, which, zeros):
    g = torch.Generator().manual_seed(d_in)
    counts = [40, 0, 70, 1]
    off = torch.tensor([0] + counts).cumsum(0).int()
    rows, N, dt = int(off[-1]), 4, R.DT[dtype]

    def make(*s):
        v = torch.randint(1, 3, s, generator=g).float()
        v *= torch.where(torch.rand(s, generator=g) < 0.5, 1.0, -1.0)
        return (v * (torch.rand(s, generator=g) > 0.2) if zeros else v).to(dt)

    x, dy, W = make(rows, d_in), make(rows, d_out), make(N, d_out, d_in)
    if which != "matrices":
        special(x, dtype, g, 20), special(dy, dtype, g, 20)
    if which != "rows":
        special(W, dtype, g, 30)
    dev = [t.cuda() for t in (x, dy, W)]
    y, dx = torch.empty(rows, d_out, dtype=dt, device="cuda"), torch.empty(rows, d_in, dtype=dt, device="cuda")
    dW = torch.empty(N, d_out, d_in, device="cuda")
    dm = B.group_dims(rows, N, d_in, d_out, dtype)
    B.check(B.pr2_grouped_gemm(dm, dev[0], dev[2], off.cuda(), y))
    B.check(B.pr2_grouped_gemm_backward(dm, dev[1], dev[2], off.cuda(), dx))
    B.check(B.pr2_grouped_gemm_weight_grad(dm, dev[1], dev[0], off.cuda(), dW))
    for e, r in R.spans(off, rows):
        same(y[r].cpu(), plain(x[r], W[e].t()))
        same(dx[r].cpu(), plain(dy[r], W[e]))
        same(dW[e].cpu(), plain(dy[r].t(), x[r]))


def test_many_rows_with_one_infinity():
    """It stays one through the chunks that are added up."""
    rows = 3000
    x, dy = torch.ones(rows, 40, device="cuda"), torch.ones(rows, 24, device="cuda")
    x[17, 3], x[2900, 5], dy[1000, 7], x[2000, 9] = INF, -INF, INF, 3.0
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    dW = torch.empty(1, 24, 40, device="cuda")
    B.check(B.pr2_grouped_gemm_weight_grad(B.group_dims(rows, 1, 40, 24, "fp32"), dy, x, off, dW))
    want = torch.full((24, 40), float(rows), device="cuda")
    want[:, 9] += 2
    want[:, 3], want[:, 5] = INF, -INF
    want[7] = INF
    want[7, 5] = NAN
    same(dW[0], want)
