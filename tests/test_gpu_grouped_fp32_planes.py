"""Single products of fp32 operands in the experts' products: each output is one term, whose place in the sum goes
through all of them, so that nothing averages out.  A term is the exact product of the upper planes, the sum of
seven products below 2^-6 of it in a truncating accumulator (7 steps of 2 U of that: 0.22 U), a rest below 2^-32
and one rounding: U.  Together 1.25 U.
"""
import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


def full(g, *shape):
    """All 24 bits, any sign, exponents of an everyday range."""
    v = torch.rand(*shape, generator=g, dtype=torch.float64) + 1
    v *= torch.exp2(torch.randint(-12, 12, shape, generator=g).double())
    return torch.where(torch.rand(*shape, generator=g) < 0.5, -v, v).float()


def close(got, want):
    assert ((got.double().cpu() - want).abs() <= 1.25 * R.U * want.abs()).all()


@pytest.mark.parametrize("d_in,d_out", [(64, 40), (200, 136), (515, 33)])
def test_one_term(d_in, d_out):
    g = torch.Generator().manual_seed(d_in)
    rows = 2 * max(d_in, d_out) + 3
    x, dy, W = full(g, rows, d_in), full(g, rows, d_out), full(g, 1, d_out, d_in)
    r, off = torch.arange(rows), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    dm = B.group_dims(rows, 1, d_in, d_out, "fp32")
    one = torch.zeros_like(x)
    one[r, r % d_in] = x[r, r % d_in]
    y = torch.empty(rows, d_out, device="cuda")
    B.check(B.pr2_grouped_gemm(dm, one.cuda(), W.cuda(), off, y))
    close(y, x[r, r % d_in].double()[:, None] * W[0].double().t()[r % d_in])
    one = torch.zeros_like(dy)
    one[r, r % d_out] = dy[r, r % d_out]
    dx = torch.empty(rows, d_in, device="cuda")
    B.check(B.pr2_grouped_gemm_backward(dm, one.cuda(), W.cuda(), off, dx))
    close(dx, dy[r, r % d_out].double()[:, None] * W[0].double()[r % d_out])
    for row in (0, 31, 32, rows - 1):  # the term of one row, whatever its place in a K block
        one = torch.zeros_like(dy)
        one[row] = dy[row]
        dW = torch.empty(1, d_out, d_in, device="cuda")
        B.check(B.pr2_grouped_gemm_weight_grad(dm, one.cuda(), x.cuda(), off, dW))
        close(dW[0], dy[row].double()[:, None] * x[row].double())


def test_a_second_pair():
    """The gradient of the rows takes both pairs into one sum: one term, of either."""
    g = torch.Generator().manual_seed(3)
    rows, d_in, d_out = 150, 72, 75
    dy, W = [full(g, rows, d_out) for _ in range(2)], [full(g, 1, d_out, d_in) for _ in range(2)]
    r, off = torch.arange(rows), torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    at, first = r % d_out, r < d_out
    one = [torch.zeros_like(d) for d in dy]
    for p in range(2):
        mine = first if p == 0 else ~first
        one[p][r[mine], at[mine]] = dy[p][r[mine], at[mine]]
    dx = torch.empty(rows, d_in, device="cuda")
    B.check(B.pr2_grouped_gemm_backward(B.group_dims(rows, 1, d_in, d_out, "fp32"), one[0].cuda(), W[0].cuda(), off, dx,
                                        one[1].cuda(), W[1].cuda()))
    want = torch.where(first[:, None], dy[0][r, at].double()[:, None] * W[0][0].double()[at],
                       dy[1][r, at].double()[:, None] * W[1][0].double()[at])
    close(dx, want)
