"""fp32 operands next to the type's smallest values: an operand counts to 2^-24 of its value or to 2^-134, whichever
is more (the lowest of its three bf16 planes ends at 2^-133).  A single term: 1.25 U of it as for other values, and
2^-134 of each operand times the other."""
import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e", [-95, -105, -109, -110, -111, -118, -125, -126, -127, -133, -134, -140, -149])
@pytest.mark.parametrize("other", [20, 90, 126])
def test_one_small_operand(e, other):
    g = torch.Generator().manual_seed(-e)
    rows, d_in, d_out = 48, 64, 40
    value = (torch.rand(rows, generator=g, dtype=torch.float64) + 1) * 2.0 ** e
    x, W = torch.zeros(rows, d_in), torch.zeros(1, d_out, d_in)
    r = torch.arange(rows)
    x[r, r] = value.float()
    W[0] = ((torch.rand(d_out, d_in, generator=g, dtype=torch.float64) + 1) * 2.0 ** other).float()
    small, big = x[r, r].double()[:, None], W[0].double().t()[r]
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    y, dW = torch.empty(rows, d_out, device="cuda"), torch.empty(1, d_out, d_in, device="cuda")
    dm = B.group_dims(rows, 1, d_in, d_out, "fp32")
    B.check(B.pr2_grouped_gemm(dm, x.cuda(), W.cuda(), off, y))
    tol = 1.25 * R.U * small * big + 2.0 ** -134 * (big + small) + 2.0 ** -149
    assert ((y.cpu().double() - small * big).abs() <= tol).all()
    dy = W[0].t()[r].contiguous()  # one row's gradient times the same small value
    B.check(B.pr2_grouped_gemm_weight_grad(dm, dy.cuda(), x.cuda(), off, dW))
    assert ((dW[0].cpu().double().t()[r] - small * big).abs() <= tol).all()
