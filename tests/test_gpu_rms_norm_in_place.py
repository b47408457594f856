"""The norm's gradient written over the gradient of the sum (ds is dsum itself): the bits of the separate result, for
rows that a group walks one of and many of, for rows that are read twice (above 8192 columns), and off 16 bytes."""
import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,d,pad", [(37, 521, 0), (37, 2048, 0), (5000, 2048, 0), (5000, 2048, 8), (20000, 200, 0),
                                        (4000, 4096, 0), (1500, 8192, 0), (700, 9000, 0), (701, 9001, 0), (650, 32768, 0),
                                        (3000, 1023, 1)])
def test_over_dsum(rows, d, pad, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    dt, ld = R.DT[dtype], d + pad
    s, dy, dsum = (torch.randn(rows, d, generator=g, device="cuda").to(dt) for _ in range(3))
    w = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
    dm = B.norm_dims(rows, d, dtype, ld)
    ws = B.alloc_norm_workspace(dm)
    dw = [torch.full((d,), 7.0, device="cuda") for _ in range(2)]
    s, given, apart, into = R.place(s, ld, 0), R.place(dsum, ld, 0), R.place(dsum, ld, 0), R.place(dsum, ld, 0)
    apart.zero_()
    B.check(B.pr2_rmsnorm_backward(dm, s, w, dy, given, apart, dw[0], ws))
    for _ in range(3):
        into.copy_(dsum)
        B.check(B.pr2_rmsnorm_backward(dm, s, w, dy, into, into, dw[1], ws))
        assert torch.equal(apart, into) and torch.equal(dw[0], dw[1])
    want, size, ww, wsize = R.norm_backward(s, w, dy, dsum, 1e-6)
    assert ((into.double() - want).abs() <= R.HALF[dtype] * want.abs() + 48 * R.U * size + 1e-38).all()
    assert ((dw[1].double() - ww).abs() <= (96 + rows) * R.U * wsize + 1e-38).all()
    if pad:
        assert (into.as_strided((rows, ld), (ld, 1), into.storage_offset())[:-1, d:] == 7).all()
