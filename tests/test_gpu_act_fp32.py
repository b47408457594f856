"""fp32 activations and their gradients keep the accuracy of 32 bits over the whole range of the sigmoid.

act = g s u: the exponential is good to 2^-22 (2 units), 1 + e, the division and the two products to 2^-24 each:
4.8e-7 of its size.  dup = dact g s the same.  dgate = dact u s (1 + g (1 - s)): 1 - s is off by 2^-22 at most, so
1e-6 of |dact u s| (1 + |g|).  Sums of such terms that end in the denormal range: 1e-38."""
import pytest
import torch

import train_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [65536, 65537])
def test_activation_over_the_range_of_the_sigmoid(m):
    g = torch.linspace(-85, 85, m)[None]
    u = torch.linspace(0.5, 2.0, m)[None]
    dm = B.act_dims(1, m, "fp32")
    act = torch.empty(1, m, device="cuda")
    q, scale = torch.empty(1, 2, m, dtype=torch.int8, device="cuda"), torch.empty(1, 2, -(-m // 128), device="cuda")
    B.check(B.pr2_swiglu_checkpoint(dm, g.cuda(), u.cuda(), act, q, scale))
    want = R.swiglu(g.double(), u.double())
    err = (act.cpu().double() - want).abs()
    assert (err <= 4.8e-7 * want.abs() + 1e-38).all(), float((err / want.abs().clamp(min=1e-38)).max())


@pytest.mark.parametrize("m", [256, 255])
def test_gradients_over_the_range_of_the_sigmoid(m):
    """q runs over all its values; a row's scale puts gate's largest at 0.1 to 85."""
    tops = torch.tensor([0.1, 1.0, 5.0, 20.0, 50.0, 85.0])
    rows, G = tops.numel(), -(-m // 128)
    q = (torch.arange(m) - 127).clamp(-127, 127).to(torch.int8).expand(rows, 2, m).contiguous()
    scale = torch.stack([tops / 127, torch.ones(rows)], 1)[:, :, None].expand(rows, 2, G).contiguous()
    dact = torch.linspace(0.5, 1.5, m).expand(rows, m).contiguous()
    dg, du, act = (torch.empty(rows, m, device="cuda") for _ in range(3))
    B.check(B.pr2_swiglu_checkpoint_backward(B.act_dims(rows, m, "fp32"), dact.cuda(), q.cuda(), scale.cuda(), dg, du, act))
    g, u = ((q[:, i].float() * scale[:, i, :1]).double() for i in (0, 1))  # (held values: rounded to 32 bits)
    want = R.swiglu_backward(g, u, dact.double())
    size = 1e-6 * (dact * u * torch.sigmoid(g)).abs() * (1 + g.abs()), 4.8e-7 * want[1].abs(), 4.8e-7 * want[2].abs()
    for got, exact, bound in zip((dg, du, act), want, size):
        err = (got.cpu().double() - exact).abs()
        assert (err <= bound + 1e-38).all(), float((err - bound).max())
