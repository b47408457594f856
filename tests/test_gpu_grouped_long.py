"""The experts' products with 16-bit results over long sums, against the plain 64-bit form.

All terms have one sign, where an accumulator that cuts bits off errs to one side.  Of at most 1024 MMAs in turn each
is off by at most 2 U of the accumulator's sum, and the parts are added with rounding, U for each of them; then one
rounding, by half a step of the value.  Whole numbers whose sums stay below 2^24 are exact until that rounding.
"""
import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu
MMAS = 1024


def half_step(want):
    return torch.exp2(torch.floor(torch.log2(want.abs())) - 8)  # bf16: 8 bits


def check(got, want, parts, exact):
    if exact:
        assert torch.equal(got, want.to(got.dtype))
    else:
        assert ((got.double() - want).abs() <= half_step(want) + (2 * MMAS + parts) * R.U * want).all()


def make(g, exact, *shape):
    if exact:
        return torch.randint(0, 3, shape, generator=g, device="cuda").float()
    return torch.rand(*shape, generator=g, device="cuda")


# length of the sums, the other width, rows of the experts
CASES = [(8200, 40, [3, 0, 300]), (16384, 40, [3, 0, 300]), (16392, 40, [3, 0, 300]), (16385, 37, [1, 70]),
         (32784, 136, [257, 0, 5]), (32768, 264, [385, 16]), (131088, 24, [40]), (1 << 17, 31, [2, 33]), (1 << 20, 24, [33])]


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("pairs", [1, 2])
@pytest.mark.parametrize("K,d,counts", CASES)
def test_forward(K, d, counts, pairs, exact):
    g = torch.Generator(device="cuda").manual_seed(K + d)
    rows, N = sum(counts), len(counts)
    off = torch.tensor([0] + counts).cumsum(0).int()
    x = make(g, exact, rows, K).bfloat16()
    W = [make(g, exact, N, d, K).bfloat16() for _ in range(pairs)]
    y = [torch.full((rows, d), -7.0, device="cuda").bfloat16() for _ in range(pairs)]
    two = (W[1], y[1]) if pairs == 2 else (None, None)
    B.check(B.pr2_grouped_gemm(B.group_dims(rows, N, K, d), x, W[0], off.cuda(), y[0], *two))
    for got, w in zip(y, W):
        check(got, R.grouped(x, w, off)[0], K // 16384 + 1, exact)


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("pairs", [1, 2])
@pytest.mark.parametrize("K,d,counts", CASES)
def test_gradient_of_the_rows(K, d, counts, pairs, exact):
    """The sum goes over the columns of both matrices."""
    g = torch.Generator(device="cuda").manual_seed(K + d)
    rows, N = sum(counts), len(counts)
    off = torch.tensor([0] + counts).cumsum(0).int()
    dy = [make(g, exact, rows, K).bfloat16() for _ in range(pairs)]
    W = [make(g, exact, N, K, d).bfloat16() for _ in range(pairs)]
    dx = torch.full((rows, d), -7.0, device="cuda").bfloat16()
    two = (dy[1], W[1]) if pairs == 2 else (None, None)
    B.check(B.pr2_grouped_gemm_backward(B.group_dims(rows, N, d, K), dy[0], W[0], off.cuda(), dx, *two))
    check(dx, R.grouped_backward(dy, W, off)[0], pairs * (K // 16384 + 1), exact)


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("pairs", [1, 2])
@pytest.mark.parametrize("K,d,counts", CASES)
def test_8bit(K, d, counts, pairs, exact):
    g = torch.Generator(device="cuda").manual_seed(K + d)
    rows, N = sum(counts), len(counts)
    off = torch.tensor([0] + counts).cumsum(0).int()
    q = make(g, exact, rows, K).to(R.F8)
    W = [make(g, exact, N, d, K).to(R.F8) for _ in range(pairs)]
    scale = torch.exp2(torch.arange(rows, device="cuda") % 5 - 2.0)
    ws = [torch.exp2(torch.arange(N * d, device="cuda") % 3 - 1.0).view(N, d) for _ in range(pairs)]
    y = [torch.full((rows, d), -7.0, device="cuda").bfloat16() for _ in range(pairs)]
    two = (W[1], ws[1], y[1]) if pairs == 2 else (None, None, None)
    B.check(B.pr2_grouped_gemm_8bit(B.group_dims(rows, N, K, d), q, scale, W[0], ws[0], off.cuda(), y[0], *two))
    for got, w, s in zip(y, W, ws):
        want = R.grouped(q.float(), w.float(), off)[0]
        for e, r in R.spans(off, rows):
            want[r] *= scale[r, None].double() * s[e].double()
        check(got, want, K // 32768 + 1, exact)
