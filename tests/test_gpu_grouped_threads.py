"""The experts' products from several host threads at once, each with its own stream and buffers: no call
refuses another's launch, and each gives the bits it gives alone.  The sides differ in the number of experts,
which sets the shared memory that a launch takes."""
import threading

import pytest
import torch

import layers_reference as R
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


def _calls(kind, N, dtype):
    """A function that issues one call on a stream, and the tensor that it writes."""
    g = torch.Generator().manual_seed(N)
    rows, d_in, d_out, dt = 2 * N, 64, 72, R.DT[dtype]
    make = lambda *s: torch.randn(*s, generator=g).to(dt).cuda()  # noqa: E731
    x, W, dy = make(rows, d_in), make(N, d_out, d_in), make(rows, d_out)
    off = (2 * torch.arange(N + 1)).int().cuda()
    dm = B.group_dims(rows, N, d_in, d_out, dtype)
    if kind == "forward":
        y = torch.empty_like(dy)
        return lambda s: B.pr2_grouped_gemm(dm, x, W, off, y, stream=s), y
    if kind == "rows":
        dx = torch.empty_like(x)
        return lambda s: B.pr2_grouped_gemm_backward(dm, dy, W, off, dx, stream=s), dx
    if kind == "matrices":
        dW = torch.empty(N, d_out, d_in, device="cuda")
        return lambda s: B.pr2_grouped_gemm_weight_grad(dm, dy, x, off, dW, stream=s), dW
    q, Wq, y = x.to(R.F8), W.to(R.F8), torch.empty_like(dy)
    scale, ws = torch.ones(rows, device="cuda"), torch.ones(N, d_out, device="cuda")
    return lambda s: B.pr2_grouped_gemm_8bit(dm, q, scale, Wq, ws, off, y, stream=s), y


@pytest.mark.parametrize("kind,dtype", [("forward", "bf16"), ("forward", "fp32"), ("rows", "bf16"), ("matrices", "bf16"),
                                        ("8bit", "bf16")])
def test_products_from_two_threads(kind, dtype, n=8000):
    B.load()
    sides = [_calls(kind, N, dtype) for N in (16, 1000)]
    want = []
    for call, out in sides:
        B.check(call(None))
        torch.cuda.synchronize()
        want.append(out.clone())
    codes = [[], []]
    start = threading.Barrier(2)

    def work(i):
        torch.zeros(1, device="cuda")  # the device's context is current in this thread
        stream = torch.cuda.Stream()
        start.wait()
        codes[i] = [sides[i][0](stream) for _ in range(n)]
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert [sum(c != 0 for c in side) for side in codes] == [0, 0]
    for (_, out), ref in zip(sides, want):
        assert torch.equal(out, ref)
