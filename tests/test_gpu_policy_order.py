"""Policy loss of batches whose tokens are dealt out by weight: right behind the kernels that write its inputs,
all of them, the same bits as with the stream drained before the call; and masks of every kind."""
import pytest
import torch

import test_gpu_policy_loss as base
from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,dtype,grad", [(1300, 52001, torch.bfloat16, True), (900, 30003, torch.float32, True),
                                            (1400, 131001, torch.bfloat16, False), (3000, 30003, torch.float32, False)])
def test_inputs_written_right_before_the_call(T, V, dtype, grad):
    g = torch.Generator(device="cuda").manual_seed(T)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    sets = []
    for _ in range(2):
        w = (torch.rand(T, generator=g, device="cuda") > 0.2).float() / T
        sets.append([make(T, V).to(dtype), torch.randint(0, V, (T,), generator=g, device="cuda").int(), w, make(T),
                     make(T) - 11, make(T) - 11])
    now = [torch.zeros_like(x) for x in sets[0]]
    dm = B.policy_dims(T, V, "fp32" if dtype == torch.float32 else "bf16", kl_coef=0.05)
    ws = B.alloc_policy_workspace(dm)
    loss, logp, ent = torch.zeros(4, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    out = torch.zeros_like(now[0]) if grad else None

    def call():
        B.check(B.pr2_policy_loss(dm, *now, loss, logp, ent, out, ws))
        return [x.clone() for x in (loss, logp, ent)] + ([out.double().sum(1)] if grad else [])

    alone = []
    for s in sets:
        for x, y in zip(now, s):
            x.copy_(y)
        torch.cuda.synchronize()
        alone.append(call())
        torch.cuda.synchronize()
    seen = []
    for i in range(20):
        order = range(6) if i % 4 < 2 else range(5, -1, -1)  # (each of them is the last before some call)
        for x in now:
            x.zero_()
        for j in list(order)[i % 6:] + list(order)[:i % 6]:
            now[j].copy_(sets[i % 2][j])
        seen.append(call())
    torch.cuda.synchronize()
    for i, got in enumerate(seen):
        assert all(torch.equal(a, b) for a, b in zip(got, alone[i % 2])), i


@pytest.mark.parametrize("kind", ["none", "all", "first half", "second half", "all but the last", "runs", "random"])
@pytest.mark.parametrize("dtype,T,V,grad", [("bf16", 1400, 52001, True), ("fp32", 700, 40000, True),
                                            ("bf16", 6200, 16400, True), ("bf16", 1400, 131001, False)])
def test_masked_tokens(dtype, T, V, grad, kind):
    base.test_masked_tokens_in_large_batches(dtype, T, V, grad, kind)
