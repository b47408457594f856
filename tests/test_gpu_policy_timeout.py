"""Policy loss behind a wait that ran out: with PR2_STATUS_TIMEOUT in the status word the loss is NaN, as it is
when a wait of the call itself runs out, whichever kernel the sizes take."""
import math

import pytest
import torch

from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("T,V", [(1, 50), (300, 500), (1, 3000), (1, 40000), (1, 131072), (20, 40000), (900, 4200),
                                 (1300, 52000)])
def test_loss_behind_a_timeout(T, V, grad):
    logits = torch.randn(T, V, device="cuda").bfloat16()
    target = torch.zeros(T, dtype=torch.int32, device="cuda")
    adv = torch.ones(T, device="cuda")
    out = torch.empty_like(logits) if grad else None
    dm = B.policy_dims(T, V, "bf16")
    ws = B.alloc_policy_workspace(dm)
    for bits, bad in ((0, False), (B.PR2_STATUS_TIMEOUT, True), (B.PR2_STATUS_BAD_INDEX, False), (0, False)):
        status = torch.tensor([bits], dtype=torch.int32, device="cuda")
        loss = torch.full((4,), 7.0, device="cuda")
        B.check(B.pr2_policy_loss(dm, logits, target, None, adv, None, None, loss, None, None, out, ws, status=status))
        got = loss.tolist()
        assert int(status.item()) == bits
        assert all(math.isnan(x) for x in got) if bad else all(math.isfinite(x) for x in got), (bits, got)
