"""Gradient of the matrices with experts of so many rows that one job takes longer than the limit of a wait
for a step of the pipeline (2 s): its waits for the end of a job take as long as the job.  All values are 1, so
the sums are the numbers of rows, exact in fp32 whatever the order (multiples of 32 below 2^29)."""
import time

import pytest
import torch

from paper_2606_00395_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,width,tail", [("fp32", 1 << 27, 1, 0), ("bf16", 1 << 29, 8, 0),
                                                   ("bf16", 1 << 29, 8, 32)])
def test_a_job_of_seconds(dtype, rows, width, tail):
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    x = torch.ones(rows, width, dtype=dt, device="cuda")
    x[-3:] = float("nan")  # of no expert
    many = rows - 128 + tail  # tail: its last K block has 32 rows
    off = torch.tensor([0, many, many + 7, rows - 3], dtype=torch.int32, device="cuda")
    dW = torch.full((3, width, width), -7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dm = B.group_dims(rows, 3, width, width, dtype, flags=B.PR2_F_SYNC_STATUS)
    torch.cuda.synchronize()
    t0 = time.time()
    code = B.pr2_grouped_gemm_weight_grad(dm, x, x, off, dW, status=status)
    print(f"{time.time() - t0:.2f} s")
    assert code == 0 and int(status.item()) == 0
    want = (off[1:] - off[:-1]).float().view(3, 1, 1).expand_as(dW)
    assert torch.equal(dW, want)
