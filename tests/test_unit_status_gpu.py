"""A wait that runs out in any part of the library is reported by the next check, once that part has been used."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys
import torch
sys.path.insert(0, sys.argv[1])
from paper_2605_09825_b200 import api

x = torch.ones(304, 64, dtype=torch.bfloat16, device="cuda")
w = torch.ones(64, device="cuda")
ids = torch.arange(304, device="cuda") % 64
lse = torch.full((304,), 70.0, device="cuda")
# the call, and the part whose kernels have waits that it uses
calls = [(lambda: api.linear_fprop(x[:64], x[:64]), 0),
         (lambda: api.linear_pass_block128(api.PASS_FPROP, x[:64], x[:64]), 1),
         (lambda: api.residual_norm_forward(x, x, w_pre=w), 2),
         (None, 3),
         (lambda: api.gated_linear_forward(x[:40], x, x), 4),
         (lambda: api.embedding_backward(ids, x, 64), 5)]
dense = {"gated": lambda: api.gated_linear_forward(x, x, x),
         "gated_gradient": lambda: api.gated_linear_backward(x[:, :64], x, x[:64], x[:64], (x, x)),
         "loss": lambda: api.linear_logprobs_forward(x, x, ids),
         "loss_gradient": lambda: api.linear_logprobs_backward(x, x, ids, lse, lse)}
calls[3] = (dense[sys.argv[2]], 3)
for call, part in calls:
    call()
    api.check()
    for again in range(2):
        api.selftest_unit_timeout(part)
        try:
            api.check()
        except api.Mxfp4Error as e:
            assert e.status == -7, (part, e)
        else:
            raise AssertionError(f"part {part}: nothing reported")
        api.check()                       # cleared by the failing check
    call()
    api.check()                           # and the next call is not held responsible
print("reported")
"""


@pytest.mark.parametrize("use", ["gated", "gated_gradient", "loss", "loss_gradient"])
def test_a_wait_that_runs_out_is_reported_whatever_part_it_is_in(use):
    res = subprocess.run([sys.executable, "-c", CHILD, ROOT, use], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and "reported" in res.stdout, res.stderr[-3000:]
