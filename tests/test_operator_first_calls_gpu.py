"""Two host threads make their FIRST calls of the operators around the linears at the same moment (fresh process, so the
resident grid sizes and each kernel's shared-memory attribute are still unset): both must succeed and give the
results a single thread gets."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys, threading
import torch
sys.path.insert(0, sys.argv[1])
from paper_2605_09825_b200 import api
which = sys.argv[2]
api.load_library()
torch.cuda.init()
rand = lambda *s: torch.randn(*s, device="cuda")
torch.manual_seed(1)
w = rand(8200)
data = [[rand(*s).bfloat16() for s in ((300, 400), (520, 400), (9, 8200), (9, 8200), (9, 8200), (3, 40000))] for _ in range(2)]
calls = {
    "product": lambda a, b, u, x, dh, z: (api.linear_pass_block128(api.PASS_FPROP, a, b),),
    "norm": lambda a, b, u, x, dh, z: api.residual_norm_forward(u, x, w, w),
    "norm_gradient": lambda a, b, u, x, dh, z: api.residual_norm_backward(dh, None, u, x, w, w),
    "logprobs": lambda a, b, u, x, dh, z: api.logprobs_forward(z, None, 5),
}
call = calls[which]
torch.cuda.synchronize()
streams = [torch.cuda.Stream() for _ in range(2)]
gate = threading.Barrier(2)
out, err = [None, None], [None, None]
def work(i):
    try:
        with torch.cuda.stream(streams[i]):
            gate.wait()
            out[i] = call(*data[i])
            streams[i].synchronize()
    except Exception as exc:
        err[i] = repr(exc)
th = [threading.Thread(target=work, args=(i,)) for i in range(2)]
[t.start() for t in th]; [t.join() for t in th]
assert err == [None, None], err
api.check()
for i in range(2):
    want = call(*data[i])
    api.check()
    assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(out[i], want)), i
print("threads-ok")
"""


@pytest.mark.parametrize("which", ["product", "norm", "norm_gradient", "logprobs"])
def test_two_threads_first_call(which):
    res = subprocess.run([sys.executable, "-c", CHILD, ROOT, which], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and "threads-ok" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]
