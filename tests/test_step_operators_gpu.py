"""What holds for every call of a training step's two ends: it runs on the stream that is current when it is made, two
host threads may make their first calls at the same moment, calls on two streams do not disturb one another, and the
bounds-checking build finds no shared-memory address outside its buffer."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2605_09825_b200 import api, build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DELAY_CYCLES = 20_000_000


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def flat(r):
    out = []
    for t in r if isinstance(r, (tuple, list)) else (r,):
        out += flat(t) if isinstance(t, (tuple, list)) else [t] if t is not None else []
    return out


def ids(n, vocab):
    return torch.arange(n, device="cuda") * 7919 % vocab


def clip(a, b):
    out = [torch.empty_like(a), torch.empty_like(b, dtype=torch.float32)]
    return api.clip_grads([a, b], 0.5, out), out


# name: the call, and inputs that arrive late
CASES = {
    "gated_1": (lambda x, g, u: api.gated_linear_forward(x, g, u), lambda: (rand(1, 136), rand(72, 136, seed=1), rand(72, 136, seed=2))),
    "gated_40": (lambda x, g, u: api.gated_linear_forward(x, g, u), lambda: (rand(40, 136), rand(72, 136, seed=1), rand(72, 136, seed=2))),
    "gated_700": (lambda x, g, u: api.gated_linear_forward(x, g, u), lambda: (rand(700, 136), rand(72, 136, seed=1), rand(72, 136, seed=2))),
    "gated_gradient": (lambda dh, x, g, u, a, b: api.gated_linear_backward(dh, x, g, u, (a, b)),
                       lambda: (rand(300, 72), rand(300, 136), rand(72, 136, seed=1), rand(72, 136, seed=2), rand(300, 72, seed=3),
                                rand(300, 72, seed=4))),
    "loss": (lambda x, w: api.linear_logprobs_forward(x, w, ids(300, 3001)), lambda: (rand(300, 72), rand(3001, 72, seed=1))),
    "loss_gradient": (lambda x, w, lse: api.linear_logprobs_backward(x, w, ids(300, 3001), lse, torch.ones_like(lse)),
                      lambda: (rand(300, 72), rand(3001, 72, seed=1) * 0.1, 9 + rand(300, dtype=torch.float32))),
    "lookup": (lambda t: api.embedding_forward(ids(300, 100), t, 2.0), lambda: (rand(100, 136),)),
    "table_gradient": (lambda d: api.embedding_backward(ids(3000, 100), d, 100), lambda: (rand(3000, 136),)),
    "norm": (lambda a, b: api.grad_norm([a, b]), lambda: (rand(100000), rand(37))),
    "clip": (clip, lambda: (rand(100000), rand(37))),
}


@pytest.mark.parametrize("name", CASES)
def test_late_inputs_on_a_side_stream(name):
    call, make = CASES[name]
    real = make()
    old = [t.flip(0).mul(2).contiguous() for t in real]
    stale = [t.clone() for t in flat(call(*old))]
    want = [t.clone() for t in flat(call(*real))]
    assert any(not torch.equal(a, b) for a, b in zip(stale, want))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(DELAY_CYCLES)
        for buf, t in zip(old, real):
            buf.copy_(t)
        got = call(*old)
        assert not side.query(), "the delay was over before the call was made"
    side.synchronize()
    api.check()
    assert all(torch.equal(a, b) for a, b in zip(flat(got), want))


@pytest.mark.parametrize("name", CASES)
def test_two_streams_at_once(name):
    call, make = CASES[name]
    sets = [make(), [t.flip(0).contiguous() for t in make()]]
    want = [[t.clone() for t in flat(call(*s))] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(call(*sets[i]))
    torch.cuda.synchronize()
    api.check()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(flat(r), want[i]))


@pytest.mark.parametrize("name", CASES)
def test_captured_while_an_eager_call_and_another_graph_run(name):
    call, make = CASES[name]
    real = make()
    want = [t.clone() for t in flat(call(*real))]
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call(*real))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        eager = call(*real)
    torch.cuda.synchronize()
    api.check()
    for r in (*outs, eager):
        assert all(torch.equal(a, b) for a, b in zip(flat(r), want))


FIRST = r"""
import sys, threading
import torch
sys.path.insert(0, sys.argv[1])
sys.path.insert(0, sys.argv[1] + "/tests")
from paper_2605_09825_b200 import api
import test_step_operators_gpu as t
call, make = t.CASES[sys.argv[2]]
data = [make(), [x.flip(0).contiguous() for x in make()]]
torch.cuda.synchronize()
got, errors, gate = [None, None], [], threading.Barrier(2)
def run(i):
    try:
        with torch.cuda.stream(torch.cuda.Stream()):
            gate.wait()
            got[i] = call(*data[i])
            torch.cuda.current_stream().synchronize()
    except Exception as e:
        errors.append(e)
threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
[x.start() for x in threads]
[x.join() for x in threads]
api.check()
assert not errors, errors
for i in range(2):
    assert all(torch.equal(a, b) for a, b in zip(t.flat(got[i]), t.flat(call(*data[i]))))
"""


@pytest.mark.parametrize("name", ["gated_40", "gated_gradient", "loss_gradient", "table_gradient", "clip"])
def test_first_calls_of_two_threads(name):
    res = subprocess.run([sys.executable, "-c", FIRST, ROOT, name], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]


BOUNDS = r"""
import sys
sys.path.insert(0, sys.argv[1])
from paper_2605_09825_b200 import api
assert api.bounds_checked(), "the child did not load the bounds-checking build"
import pytest
sys.exit(pytest.main(["-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gated_linear_gpu.py",
                      "tests/test_linear_logprobs_gpu.py", "tests/test_embedding_gpu.py", "tests/test_grad_norm_gpu.py"]))
"""


def test_suites_pass_under_the_bounds_checking_build():
    lib = build.build_library(bounds=True)
    res = subprocess.run([sys.executable, "-c", BOUNDS, ROOT], cwd=ROOT, env=dict(os.environ, MXFP4_LIBRARY=lib),
                         capture_output=True, text=True, timeout=1800)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
    assert " passed" in res.stdout and "failed" not in res.stdout
