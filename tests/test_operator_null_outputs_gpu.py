"""Results that a caller of the C ABI may leave out (NULL): whatever is asked for is, bit for bit, what the call that asks
for everything gives, and nothing else is needed for it."""
import ctypes
import itertools

import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

PARTS = ("dx", "dbranch", "dgate", "dw_post", "dw_pre")


def rand(*shape, dtype=torch.bfloat16, seed=0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("tokens,width", [(37, 520), (9, 8200)])
@pytest.mark.parametrize("gate_kind", [api.GATE_NONE, api.GATE_CHANNEL, api.GATE_ELEMENT])
def test_residual_norm_gradients(gate_kind, tokens, width):
    lib = api.load_library()
    stream = torch.cuda.current_stream().cuda_stream
    u, y, dh, dy = (rand(tokens, width, seed=s) for s in range(4))
    w_post, w_pre = (rand(width, dtype=torch.float32, seed=s) for s in (5, 6))
    gate = {api.GATE_NONE: None, api.GATE_CHANNEL: rand(width, dtype=torch.float32, seed=7),
            api.GATE_ELEMENT: rand(tokens, width, seed=7)}[gate_kind]
    want = dict(zip(PARTS, api.residual_norm_backward(dh, dy, u, y, w_post, w_pre, gate, api.GATE_SIGMOID)))
    desc = api.NormDesc(tokens, width, u.data_ptr(), width, y.data_ptr(), width, gate.data_ptr() if gate is not None else None,
                        width, w_post.data_ptr(), w_pre.data_ptr(), api.OUT_BF16, gate_kind, api.GATE_SIGMOID, 1.0, 1.0, 1e-5)
    ws = torch.empty(lib.mxfp4_residual_norm_workspace_bytes(tokens, width), dtype=torch.uint8, device="cuda")
    names = [n for n in PARTS if want[n] is not None]
    for asked in itertools.product((False, True), repeat=len(names)):
        got = {n: torch.full_like(want[n], 7.0) for n, a in zip(names, asked) if a}
        vectors = any(t.dim() == 1 for t in got.values())
        p = lambda n: got[n].data_ptr() if n in got else None
        ld = lambda n: width if n in got else 0
        rc = lib.mxfp4_residual_norm_backward(
            ctypes.byref(desc), dh.data_ptr(), width, dy.data_ptr(), width, p("dx"), ld("dx"), p("dbranch"), ld("dbranch"),
            p("dgate"), ld("dgate"), p("dw_post"), p("dw_pre"), ws.data_ptr() if vectors else None,
            ws.numel() if vectors else 0, stream)
        assert rc == 0, (rc, list(got))
        api.check()
        assert all(torch.equal(got[n], want[n]) for n in got), list(got)


@pytest.mark.parametrize("tokens,vocab", [(1, 50000), (5, 999), (700, 999)])
@pytest.mark.parametrize("top", [0, 4])
def test_log_probabilities_without_entropy(tokens, vocab, top):
    lib = api.load_library()
    x, t = rand(tokens, vocab), torch.arange(tokens, device="cuda")
    logp, _, lse, top_logp, top_index = api.logprobs_forward(x, t, top)
    outs = [torch.full((tokens,), 7.0, device="cuda") for _ in range(2)]
    tl = torch.empty(tokens, max(top, 1), device="cuda")
    ti = torch.empty(tokens, max(top, 1), dtype=torch.int64, device="cuda")
    ws = torch.empty(max(lib.mxfp4_logprobs_workspace_bytes(tokens, vocab, top), 16), dtype=torch.uint8, device="cuda")
    for with_target in (True, False):
        rc = lib.mxfp4_logprobs_forward(
            x.data_ptr(), api.OUT_BF16, tokens, vocab, vocab, t.data_ptr() if with_target else None, 1.0,
            outs[0].data_ptr() if with_target else None, None, outs[1].data_ptr(), top, tl.data_ptr() if top else None,
            ti.data_ptr() if top else None, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        api.check()
        assert torch.equal(outs[0], logp) and torch.equal(outs[1], lse)
        if top:
            assert torch.equal(tl, top_logp) and torch.equal(ti, top_index)
