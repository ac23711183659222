"""Refusals of the gated projections, the loss from the output layer's input, the embeddings and the gradient norm: found on
the host, before the device is looked at, and reported as status codes.  No GPU needed."""
import ctypes

import pytest
import torch

from paper_2605_09825_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.load_library()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(1 << 14)
    p.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


HUGE = 0x7FFFFFF8
INF, NAN = float("inf"), float("nan")


def test_sizes(lib):
    g = lib.mxfp4_gated_linear_workspace_bytes
    assert g(1024, 4096, 14336) == 2 * 1024 * 14336 * 2 and g(100, 64, 64) == 2 * 12800     # tiles enough; too short to split
    assert g(64, 4096, 14336) == 2 * 64 * 14336 * 2 + 9 * 256 * 4096 * 4
    assert g(0, 8, 8) == g(8, 8, 0) == g(8, 8, 12) == g(8, 12, 8) == g(HUGE, 8, 8) == 0
    l = lib.mxfp4_linear_logprobs_workspace_bytes
    assert l(1, 64, 1000, 0) == 32 * 16 * 8 + 32 * 4 and l(8192, 64, 1000, 0) == 8192 * 8 * 8 + 8192 * 4
    assert l(16384, 64, 128256, 0) == l(1 << 20, 64, 128256, 0) < 1 << 28         # does not grow with the text
    assert l(100, 64, 500, 1) == 100864                                           # one piece, too short to split: 100 * 504 * 2, rounded up
    assert l(8192, 8192, 128256, 1) == 8192 * 16384 * 2 + 8192 * 8192 * 4         # several pieces
    assert l(0, 8, 8, 0) == l(8, 12, 8, 0) == l(8, 8, 0, 1) == l(HUGE, 8, 8, 1) == 0
    e = lib.mxfp4_embedding_workspace_bytes
    assert e(1, 10, 8) == 3 * 256 + 64 and e(100, 10, 8) == 2 * 1024 + 256 + 13 * 64
    assert e(0, 8, 8) == e(8, 8, 12) == e(1 << 31, 8, 8) == e(8, 0, 8) == 0
    n = lib.mxfp4_grad_norm_workspace_bytes
    assert n(1) == n(640) == n(641) // 2 and n(0) == n(-1) == 0


def gated(p, **kw):
    d = api.GatedDesc(4, 64, 32, p, 64, p, 64, p, 64, 2)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


def test_gated_linear(lib, p):
    def fwd(h=p, ld_h=32, gate=p, up=p, ld_kept=32, **kw):
        return lib.mxfp4_gated_linear_forward(gated(p, **kw), h, ld_h, gate, up, ld_kept, None)

    def bwd(dh=p, ld_dh=32, gate=p, up=p, ld_kept=32, dx=p, ld_dx=64, dg=p, du=p, ld_dw=64, kind=0, ws=p, n=1 << 13, **kw):
        return lib.mxfp4_gated_linear_backward(gated(p, **kw), dh, ld_dh, gate, up, ld_kept, dx, ld_dx, dg, du, ld_dw, kind, ws, n,
                                               None)

    assert lib.mxfp4_gated_linear_forward(None, p, 32, p, p, 32, None) == -1
    for call in (fwd, bwd):
        for kw in ({"x": None}, {"w_gate": None}, {"w_up": None}, {"gate": None}, {"up": None}):
            assert call(**kw) == -1, kw
        assert call(act=6) == call(act=-1) == -4
        for kw in ({"tokens": 0}, {"in_features": 0}, {"features": 0}, {"in_features": 60}, {"features": 28}, {"ld_x": 56},
                   {"ld_gate": 56}, {"ld_up": 56}, {"ld_kept": 24}, {"tokens": HUGE}, {"features": HUGE}, {"in_features": HUGE}):
            assert call(**kw) == -2, kw
        for kw in ({"x": p + 2}, {"w_gate": p + 8}, {"w_up": p + 4}, {"gate": p + 2}, {"up": p + 8}, {"ld_x": 68}, {"ld_gate": 68},
                   {"ld_up": 68}, {"ld_kept": 36}):
            assert call(**kw) == -3, kw
    assert fwd(h=None) == -1 and fwd(ld_h=24) == -2 and fwd(h=p + 2) == fwd(ld_h=36) == -3
    assert bwd(dh=None) == bwd(dg=None) == bwd(du=None) == bwd(dx=None, dg=None, du=None) == -1
    assert bwd(kind=2) == -4
    assert bwd(ld_dh=24) == bwd(ld_dx=56) == bwd(ld_dw=56) == -2
    assert bwd(dh=p + 2) == bwd(dx=p + 8) == bwd(dg=p + 8) == bwd(du=p + 8) == bwd(ld_dh=36) == bwd(ld_dx=68) == bwd(ld_dw=68) == -3
    assert bwd(ws=None) == bwd(n=511) == -5 and bwd(ws=p + 8) == -3


def test_residual_norm_keeps_to_its_own_activations(lib, p):
    for act in (api.GATE_GELU, api.GATE_GELU_TANH, api.GATE_RELU):
        d = api.NormDesc(4, 64, p, 64, p, 64, p, 64, p, p, 0, api.GATE_ELEMENT, act, 1.0, 1.0, 1e-5)
        assert lib.mxfp4_residual_norm_forward(ctypes.byref(d), p, 64, p, 64, None) == -4


def test_linear_logprobs(lib, p):
    def fwd(x=p, ld_x=64, w=p, ld_w=64, T=4, D=64, V=100, t=p, scale=1.0, logp=p, lse=p, ws=p, n=1 << 13):
        return lib.mxfp4_linear_logprobs_forward(x, ld_x, w, ld_w, T, D, V, t, scale, logp, lse, ws, n, None)

    def bwd(x=p, ld_x=64, w=p, ld_w=64, T=4, D=64, V=100, t=p, scale=1.0, lse=p, gl=p, gn=p, dx=p, ld_dx=64, dw=p, ld_dw=64,
            kind=0, ws=p, n=1 << 13):
        return lib.mxfp4_linear_logprobs_backward(x, ld_x, w, ld_w, T, D, V, t, scale, lse, gl, gn, dx, ld_dx, dw, ld_dw, kind, ws, n,
                                                  None)

    for call in (fwd, bwd):
        assert call(x=None) == call(w=None) == call(lse=None) == -1
        assert call(scale=0.0) == call(scale=-1.0) == call(scale=INF) == call(scale=NAN) == -4
        for kw in ({"T": 0}, {"D": 0}, {"V": 0}, {"D": 60}, {"ld_x": 56}, {"ld_w": 56}, {"T": HUGE}, {"V": HUGE}, {"D": HUGE}):
            assert call(**kw) == -2, kw
        assert call(x=p + 2) == call(w=p + 8) == call(ld_x=68) == call(ld_w=68) == call(ws=p + 8) == -3
        assert call(ws=None) == call(n=64) == -5
    assert fwd(t=None) == fwd(logp=None) == -1
    assert bwd(gl=None, gn=None) == bwd(t=None) == bwd(dx=None, dw=None) == -1
    assert bwd(kind=2) == -4 and bwd(ld_dx=56) == bwd(ld_dw=56) == -2
    assert bwd(dx=p + 8) == bwd(dw=p + 8) == bwd(ld_dx=68) == bwd(ld_dw=68) == -3


def test_embedding(lib, p):
    def fwd(ids=p, T=4, table=p, kind=0, V=10, W=64, ld_t=64, scale=1.0, out=p, out_kind=0, ld_o=64, ws=None, n=0):
        return lib.mxfp4_embedding_forward(ids, T, table, kind, V, W, ld_t, scale, out, out_kind, ld_o, None)

    def bwd(ids=p, T=4, table=p, kind=0, V=10, W=64, ld_t=64, scale=1.0, out=p, out_kind=0, ld_o=64, ws=p, n=1 << 13):
        return lib.mxfp4_embedding_backward(ids, T, out, out_kind, ld_o, V, W, scale, table, kind, ld_t, 0, ws, n, None)

    for call in (fwd, bwd):
        assert call(ids=None) == call(table=None) == call(out=None) == -1
        assert call(kind=2) == call(out_kind=2) == call(scale=INF) == call(scale=NAN) == -4
        for kw in ({"T": 0}, {"V": 0}, {"W": 0}, {"W": 60}, {"ld_t": 56}, {"ld_o": 56}, {"T": 1 << 30}, {"V": 1 << 30}, {"W": 1 << 30}):
            assert call(**kw) == -2, kw
        assert call(table=p + 2) == call(out=p + 8) == call(ld_t=68) == call(ld_o=68) == -3
    assert bwd(ws=None) == bwd(n=512) == -5 and bwd(ws=p + 8) == -3


def test_grad_norm(lib, p):
    def call(ptrs=(p, p + 256), numel=(8, 8), kinds=(0, 1), max_norm=1.0, eps=1e-6, out=None, out_kinds=None, norm=p, ws=p, n=1 << 13,
             count=None):
        c = len(ptrs)
        vps = (ctypes.c_void_p * c)(*ptrs)
        outs = (ctypes.c_void_p * c)(*(ptrs if out is None else out))
        ks, oks = (ctypes.c_int32 * c)(*kinds), (ctypes.c_int32 * c)(*(kinds if out_kinds is None else out_kinds))
        ns, c = (ctypes.c_int64 * c)(*numel), c if count is None else count
        rc = lib.mxfp4_clip_grads(vps, ns, ks, c, max_norm, eps, outs, oks, norm, ws, n, None)
        if out is None and out_kinds is None and max_norm == 1.0 and eps == 1e-6 and rc != -2:
            assert lib.mxfp4_grad_norm(vps, ns, ks, c, norm, ws, n, None) == rc
        return rc

    assert lib.mxfp4_grad_norm(None, None, None, 1, p, p, 1 << 13, None) == -1 and call(norm=None) == -1
    assert call(ptrs=(p, None)) == call(out=(None, p)) == -1
    assert call(kinds=(0, 2)) == call(out_kinds=(2, 0)) == -4
    assert call(max_norm=-1.0) == call(max_norm=NAN) == call(eps=-1.0) == call(eps=NAN) == call(eps=INF) == -4
    assert call(count=0) == call(numel=(8, -1)) == -2
    assert call(ptrs=(p + 1, p + 256)) == call(ptrs=(p, p + 258)) == call(norm=p + 2) == call(ws=p + 8) == -3
    assert call(ws=None) == call(n=100) == -5
    # outputs that overlap: the same tensor twice, a neighbour's elements, an input's, its own in another type or shifted
    assert call(ptrs=(p, p), kinds=(0, 0)) == -2
    assert call(ptrs=(p, p + 14), kinds=(0, 0)) == -2
    assert call(out=(p + 512, p + 520), out_kinds=(0, 0)) == -2
    assert call(out=(p + 512, p)) == call(out=(p + 256, p + 512)) == -2
    assert call(out=(p, p + 256), out_kinds=(1, 1)) == call(out=(p + 2, p + 256)) == -2


def test_python_binding_checks_types_and_shapes_on_the_host():
    x, ids = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: api.gated_linear_forward(x, x, x), lambda: api.linear_logprobs_forward(x, x, ids),
                 lambda: api.embedding_forward(ids, x), lambda: api.embedding_backward(ids, x, 10),
                 lambda: api.grad_norm([x]), lambda: api.clip_grads([x], 1.0), lambda: api.grad_norm([x.half()])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(api.Mxfp4Error):
        api.grad_norm([])
