"""Refusals of the 128-block product, the residual norm and the log probabilities: found on the host, before
the device is looked at, and reported as status codes.  No GPU needed."""
import ctypes

import pytest

from paper_2605_09825_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.load_library()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(1 << 12)
    p.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


BIG = 0x7FFFFFF0


def test_sizes(lib):
    s = lib.mxfp4_block128_scales_bytes
    assert s(256, 512, api.BLOCK_1X128) == 4 * 256 * 4 and s(256, 512, api.BLOCK_128X128) == 4 * 2 * 4
    assert s(130, 144, api.BLOCK_1X128) == 2 * 256 * 4 and s(130, 144, api.BLOCK_128X128) == 2 * 2 * 4
    assert s(0, 128, 2) == s(128, 0, 2) == s(128, 120, 2) == s(128, 128, api.BLOCK_1X32) == 0
    w = lib.mxfp4_gemm_block128_workspace_bytes
    assert w(8192, 4096, 4096) == 0 and w(1, 4096, 128) == 0          # enough tiles; nothing to split
    assert w(40, 4096, 14336) % (40 * 4096 * 4) == 0 and w(40, 4096, 14336) > 0 and w(1, 4096, 14336) == 0
    assert w(0, 8, 128) == w(8, 8, 100) == 0
    lw = lib.mxfp4_linear_pass_block128_workspace_bytes
    assert lw(8192, 4096, 6144, 0) >= 8192 * 4096 + 6144 * 4096
    assert lw(100, 64, 64, 2) == 0 and lw(8, 8, 8, 3) == 0            # tokens are the reduction of the weight gradient
    n = lib.mxfp4_residual_norm_workspace_bytes
    assert n(1, 4096) == 3 * 4096 * 4 and n(1 << 20, 4096) < 1 << 26 and n(4, 12) == n(0, 8) == n(4, 16392) == 0
    l = lib.mxfp4_logprobs_workspace_bytes
    assert l(8192, 128256, 20) == 0 and l(1, 128256, 20) > 0 and l(1, 128256, 33) == l(0, 10, 1) == 0


def test_quantize_block128(lib, p):
    q = lib.mxfp4_quantize_block128
    for bad in ((None, 16, 16, 16, 1, 2, p, p), (p, 16, 16, 16, 1, 2, None, p), (p, 16, 16, 16, 1, 2, p, None)):
        assert q(*bad, None) == -1
    assert q(p, 16, 16, 16, 2, 2, p, p, None) == -4
    assert q(p, 16, 16, 16, 1, api.BLOCK_1X32, p, p, None) == -4
    for rows, cols, ld, axis in ((0, 16, 16, 1), (16, 0, 16, 1), (16, 24, 24, 1), (24, 16, 16, 0), (16, 32, 16, 1),
                                 (BIG, BIG, BIG, 1), (1 << 31, 16, 16, 1)):
        assert q(p, rows, cols, ld, axis, 2, p, p, None) == -2
    assert q(p + 2, 16, 16, 16, 1, 2, p, p, None) == q(p, 16, 16, 20, 1, 2, p, p, None) == -3
    assert q(p, 16, 16, 16, 1, 2, p + 8, p, None) == q(p, 16, 16, 16, 1, 2, p, p + 4, None) == -3


def test_gemm_block128(lib, p):
    g = lib.mxfp4_gemm_block128
    call = lambda a=p, sa=p, b=p, sb=p, shape=3, M=128, N=128, K=128, out=p, dtype=0, ld=128, ws=None, n=0: \
        g(a, sa, b, sb, shape, M, N, K, out, dtype, ld, ws, n, None)
    for name in ("a", "sa", "b", "sb", "out"):
        assert call(**{name: None}) == -1 and call(**{name: p + 8}) == -3
    assert call(shape=0) == call(dtype=2) == -4
    assert call(M=0) == call(N=0) == call(K=0) == call(K=120) == call(ld=120) == call(M=BIG, N=BIG, ld=BIG) == -2
    assert call(N=100, ld=100) == -3
    assert call(M=40, N=4096, K=14336, ld=4096) == -5                  # split along K: needs its workspace
    assert call(M=40, N=4096, K=14336, ld=4096, ws=p, n=64) == -5


def test_linear_pass_block128(lib, p):
    f = lib.mxfp4_linear_pass_block128
    assert f(3, p, p, p, 16, 16, 16, 0, p, 1 << 20, None) == -4
    assert f(0, None, p, p, 16, 16, 16, 0, p, 1 << 20, None) == -1
    assert f(0, p, p, p, 16, 16, 16, 5, p, 1 << 20, None) == -4
    assert f(0, p, p, p, 0, 16, 16, 0, p, 1 << 20, None) == -2
    assert f(0, p, p, p, 16, 24, 16, 0, p, 1 << 20, None) == -2        # reduction not a multiple of 16
    assert f(2, p, p, p, 24, 16, 16, 0, p, 1 << 20, None) == -2
    assert f(0, p, p, p, 16, 16, 12, 0, p, 1 << 20, None) == -2
    assert f(0, p, p, p, 16, 16, 16, 0, None, 0, None) == f(0, p, p, p, 16, 16, 16, 0, p, 64, None) == -5
    assert f(0, p, p, p, 16, 16, 16, 0, p + 16, 1 << 20, None) == -3
    assert f(0, p + 2, p, p, 16, 16, 16, 0, p, 1 << 20, None) == -3


def desc(p, **kw):
    d = api.NormDesc(4, 64, p, 64, p, 64, None, 0, p, p, 0, 0, 0, 1.0, 1.0, 1e-5)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


def test_residual_norm(lib, p):
    def fwd(y=p, ld_y=64, h=p, ld_h=64, **kw):
        return lib.mxfp4_residual_norm_forward(desc(p, **kw), y, ld_y, h, ld_h, None)

    def bwd(dh=p, ld_dh=64, dy=p, ld_dy=64, dx=p, dbranch=p, dgate=None, dw_post=p, dw_pre=p, ws=p, n=1 << 20, **kw):
        return lib.mxfp4_residual_norm_backward(desc(p, **kw), dh, ld_dh, dy, ld_dy, dx, 64, dbranch, 64, dgate, 64,
                                                dw_post, dw_pre, ws, n, None)

    assert lib.mxfp4_residual_norm_forward(None, p, 64, p, 64, None) == -1
    for call in (fwd, bwd):
        assert call(branch=None) == call(gate=p) == call(gate_kind=1) == -1
        assert call(gate_kind=3, gate=p) == call(gate_act=3) == call(stream_dtype=2) == call(eps=-1.0) == call(eps=float("nan")) == -4
        for kw in ({"tokens": 0}, {"width": 0}, {"width": 60}, {"width": 16392}, {"ld_branch": 56}, {"ld_stream": 56},
                   {"tokens": 1 << 31}, {"gate_kind": 2, "gate": p, "ld_gate": 56}):
            assert call(**kw) == -2, kw
        for kw in ({"branch": p + 2}, {"stream": p + 8}, {"w_post": p + 4}, {"w_pre": p + 8}, {"ld_branch": 68},
                   {"gate_kind": 2, "gate": p, "ld_gate": 68}, {"gate_kind": 1, "gate": p + 4}):
            assert call(**kw) == -3, kw
    assert fwd(y=None) == fwd(h=None) == fwd(w_pre=None) == -1         # h exactly when w_pre is there
    assert fwd(ld_y=56) == fwd(ld_h=56) == -2
    assert fwd(y=p + 2) == fwd(ld_h=68) == -3
    assert bwd(dh=None) == bwd(stream=None) == bwd(w_pre=None) == -1
    assert bwd(w_pre=None, dw_pre=None, dh=None, dy=None) == -1        # no gradient at all
    assert bwd(dgate=p) == bwd(w_post=None) == -1                      # a gradient of what is not there
    assert bwd(ld_dh=56) == bwd(ld_dy=56) == -2
    assert bwd(dx=p + 4) == bwd(dw_post=p + 8) == bwd(ws=p + 8) == -3
    assert bwd(ws=None) == bwd(n=16) == -5


def test_logprobs(lib, p):
    def fwd(x=p, dtype=0, T=4, V=100, ld=100, t=p, scale=1.0, logp=p, ent=p, lse=p, k=2, tv=p, ti=p, ws=p, n=1 << 20):
        return lib.mxfp4_logprobs_forward(x, dtype, T, V, ld, t, scale, logp, ent, lse, k, tv, ti, ws, n, None)

    def bwd(x=p, dtype=0, T=4, V=100, ld=100, t=p, scale=1.0, lse=p, ent=p, gl=p, ge=p, d=p, ld_d=100):
        return lib.mxfp4_logprobs_backward(x, dtype, T, V, ld, t, scale, lse, ent, gl, ge, d, ld_d, None)

    for call in (fwd, bwd):
        assert call(x=None) == call(lse=None) == -1
        assert call(dtype=2) == call(scale=0.0) == call(scale=-1.0) == call(scale=float("inf")) == call(scale=float("nan")) == -4
        assert call(T=0) == call(V=0) == call(ld=99) == call(V=1 << 30, ld=1 << 30) == call(T=1 << 31) == -2
        assert call(x=p + 1) == call(x=p + 2, dtype=1) == -3
    assert fwd(t=None) == fwd(logp=None) == fwd(tv=None) == fwd(ti=None) == -1
    assert fwd(k=33) == fwd(k=-1) == -4
    assert fwd(T=1, V=128256, ld=128256, ws=None) == fwd(T=1, V=128256, ld=128256, n=16) == -5
    assert fwd(T=1, V=128256, ld=128256, ws=p + 8) == -3
    assert bwd(d=None) == bwd(t=None) == bwd(ent=None) == -1
    assert bwd(ld_d=99) == -2
    assert bwd(d=p + 1) == -3


def test_python_binding_checks_types_and_shapes_on_the_host():
    import torch
    x = torch.zeros(4, 64)
    for call in (lambda: api.quantize_block128(x), lambda: api.logprobs_forward(x.half()),
                 lambda: api.residual_norm_forward(x), lambda: api.linear_pass_block128(0, x, x)):
        with pytest.raises(ValueError):
            call()


def test_stream_dtype_against_a_given_stream():
    """The type of the result follows a given stream; asking for another one is refused, not ignored."""
    import torch
    u = torch.zeros(4, 64, dtype=torch.bfloat16)
    for stream, dtype in ((u, torch.float32), (u.float(), torch.bfloat16)):
        with pytest.raises(ValueError, match="stream_dtype"):
            api.residual_norm_forward(u, stream, stream_dtype=dtype)
