"""Norm after a block, gate, scaled residual and norm before the next block, forward and backward,
against the formulas in 64 bits."""
import itertools

import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu

EPS = 1e-5
ACTS = {api.GATE_LINEAR: lambda g: g, api.GATE_SIGMOID: torch.sigmoid, api.GATE_SILU: torch.nn.functional.silu}


def make(tokens, width, stream=torch.bfloat16, x=True, post=True, pre=True, gate="element", seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std
    mat = lambda dtype, std=1.0: n(tokens, width + pad, std=std).to(dtype)[:, :width]
    branch = mat(torch.bfloat16)
    branch[:, 0] *= 20.0
    return {"branch": branch, "stream": mat(stream, 3.0) if x else None, "dtype": stream,
            "w_post": 1 + n(width, std=0.2) if post else None, "w_pre": 1 + n(width, std=0.2) if pre else None,
            "gate": {"none": None, "channel": 0.5 + n(width, std=0.3), "element": mat(torch.bfloat16)}[gate],
            "dh": mat(torch.bfloat16, 1e-2) if pre else None, "dy": mat(stream, 1e-2)}


def rms(v):
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS)


def reference(t, act, skip, scale, leaves=None):
    """(y, sum of the two terms' magnitudes) in 64 bits, from the leaves if given (for autograd)."""
    get = lambda k: (leaves[k] if leaves is not None else t[k].double()) if t[k] is not None else None
    b = get("branch")
    if t["w_post"] is not None:
        b = rms(b) * get("w_post")
    if t["gate"] is not None:
        b = b * ACTS[act](get("gate"))
    x = skip * get("stream") if t["stream"] is not None else torch.zeros_like(b)
    return x + scale * b, (x.abs() + (scale * b).abs()).detach()


def step(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23


def check(got, ref, size, dtype, what):
    """Half a step of the type, and 2^-19 of the magnitudes that were added up: fp32 arithmetic, the
    exponential (its error grows with the gate, here below 8) and sums over a row."""
    tol = step(dtype) * ref.abs() + 2.0 ** -19 * size + 1e-30
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {((got.double() - ref).abs() / tol).max():.3g}"


def forward_and_check(t, act, skip, scale):
    y, h = api.residual_norm_forward(t["branch"], t["stream"], t["w_post"], t["w_pre"], t["gate"], act, skip, scale, EPS,
                                     t["dtype"])
    ref, size = reference(t, act, skip, scale)
    check(y, ref, size, t["dtype"], "y")
    if t["w_pre"] is not None:
        want = rms(y.double()) * t["w_pre"].double()              # the norm is of the stored stream
        check(h, want, want.abs(), torch.bfloat16, "h")
    else:
        assert h is None
    return y


def backward_and_check(t, y, act, skip, scale):
    got = dict(zip(("stream", "branch", "gate", "w_post", "w_pre"), api.residual_norm_backward(
        t["dh"], t["dy"], t["branch"], y if t["w_pre"] is not None else None, t["w_post"], t["w_pre"], t["gate"], act,
        skip, scale, EPS)))
    leaf = {k: t[k].double().requires_grad_() for k in ("branch", "stream", "w_post", "w_pre", "gate") if t[k] is not None}
    d = t["dy"].double()
    size = d.abs()
    if t["w_pre"] is not None:
        yl = y.double().requires_grad_()
        (rms(yl) * leaf["w_pre"]).backward(t["dh"].double())
        d = d + yl.grad
        r = 1 / torch.sqrt(y.double().square().mean(-1, keepdim=True) + EPS)
        g = (t["dh"].double() * t["w_pre"].double()).abs()
        size = size + r * (g + (y.double() * r).abs() * (g * (y.double() * r).abs()).mean(-1, keepdim=True))
    reference(t, act, skip, scale, leaf)[0].backward(d)
    check(got["stream"], skip * d, abs(skip) * size, t["dtype"], "dx")
    # magnitudes that meet in the branch's gradients: the same chain on absolute values
    b = t["branch"].double()
    gate = ACTS[act](t["gate"].double()).abs() if t["gate"] is not None else 1.0
    r = 1 / torch.sqrt(b.square().mean(-1, keepdim=True) + EPS) if t["w_post"] is not None else 1.0
    w = t["w_post"].double().abs() if t["w_post"] is not None else 1.0
    n, e = (b * r).abs(), abs(scale) * size
    if t["gate"] is not None:
        slope = 2.0 if act != api.GATE_LINEAR else 1.0             # |act'| < 1.1, and the terms it is formed from
        per = e * n * w * slope
        if t["gate"].dim() == 1:
            check(got["gate"], leaf["gate"].grad, per.sum(0), torch.float32, "dgate")
        else:
            check(got["gate"], leaf["gate"].grad, per, torch.bfloat16, "dgate")
    if t["w_post"] is not None:
        check(got["w_post"], leaf["w_post"].grad, (e * gate * n).sum(0), torch.float32, "dw_post")
        q = e * gate * w
        check(got["branch"], leaf["branch"].grad, r * (q + n * (q * n).mean(-1, keepdim=True)), torch.bfloat16, "dbranch")
    else:
        check(got["branch"], leaf["branch"].grad, e * gate, torch.bfloat16, "dbranch")
    if t["w_pre"] is not None:
        yh = rms(y.double()).abs()
        check(got["w_pre"], leaf["w_pre"].grad, (t["dh"].double().abs() * yh).sum(0), torch.float32, "dw_pre")
    return got


PARTS = [dict(zip(("x", "post", "pre", "gate"), v))
         for v in itertools.product((True, False), (True, False), (True, False), ("none", "channel", "element"))]


@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("parts", PARTS, ids=lambda p: "-".join(str(v) for v in p.values()))
def test_every_combination_of_parts(parts, stream):
    t = make(37, 520, stream, seed=1, **parts)
    for act in ACTS if parts["gate"] != "none" else [api.GATE_LINEAR]:
        y = forward_and_check(t, act, 1.0, 0.7071)
        backward_and_check(t, y, act, 1.0, 0.7071)


@pytest.mark.parametrize("tokens,width", [(1, 8), (1, 4096), (2, 16), (5, 248), (64, 256), (700, 264), (3, 4104), (1200, 1032),
                                          (1003, 2048), (9, 8192), (301, 14336), (2, 16384), (2000, 4096)])
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
def test_sizes(tokens, width, stream):
    for gate in ("channel", "element"):
        t = make(tokens, width, stream, gate=gate, seed=tokens + width)
        y = forward_and_check(t, api.GATE_SILU, 0.9, -1.3)
        backward_and_check(t, y, api.GATE_SILU, 0.9, -1.3)


def test_strided_rows_and_padding_are_left_alone():
    t = make(33, 256, seed=5, pad=24)
    y = forward_and_check(t, api.GATE_SIGMOID, 1.0, 1.0)
    backward_and_check(t, y, api.GATE_SIGMOID, 1.0, 1.0)
    buf_y, buf_h = (torch.full((35, 280), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    api.residual_norm_forward(t["branch"], t["stream"], t["w_post"], t["w_pre"], t["gate"], api.GATE_SIGMOID,
                              y=buf_y[1:34, :256], h=buf_h[1:34, :256])
    for b in (buf_y, buf_h):
        assert (b[0] == 7).all() and (b[-1] == 7).all() and (b[:, 256:] == 7).all()
    assert torch.equal(buf_y[1:34, :256], y)


def test_in_place():
    t = make(50, 512, seed=6)
    args = (t["w_post"], t["w_pre"], t["gate"], api.GATE_SILU)
    y, h = api.residual_norm_forward(t["branch"], t["stream"], *args)
    x = t["stream"].clone()
    y2, h2 = api.residual_norm_forward(t["branch"], x, *args, y=x)
    assert y2 is x and torch.equal(x, y) and torch.equal(h, h2)
    want = api.residual_norm_backward(t["dh"], t["dy"], t["branch"], y, *args)
    dy, dh = t["dy"].clone(), t["dh"].clone()
    got = api.residual_norm_backward(dh, dy, t["branch"], y, *args, dstream=dy, dbranch=dh)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_calls_repeat_bit_for_bit():
    t = make(3000, 1024, gate="channel", seed=7)
    y, _ = api.residual_norm_forward(t["branch"], t["stream"], t["w_post"], t["w_pre"], t["gate"])
    runs = [api.residual_norm_backward(t["dh"], t["dy"], t["branch"], y, t["w_post"], t["w_pre"], t["gate"])
            for _ in range(3)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


def test_zero_rows_huge_rows_and_saturated_gates():
    """A zero row has no direction but a finite norm; gates at the ends of the type close or open."""
    t = make(8, 256, seed=8)
    t["branch"][0], t["stream"][0] = 0.0, 0.0
    t["branch"][1] *= 1e15
    t["gate"][2], t["gate"][3], t["gate"][4] = -3e38, 3e38, -float("inf")
    y, h = api.residual_norm_forward(t["branch"], t["stream"], t["w_post"], t["w_pre"], t["gate"], api.GATE_SIGMOID)
    ref, size = reference(t, api.GATE_SIGMOID, 1.0, 1.0)
    check(y, ref, size, torch.bfloat16, "y")
    assert (y[0] == 0).all() and (h[0] == 0).all() and torch.isfinite(h).all()
    assert torch.equal(y[2], t["stream"][2]) and torch.equal(y[4], t["stream"][4])
    got = api.residual_norm_backward(t["dh"], t["dy"], t["branch"], y, t["w_post"], t["w_pre"], t["gate"], api.GATE_SIGMOID)
    assert all(torch.isfinite(g).all() for g in got)
    assert (got[2][2] == 0).all() and (got[2][3] == 0).all() and (got[1][4] == 0).all()


def test_gradient_against_differences():
    """Directional differences of the 64-bit forward map (fp32 stream: its rounding is far below the step)."""
    t = make(6, 128, torch.float32, gate="element", seed=9)
    y, _ = api.residual_norm_forward(t["branch"], t["stream"], t["w_post"], t["w_pre"], t["gate"], api.GATE_SILU)
    got = dict(zip(("stream", "branch", "gate", "w_post", "w_pre"), api.residual_norm_backward(
        t["dh"], t["dy"], t["branch"], y, t["w_post"], t["w_pre"], t["gate"], api.GATE_SILU)))
    base = {k: t[k].double() for k in got}

    def loss(v):
        y = reference(t, api.GATE_SILU, 1.0, 1.0, v)[0]
        return ((rms(y) * v["w_pre"] * t["dh"].double()).sum() + (y * t["dy"].double()).sum()).item()

    g = torch.Generator(device="cuda").manual_seed(1)
    for k in got:
        d = torch.randn(base[k].shape, generator=g, device="cuda", dtype=torch.float64)
        eps = 1e-5
        diff = (loss({**base, k: base[k] + eps * d}) - loss({**base, k: base[k] - eps * d})) / (2 * eps)
        # bf16 gradients carry half a step each, in random directions: four standard deviations of that sum
        tol = 4 * 2.0 ** -9 * (got[k].double() * d).norm().item() + 1e-7 * (got[k].double() * d).abs().sum().item()
        assert abs((got[k].double() * d).sum().item() - diff) <= tol, k
