"""Gradient norm and clipping against 64 bits.

Bounds.  A sum of the squares of eight elements in fp32 is off by 8 * 2^-24 of itself, the rest is in fp64; the norm's
relative error is half of that and its own rounding: 5 * 2^-24.  A clipped element carries the norm's error, three
roundings of the factor and its own half step.
"""
import pytest
import torch

from paper_2605_09825_b200 import api

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def memory_returned():
    """What the large cases had goes back to the device: the allocator would otherwise give it back in some later test,
    which waits for all of the device's work."""
    yield
    torch.cuda.empty_cache()


BF16, FP32 = torch.bfloat16, torch.float32
STEP = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}
NORM = 5 * 2.0 ** -24


def norm64(tensors):
    return sum(t.double().square().sum() for t in tensors).sqrt() if tensors else 0.0


def make(sizes, kinds, seed=0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n + offset, generator=gen, device="cuda").to(kinds[i % len(kinds)])[offset:] for i, n in enumerate(sizes)]


def check_clip(tensors, max_norm, out, norm, eps=1e-6):
    want = norm64(tensors)
    assert abs(norm.double() - want) <= NORM * want
    factor = min(1.0, max_norm / (float(want) + eps))
    for t, o in zip(tensors, out):
        ref = t.double() * factor
        assert o.shape == t.shape
        assert ((o.double() - ref).abs() <= (STEP[o.dtype] + NORM + 4 * 2.0 ** -24) * ref.abs() + 1e-45).all()


SIZES = [[1], [7], [16384], [16385, 1, 3], [5, 0, 100001, 8], [40000] * 20, list(range(1, 300)), [3] * 700 + [100000], [1 << 22, 33]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("kinds", [[BF16], [FP32], [BF16, FP32]], ids=["bf16", "fp32", "mixed"])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_norm_and_clip(sizes, kinds, offset):
    tensors = make(sizes, kinds, offset=offset)
    norm = api.grad_norm(tensors)
    assert norm.shape == () and norm.dtype == FP32
    for max_norm in (0.3, 1e9):
        for out_kinds in (kinds, kinds[::-1], [FP32], [BF16]):
            out = [torch.full((t.numel() + 2,), 7.0, dtype=out_kinds[i % len(out_kinds)], device="cuda") for i, t in enumerate(tensors)]
            inner = [o[1:-1] for o in out]
            got = api.clip_grads(tensors, max_norm, inner)
            assert torch.equal(got, norm)
            check_clip(tensors, max_norm, inner, got)
            assert all(o[0] == 7 and o[-1] == 7 for o in out)
    copies = [t.clone() for t in tensors]
    got = api.clip_grads(copies, 0.5)
    api.check()
    # a copy starts at another alignment, so other elements share a fp32 sum: both norms are within NORM of the exact one
    assert abs(got.double() - norm.double()) <= 2 * NORM * norm.double()
    check_clip(tensors, 0.5, copies, got)


def test_in_place_below_the_limit_changes_nothing():
    tensors = make([1000, 33], [BF16, FP32])
    copies = [t.clone() for t in tensors]
    api.clip_grads(copies, float("inf"))
    api.clip_grads(copies, float(norm64(tensors)) * 1.01)
    api.check()
    assert all(torch.equal(a, b) for a, b in zip(tensors, copies))


@pytest.mark.parametrize("size", [1e-40, 1e-30, 1e-22, 1e-15, 1e15, 1e19, 1e30])
@pytest.mark.parametrize("kind", [BF16, FP32])
def test_elements_whose_squares_leave_fp32(size, kind):
    tensors = [(t.float() * size).to(kind) for t in make([1000, 17], [FP32])]
    want = norm64(tensors)
    norm = api.grad_norm(tensors)
    api.check()
    assert abs(norm.double() - want) <= NORM * want + 2.0 ** -149


def test_small_elements_beside_large_ones():
    t = torch.full((8192,), 1e-3, device="cuda")
    t[5] = 1e4
    want = norm64([t])
    assert abs(api.grad_norm([t]).double() - want) <= NORM * want
    one = torch.zeros(4096, device="cuda")
    one[4000] = 3e-30
    assert abs(api.grad_norm([one]).double() - 3e-30) <= 1e-6 * 3e-30
    assert api.grad_norm([torch.zeros(100, device="cuda"), -torch.zeros(9, device="cuda")]) == 0
    api.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kind", [BF16, FP32])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad, kind):
    for at in (0, 3, 16384, 20004):
        tensors = make([20005, 9], [kind])
        tensors[0][at] = bad
        copies = [t.clone() for t in tensors]
        out = [torch.zeros_like(t) for t in tensors]
        norms = [api.grad_norm(tensors), api.clip_grads(copies, 1.0), api.clip_grads(tensors, 1.0, out)]
        api.check()
        assert all(n.isnan() if bad != bad else n == float("inf") for n in norms)
        for t, c, o in zip(tensors, copies, out):
            same = lambda a, b: torch.equal(a.nan_to_num(5, 6, 7), b.nan_to_num(5, 6, 7))
            assert same(t, c) and same(t, o)


def test_a_norm_past_fp32():
    tensors = [torch.full((100,), 3e38, device="cuda")]
    copy = tensors[0].clone()
    assert api.clip_grads([copy], 1.0) == float("inf")
    api.check()
    assert torch.equal(copy, tensors[0])


def test_zero_limit_and_zero_gradients():
    t = make([100], [FP32])
    z = torch.zeros(100, device="cuda")
    api.clip_grads(t, 0.0)
    assert (t[0] == 0).all()
    assert api.clip_grads([z], 0.0, eps=0.0) == 0 and (z == 0).all()
    api.check()


def test_repeats_bit_for_bit_and_as_a_graph():
    tensors = make([100000, 31, 7000, 1 << 20], [BF16, FP32])
    out = [torch.empty_like(t) for t in tensors]
    norm = api.clip_grads(tensors, 0.7, out)
    first = [o.clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = api.clip_grads(tensors, 0.7, out)
    for o in out:
        o.zero_()
    graph.replay()
    api.check()
    assert torch.equal(norm, replayed) and all(torch.equal(a, b) for a, b in zip(first, out))
    for t in tensors:
        t.mul_(2)
    graph.replay()
    assert abs(replayed.double() - 2 * norm.double()) <= 2 * NORM * norm.double()


def test_a_shape_of_its_own_and_many_more_tensors_than_a_launch_takes():
    gen = torch.Generator(device="cuda").manual_seed(1)
    flat = torch.randn(2000 * 24, generator=gen, device="cuda")
    tensors = [flat[i * 24: i * 24 + 20].view(4, 5) for i in range(2000)]
    out = [torch.empty(20, dtype=BF16, device="cuda") for _ in tensors]
    norm = api.clip_grads(tensors, 2.0, out)
    api.check()
    check_clip([t.flatten() for t in tensors], 2.0, out, norm)
