"""Token embeddings against the definition in 64 bits.

Bounds.  The lookup rounds one product: half a step of the result's type.  A sum of n fp32 terms is off by at most
n * 2^-24 of the sum of their magnitudes (every addition rounds a partial sum that is no larger), the scaling and the
result's type add their half steps.  Gradients that are small whole numbers make every sum exact.
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
OUT = {BF16: api.OUT_BF16, FP32: api.OUT_FP32}


def gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make_ids(kind, tokens, vocab, gen):
    if kind == "same":
        return torch.full((tokens,), vocab // 2, device="cuda")
    if kind == "ascending":
        return torch.arange(tokens, device="cuda") % vocab
    if kind == "descending":
        return vocab - 1 - torch.arange(tokens, device="cuda") % vocab
    if kind == "none":
        return torch.full((tokens,), -1, device="cuda")
    u = torch.rand(tokens, generator=gen, device="cuda")
    ids = (vocab ** u - 1).long().clamp(max=vocab - 1) if kind == "text" else (u * vocab).long().clamp(max=vocab - 1)
    ids[torch.rand(tokens, generator=gen, device="cuda") < 0.05] = -1
    ids[torch.rand(tokens, generator=gen, device="cuda") < 0.02] = vocab + 3
    ids[-1], ids[0] = vocab - 1, 0
    return ids


@pytest.mark.parametrize("tokens,width,vocab", [(1, 8, 1), (1, 4096, 100), (3, 24, 7), (130, 264, 1000), (1025, 2056, 333)])
@pytest.mark.parametrize("kind", [BF16, FP32])
@pytest.mark.parametrize("out", [BF16, FP32])
def test_lookup(tokens, width, vocab, kind, out):
    gen = gen_of(tokens)
    table = torch.randn(vocab, width, generator=gen, device="cuda").to(kind)
    ids = make_ids("uniform", tokens, vocab, gen)
    got = api.embedding_forward(ids, table, 1.7, OUT[out])
    api.check()
    scale = torch.tensor(1.7).double().item()
    inside = (ids >= 0) & (ids < vocab)
    want = table.double()[ids.clamp(0, vocab - 1)] * scale
    assert got.dtype == out
    assert ((got.double() - want).abs() <= (STEP[out] + 2.0 ** -24) * want.abs())[inside].all()
    assert (got[ids < 0] == 0).all() and got[ids >= vocab].isnan().all()
    if out == kind:
        assert torch.equal(api.embedding_forward(ids, table)[inside], table[ids[inside]])


def reference(ids, d, vocab, scale):
    has = ((ids >= 0) & (ids < vocab)).nonzero()[:, 0]
    ref = torch.zeros(vocab, d.shape[1], dtype=torch.float64, device="cuda")
    return ref.index_put_((ids[has],), d.double()[has] * scale, accumulate=True)


IDS = ["uniform", "text", "same", "ascending", "descending", "none"]
SIZES = [(1, 8, 1), (1, 4096, 1000), (31, 24, 5), (32, 256, 40), (33, 264, 100000), (777, 2048, 3201), (1025, 72, 511),
         (1025, 72, 512), (5000, 136, 128256), (40000, 16, 300000)]


@pytest.mark.parametrize("tokens,width,vocab", SIZES)
@pytest.mark.parametrize("which", IDS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_whole_numbers_is_exact(tokens, width, vocab, which, accumulate):
    gen = gen_of(tokens + vocab)
    ids = make_ids(which, tokens, vocab, gen)
    d = torch.randint(-3, 4, (tokens, width), generator=gen, device="cuda").to(BF16)
    old = torch.randint(-9, 10, (vocab, width), generator=gen, device="cuda").float()
    table = old.clone() if accumulate else torch.full_like(old, float("nan"))
    got = api.embedding_backward(ids, d, vocab, 2.0, d_table=table, accumulate=accumulate)
    api.check()
    assert got is table
    assert torch.equal(got.double(), reference(ids, d, vocab, 2.0) + (old.double() if accumulate else 0))


@pytest.mark.parametrize("kind", [BF16, FP32])
@pytest.mark.parametrize("out", [BF16, FP32])
@pytest.mark.parametrize("tokens,width,vocab", [(33, 264, 1000), (3000, 520, 700), (9000, 72, 32001)])
def test_gradient(kind, out, tokens, width, vocab):
    gen = gen_of(tokens)
    ids = make_ids("text", tokens, vocab, gen)
    d = torch.randn(tokens, width, generator=gen, device="cuda").to(kind)
    scale = torch.tensor(0.37, dtype=FP32).double().item()
    got = api.embedding_backward(ids, d, vocab, 0.37, OUT[out])
    again = api.embedding_backward(ids, d, vocab, 0.37, OUT[out])
    api.check()
    assert got.dtype == out and torch.equal(got, again)
    ref, size = reference(ids, d, vocab, scale), reference(ids, d.abs(), vocab, scale)
    count = torch.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab)[:, None]
    assert ((got.double() - ref).abs() <= (count + 1) * 2.0 ** -24 * size + STEP[out] * ref.abs()).all()


def test_gradient_against_differences():
    """The lookup is linear in the table: its change along a direction, summed with d_out, is the direction's inner product
    with the gradient, up to 64-bit rounding of the formula's own."""
    gen = gen_of(9)
    table = torch.randn(50, 24, generator=gen, device="cuda")
    ids = make_ids("text", 200, 50, gen).clamp(max=49)
    d = torch.randn(200, 24, generator=gen, device="cuda")
    grad = api.embedding_backward(ids, d, 50, 1.5)
    move = torch.randn(50, 24, generator=gen, device="cuda")
    out = [api.embedding_forward(ids, t, 1.5).double() for t in (table + move, table - move)]
    slope = ((out[0] - out[1]) * d.double()).sum() / 2
    # the table's sums, the lookups and the gradient round to fp32: 200 terms of the row
    size = (d.abs().double() * 1.5 * (table.abs() + move.abs()).max()).sum()
    assert abs(slope - (grad.double() * move.double()).sum()) <= 200 * 2.0 ** -24 * size


def test_only_rows_with_tokens_are_touched_when_adding():
    ids = torch.tensor([4, -1, 4, 9, 200], device="cuda")
    room = torch.full((12, 40), 7.0, device="cuda")
    table = room[1:-1, 8:-8]
    table[4] = float("inf")
    api.embedding_backward(ids, torch.ones(5, 24, dtype=BF16, device="cuda"), 10, d_table=table, accumulate=True)
    api.check()
    want = torch.full((12, 40), 7.0, device="cuda")
    want[1:-1, 8:-8][9] = 8
    want[1:-1, 8:-8][4] = float("inf")
    assert torch.equal(room, want)


def test_strides_and_untouched_surroundings():
    gen = gen_of(3)
    ids = make_ids("text", 300, 90, gen)
    d = torch.randn(302, 80, generator=gen, device="cuda").bfloat16()[1:-1, 8:-8]
    for kind in (BF16, FP32):
        room = torch.full((92, 80), 7.0, dtype=kind, device="cuda")
        got = api.embedding_backward(ids, d, 90, d_table=room[1:-1, 8:-8])
        assert torch.equal(got, api.embedding_backward(ids, d.contiguous(), 90, out_dtype=OUT[kind]))
        assert (room[0] == 7).all() and (room[-1] == 7).all() and (room[:, :8] == 7).all() and (room[:, -8:] == 7).all()
        out = torch.full((302, 80), 7.0, dtype=kind, device="cuda")
        api.embedding_forward(ids, got, 2.0, out=out[1:-1, 8:-8])
        assert torch.equal(out[1:-1, 8:-8].nan_to_num(5), api.embedding_forward(ids, got.contiguous(), 2.0).nan_to_num(5))
        assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, :8] == 7).all() and (out[:, -8:] == 7).all()
    api.check()


def test_a_large_table():
    """Rows past 2^32 bytes, and past 2^31 elements."""
    vocab, width = 270000, 8192
    ids = torch.tensor([0, vocab - 1, 262143, vocab - 1, 131072], device="cuda")
    d = torch.ones(5, width, dtype=BF16, device="cuda")
    table = torch.full((vocab, width), 5.0, dtype=BF16, device="cuda")
    api.embedding_backward(ids, d, vocab, d_table=table)
    out = api.embedding_forward(ids, table)
    api.check()
    assert (out[[0, 2, 4]] == 1).all() and (out[[1, 3]] == 2).all()
    assert int(table.count_nonzero()) == 4 * width


def test_as_a_graph():
    gen = gen_of(4)
    ids = make_ids("text", 500, 900, gen)
    table = torch.randn(900, 136, generator=gen, device="cuda")

    def step():
        out = api.embedding_forward(ids, table, 3.0)
        return out, api.embedding_backward(ids, out, 900, 3.0)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    ids.copy_(make_ids("uniform", 500, 900, gen))
    graph.replay()
    api.check()
    assert all(torch.equal(a.nan_to_num(3), b.nan_to_num(3)) for a, b in zip(got, step()))
