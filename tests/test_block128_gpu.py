"""The 8-bit product with one fp32 scale per 128 elements on the GPU against its definition in 64 bits:
codes and scales bit for bit, products within the bound of the arithmetic."""
import numpy as np
import pytest
import torch

from gpu_util import random_bits, to_dev
from paper_2605_09825_b200 import api, synth

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -100


def blocks(x, per_row):
    r, c = x.shape
    p = np.zeros((-(-r // per_row) * per_row, -(-c // 128) * 128))
    p[:r, :c] = x
    return p.reshape(p.shape[0] // per_row, per_row, p.shape[1] // 128, 128)


def e4m3_codes(v):
    """Codes of fp64 values: nearest, ties to even, saturating, sign kept on zero."""
    a = np.abs(v)
    e = np.clip(np.frexp(a)[1] - 1, -6, None)
    q = np.rint(np.ldexp(a, 3 - e))                              # in steps of the last bit
    up = q >= 16
    e, q = np.where(up, e + 1, e), np.where(up, 8, q)
    code = np.where(q < 8, q, (e + 7) * 8 + (q - 8)).astype(np.int64)
    return (np.minimum(code, 0x7E) | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def quantize(bits, axis, square):
    """Codes [outer, K] and scales [outer blocks or rows, K blocks] of the definition."""
    x = synth.bf16_bits_to_f32(bits if axis == 1 else np.ascontiguousarray(bits.T)).astype(np.float64)
    v = blocks(x, 128 if square else 1)
    a = np.maximum(np.abs(v).max(axis=(1, 3), keepdims=True), TINY)
    inv = (448.0 / a).astype(np.float32).astype(np.float64)
    scales = (a / 448.0).astype(np.float32)[:, 0, :, 0]
    codes = e4m3_codes((v * inv).astype(np.float32).astype(np.float64))
    return codes.reshape(codes.shape[0] * codes.shape[1], -1)[: x.shape[0], : x.shape[1]], scales


def values(codes):
    return torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()


def check_quantize(bits, axis, square, src=None):
    shape = api.BLOCK_128X128 if square else api.BLOCK_1X128
    codes, scales = api.quantize_block128(to_dev(bits) if src is None else src, axis, shape)
    api.check()
    want_c, want_s = quantize(bits, axis, square)
    got_s = scales.cpu().numpy()
    assert np.array_equal(got_s[:, : want_s.shape[0]], want_s.T)
    if not square:
        assert (got_s[:, want_s.shape[0]:] == 0).all()            # rows past the last one
    bad = np.argwhere(codes.cpu().numpy() != want_c)
    assert bad.size == 0, f"{len(bad)} codes differ, first at {bad[:4].tolist()}"


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("axis", [1, 0])
@pytest.mark.parametrize("rows,cols", [(16, 16), (1, 16), (16, 1), (128, 128), (144, 272), (300, 416), (1000, 1184),
                                       (1040, 131), (96, 24)])
def test_quantize_ragged_shapes(rows, cols, axis, square):
    if (cols if axis == 1 else rows) % 16:
        pytest.skip("the reduction axis comes in multiples of 16")
    rng = np.random.default_rng(rows * 7 + cols)
    ld = -(-cols // 8) * 8 + 8
    full = random_bits(rng, rows, ld, 8)
    check_quantize(np.ascontiguousarray(full[:, :cols]), axis, square, to_dev(full)[:, :cols])


@pytest.mark.parametrize("axis", [1, 0])
def test_quantize_every_finite_bf16_pattern(axis):
    """Every pattern below a block maximum of 448 (scale 1, sub-normal codes included) and beside larger
    ones, zero blocks, blocks of sub-normal numbers."""
    pats = np.arange(1 << 16, dtype=np.uint16)
    pats = pats[(pats & 0x7F80) != 0x7F80]
    small = pats[(pats & 0x7FFF) <= 0x43E0]                      # up to 448
    n = -(-len(small) // 127)
    bits = np.zeros((n, 128), dtype=np.uint16)
    flat = np.zeros(n * 127, dtype=np.uint16)
    flat[: len(small)] = small
    bits[:, 0], bits[:, 1:] = 0x43E0, flat.reshape(n, 127)
    rest = np.zeros(-(-len(pats) // 128) * 128, dtype=np.uint16)
    rest[: len(pats)] = pats
    extra = np.zeros((2, 128), dtype=np.uint16)
    extra[1] = np.arange(128)                                    # sub-normal bf16
    bits = np.concatenate([bits, rest.reshape(-1, 128), extra])
    bits = bits[: len(bits) // 16 * 16]
    check_quantize(bits if axis == 1 else np.ascontiguousarray(bits.T), axis, False)


def product(a_codes, a_scales, b_codes, b_scales, square):
    """64-bit product and the sum of its terms' magnitudes; scales [rows or row blocks, K blocks]."""
    sp = lambda s, per, n, K: np.repeat(np.repeat(s.astype(np.float64), per, 0), 128, 1)[:n, :K]
    (M, K), N = a_codes.shape, b_codes.shape[0]
    A = values(a_codes) * sp(a_scales, 1, M, K)
    B = values(b_codes) * sp(b_scales, 128 if square else 1, N, K)
    A, B = torch.from_numpy(A).cuda(), torch.from_numpy(B).cuda()
    return (A @ B.t()).cpu().numpy(), (A.abs() @ B.abs().t()).cpu().numpy()


def tolerance(ref, S, K, bf16):
    """Four chained K = 32 instructions per block, each truncating its sums at the fp32 accumulator's last bit
    (taken as two units of 2^-23 of the block's magnitudes each), three roundings for the scales, one
    per block for the sum outside; half a bf16 step on top for bf16."""
    return (8 + 2 + 0.5 * -(-K // 128)) * 2.0 ** -23 * S + (2.0 ** -8 * np.abs(ref) if bf16 else 0.0) + 1e-38


def device_scales(s, square):
    """[rows or row blocks, K blocks] as the kernels read them."""
    t = np.ascontiguousarray(s.T)
    if not square:
        t = np.pad(t, ((0, 0), (0, -t.shape[1] % 128)))
    return torch.from_numpy(t.astype(np.float32)).cuda()


def random_operands(rng, M, N, K, square):
    def one(rows, per):
        codes = rng.integers(0, 256, (rows, K)).astype(np.uint8)
        codes[(codes & 0x7F) == 0x7F] ^= 0x11
        s = np.exp2(rng.uniform(-8, 4, (-(-rows // per), -(-K // 128)))).astype(np.float32)
        return codes, s
    return one(M, 1) + one(N, 128 if square else 1)


def run_gemm(ops, square, out_dtype, out=None):
    a_codes, a_scales, b_codes, b_scales = ops
    dev = lambda x: torch.from_numpy(x).cuda()
    got = api.gemm_block128(dev(a_codes), device_scales(a_scales, False), dev(b_codes), device_scales(b_scales, square),
                            api.BLOCK_128X128 if square else api.BLOCK_1X128, out_dtype, out)
    api.check()
    return got


SHAPES = [(8, 1000, 272), (9, 40, 4096), (16, 4096, 1040), (17, 520, 4096), (40, 4096, 2048), (256, 256, 128), (1, 8, 16), (1, 4096, 4096), (3, 520, 1040), (77, 200, 96), (128, 256, 2048), (129, 257 + 7, 400),
          (300, 392, 272), (512, 1000, 1184), (600, 24, 4112), (1100, 2056, 640), (2300, 4104, 256)]


@pytest.mark.parametrize("square", [True, False])
@pytest.mark.parametrize("out_dtype", [api.OUT_FP32, api.OUT_BF16])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_random_codes(M, N, K, out_dtype, square):
    ops = random_operands(np.random.default_rng(M + N + K), M, N, K, square)
    got = run_gemm(ops, square, out_dtype)
    ref, S = product(*ops, square)
    tol = tolerance(ref, S, K, out_dtype == api.OUT_BF16)
    bad = ~(np.abs(got.double().cpu().numpy() - ref) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} out of tolerance, first at {np.argwhere(bad)[:4].tolist()}"
    assert torch.equal(got, run_gemm(ops, square, out_dtype)), "two runs differ"


@pytest.mark.parametrize("M,N,K", [(1, 515, 2048), (40, 1001, 512), (257, 771, 128)])
@pytest.mark.parametrize("out_dtype", [api.OUT_FP32, api.OUT_BF16])
def test_gemm_writes_its_matrix_and_nothing_else(M, N, K, out_dtype):
    """Column counts that are not whole 16-byte pieces, inside a larger buffer filled with a marker."""
    ops = random_operands(np.random.default_rng(N), M, N, K, True)
    ld = -(-N // 8) * 8 + 16
    buf = torch.full((M + 2, ld), 7.0, dtype=torch.float32 if out_dtype == api.OUT_FP32 else torch.bfloat16, device="cuda")
    got = run_gemm(ops, True, out_dtype, buf[1: M + 1, :N])
    ref, S = product(*ops, True)
    assert (np.abs(got.double().cpu().numpy() - ref) <= tolerance(ref, S, K, out_dtype == api.OUT_BF16)).all()
    assert (buf[0] == 7).all() and (buf[-1] == 7).all() and (buf[:, N:] == 7).all()


# a full wave of tiles and a few left over, which are split along K; ragged in both directions
@pytest.mark.parametrize("square", [True, False])
@pytest.mark.parametrize("out_dtype", [api.OUT_FP32, api.OUT_BF16])
@pytest.mark.parametrize("M,N,K", [(40, 75 * 256 + 8, 2064), (300, 38 * 256 - 8, 2048), (2049, 2304, 2064)])
def test_gemm_left_over_tiles(M, N, K, out_dtype, square):
    assert api.load_library().mxfp4_gemm_block128_workspace_bytes(M, N, K) > 0
    test_gemm_random_codes(M, N, K, out_dtype, square)
    if square:
        test_gemm_writes_its_matrix_and_nothing_else(M, N - 5, K, out_dtype)


def test_gemm_long_reduction_of_one_sign():
    """Products of one sign are where truncating additions show: with a chain of four instructions per
    block the error stays at the fp32 sum's own level however long the reduction is."""
    K = 28672
    rng = np.random.default_rng(3)
    a, b = (rng.integers(0x30, 0x60, (n, K)).astype(np.uint8) for n in (64, 128))
    ops = (a, np.ones((64, K // 128), np.float32), b, np.ones((1, K // 128), np.float32))
    ref, S = product(*ops, True)
    err = np.abs(run_gemm(ops, True, api.OUT_FP32).double().cpu().numpy() - ref) / S
    assert err.max() < 2e-6, err.max()


@pytest.mark.parametrize("pass_,T,in_f,out_f", [(0, 333, 416, 264), (1, 300, 520, 272), (2, 400, 264, 392),
                                                (0, 1, 4096, 512), (2, 16, 8, 24), (1, 1000, 1024, 2048)])
def test_linear_pass(pass_, T, in_f, out_f):
    rng = np.random.default_rng(T + in_f)
    X, W, dY = random_bits(rng, T, in_f, 3), random_bits(rng, out_f, in_f, 2), random_bits(rng, T, out_f, 4)
    a, b = ((X, W), (dY, W), (dY, X))[pass_]
    (ax_a, ax_b), square = ((1, 1), (1, 0), (0, 0))[pass_], pass_ != 2
    ac, as_ = quantize(a, ax_a, False)
    bc, bs = quantize(b, ax_b, square)
    ref, S = product(ac, as_, bc, bs, square)
    got = api.linear_pass_block128(pass_, to_dev(a), to_dev(b), api.OUT_FP32)
    api.check()
    assert (np.abs(got.double().cpu().numpy() - ref) <= tolerance(ref, S, ac.shape[1], False)).all()
    half = api.linear_pass_block128(pass_, to_dev(a), to_dev(b), api.OUT_BF16)
    assert torch.equal(half, got.bfloat16()), "bf16 output is not the fp32 output rounded once"


def test_pass_on_a_stream_of_its_own():
    rng = np.random.default_rng(9)
    X, W = to_dev(random_bits(rng, 260, 512, 2)), to_dev(random_bits(rng, 640, 512, 2))
    want = api.linear_pass_block128(api.PASS_FPROP, X, W)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = api.linear_pass_block128(api.PASS_FPROP, X, W)
    side.synchronize()
    assert torch.equal(got, want)


def with_value(bits, places, value):
    """A copy with a bf16 pattern put in some places."""
    out = bits.copy()
    for r, c in places:
        out[r, c] = value
    return out


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("axis", [1, 0])
@pytest.mark.parametrize("nan", [0x7FC0, 0xFF81])
def test_quantize_nan_takes_its_block_and_no_other(axis, square, nan):
    """One NaN makes its block's scale and codes NaN; all other blocks are what they are without it."""
    bits = random_bits(np.random.default_rng(4), 304, 416, 3)
    clean = api.quantize_block128(to_dev(bits), axis, api.BLOCK_128X128 if square else api.BLOCK_1X128)
    at = [(17, 140), (303, 415)]
    codes, scales = api.quantize_block128(to_dev(with_value(bits, at, nan)), axis,
                                          api.BLOCK_128X128 if square else api.BLOCK_1X128)
    api.check()
    blocks_hit = torch.zeros_like(scales, dtype=torch.bool)
    codes_hit = torch.zeros_like(codes, dtype=torch.bool)
    for r, c in at:
        o, k = (r, c) if axis == 1 else (c, r)
        t, row = k // 128, o // 128 if square else o
        blocks_hit[t, row] = True
        rows = slice(row * 128, row * 128 + 128) if square else slice(o, o + 1)
        codes_hit[rows, t * 128: t * 128 + 128] = True
    assert torch.isnan(scales[blocks_hit]).all() and torch.equal(scales[~blocks_hit], clean[1][~blocks_hit])
    assert ((codes[codes_hit] & 0x7F) == 0x7F).all() and torch.equal(codes[~codes_hit], clean[0][~codes_hit])


@pytest.mark.parametrize("M", [3, 40])
@pytest.mark.parametrize("value", [0x7FC0, 0x7F80, 0xFF80])
def test_nan_and_infinity_reach_every_product_of_their_block(M, value):
    """A row of A, and the 128 columns that share a block of B, are NaN; everything else is as without them."""
    rng = np.random.default_rng(M)
    a, b = random_bits(rng, M, 272, 2), random_bits(rng, 400, 272, 2)
    mul = lambda x, y: api.gemm_block128(*api.quantize_block128(to_dev(x)),
                                         *api.quantize_block128(to_dev(y), api.AXIS_COLS, api.BLOCK_128X128), out_dtype=api.OUT_FP32)
    clean = mul(a, b)
    got = mul(with_value(a, [(2, 270)], value), b)
    assert torch.isnan(got[2]).all()
    got[2] = clean[2]
    assert torch.equal(got, clean)
    got = mul(a, with_value(b, [(130, 3)], value))
    api.check()
    assert torch.isnan(got[:, 128:256]).all()
    got[:, 128:256] = clean[:, 128:256]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("M,N,K", [(1, 515, 144), (3, 1, 272), (40, 515, 272), (300, 1001, 400)])
@pytest.mark.parametrize("out_dtype", [api.OUT_FP32, api.OUT_BF16])
def test_gemm_makes_room_for_ragged_columns(M, N, K, out_dtype):
    """Without `out` any number of columns works: the binding pads the rows it allocates."""
    ops = random_operands(np.random.default_rng(N + K), M, N, K, True)
    got = run_gemm(ops, True, out_dtype)
    assert got.shape == (M, N)
    ref, S = product(*ops, True)
    assert (np.abs(got.double().cpu().numpy() - ref) <= tolerance(ref, S, K, out_dtype == api.OUT_BF16)).all()
