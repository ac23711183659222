"""How long a sum the 16-bit product takes: below 2^30 elements, below 2^29 for the sum of two products.  Found on the host before
anything is launched, the same for every number of tokens.  No GPU needed."""
import ctypes

import pytest

from paper_2605_09825_b200 import api, build

LONGEST = (1 << 30) - 64


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return api.load_library()


@pytest.fixture(scope="module")
def p():
    buf = ctypes.create_string_buffer(1 << 14)
    p.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def gated(p, tokens, in_features, features):
    return ctypes.byref(api.GatedDesc(tokens, in_features, features, p, in_features, p, in_features, p, in_features, 2))


# a number of tokens for each of the three kernels
@pytest.mark.parametrize("tokens", [1, 8, 9, 160, 300, 512])
@pytest.mark.parametrize("in_features", [LONGEST + 8, 1 << 30, 0x7FFFFF00 - 2048, 0x7FFFFF00])
def test_gated_forward(lib, p, tokens, in_features):
    assert lib.mxfp4_gated_linear_forward(gated(p, tokens, in_features, 8), p, 8, p, p, 8, None) == -2


def backward(lib, p, tokens, in_features, features):
    return lib.mxfp4_gated_linear_backward(gated(p, tokens, in_features, features), p, features, p, p, features, p, in_features, p, p,
                                           in_features, 0, p, (1 << 64) - 1, None)


@pytest.mark.parametrize("sizes", [(8, 1 << 30, 8), ((1 << 30) - 56, 8, 8), (8, 8, (1 << 29) - 56), (8, 8, 1 << 30)])
def test_gated_backward(lib, p, sizes):
    assert backward(lib, p, *sizes) == -2
    assert lib.mxfp4_gated_linear_workspace_bytes(*sizes) == 0


def test_loss(lib, p):
    def fwd(T, D):
        return lib.mxfp4_linear_logprobs_forward(p, D, p, D, T, D, 8, p, 1.0, p, p, p, (1 << 64) - 1, None)

    def bwd(T, D):
        return lib.mxfp4_linear_logprobs_backward(p, D, p, D, T, D, 8, p, 1.0, p, p, p, p, D, p, D, 0, p, (1 << 64) - 1, None)

    assert fwd(4, LONGEST + 8) == bwd(4, LONGEST + 8) == fwd(4, 0x7FFFFF00) == -2
    assert bwd((1 << 30) - 56, 8) == -2
    size = lib.mxfp4_linear_logprobs_workspace_bytes
    assert size(4, LONGEST + 8, 8, 0) == size(4, LONGEST + 8, 8, 1) == size((1 << 30) - 56, 8, 8, 1) == 0
    assert size((1 << 30) - 56, 8, 8, 0) > 0             # a text of any length is scored piece by piece


def test_the_longest_are_taken(lib, p):
    """They pass the checks of their sizes: what stops them here is the workspace, looked at after these."""
    d = gated(p, 8, LONGEST, 8)
    assert lib.mxfp4_gated_linear_backward(d, p, 8, p, p, 8, p, LONGEST, p, p, LONGEST, 0, None, 0, None) == -5
    d = gated(p, LONGEST, 8, 8)
    assert lib.mxfp4_gated_linear_backward(d, p, 8, p, p, 8, p, 8, p, p, 8, 0, None, 0, None) == -5
    d = gated(p, 8, 8, (1 << 29) - 64)
    F = (1 << 29) - 64
    assert lib.mxfp4_gated_linear_backward(d, p, F, p, p, F, p, 8, p, p, 8, 0, None, 0, None) == -5
    assert lib.mxfp4_linear_logprobs_forward(p, LONGEST, p, LONGEST, 4, LONGEST, 8, p, 1.0, p, p, None, 0, None) == -5
