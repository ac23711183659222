"""The kernels at the two ends of a training step reach elements of shared arrays through the checked helpers, and every
unit's status word is looked at, as the bounds-checking build promises.  Read from the sources; no GPU needed."""
import os
import re

import pytest

from paper_2605_09825_b200 import build

# how each file writes an element of one of its shared arrays
ELEMENTS = {
    "grad_norm.cu": r"\bpart\[",
    "linear_logprobs.cu": r"\bpart\[",
    "gated_rows_kernel.cuh": r"\bpart\[",
    "gated_tokens_kernel.cuh": r"\bst\.up\[|\bst\.out\[which\]\[",
    "embedding.cu": r"\bkeys\[|\bless\[|\bsame\[|\bs\.counts\[|\bs\.start\[|\bs\.sums\[",
}
CHECKED = r"\b(?:smem_load<\w+>|smem_store|smem_get|smem_put|smem_within|smem_u32|sizeof|tma_store_2d)\("


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def without_calls(text, opening):
    """The text without the calls that match, whatever they nest."""
    out, at = [], 0
    for m in re.finditer(opening, text):
        if m.start() < at:
            continue
        out.append(text[at: m.start()])
        depth, at = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
    return "".join(out) + text[at:]


@pytest.mark.parametrize("name", ELEMENTS)
def test_elements_of_shared_arrays_are_reached_through_the_checked_helpers(name):
    text = re.sub(r"__shared__[^;]*;|\nstruct \w+ \{.*?\n\};", "", source(name), flags=re.S)      # declarations
    assert re.search(ELEMENTS[name].replace(r"\[", ""), text), "the arrays have other names"
    text = without_calls(text, CHECKED)
    raw = [" ".join(text[max(0, m.start() - 40): m.end() + 30].split()) for m in re.finditer(ELEMENTS[name], text)]
    assert not raw, raw


@pytest.mark.parametrize("unit", ["dense", "gated_linear", "linear_logprobs", "embedding", "grad_norm"])
def test_every_units_status_is_read(unit):
    check = re.search(r"int mxfp4_check\(.*?\n\}", source("libmxfp4.cu"), flags=re.S).group(0)
    assert f"{unit}_take_status(" in check
    assert any(f"int {unit}_take_status(" in source(f) for f in os.listdir(build.CSRC) if f.endswith(".cu"))


@pytest.mark.parametrize("name,kernels", [("dense_gemm_kernel.cuh", 1), ("gated_tokens_kernel.cuh", 1), ("embedding.cu", 1)])
def test_units_with_waits_are_read_in_every_build(name, kernels):
    """Their words can be set in the ordinary build too: the check must not depend on the bounds-checking one."""
    assert source(name).count("mbar_wait(") >= kernels
    check = re.search(r"int mxfp4_check\(.*?\n\}", source("libmxfp4.cu"), flags=re.S).group(0)
    always = check[: check.index("mxfp4_bounds_checked()")]
    for unit in ("dense", "gated_linear", "embedding"):
        assert f"{unit}_take_status(" in always
