"""What the bounds-checking build promises about the operators around the linears, read from their sources: elements of
shared arrays are reached through the checked helpers, and every unit's status word is looked at.  No GPU needed."""
import os
import re

import pytest

from paper_2605_09825_b200 import build

# how each file writes an element of one of its shared arrays
ELEMENTS = {
    "logprobs.cu": r"\bsc\.\w+\[|\bscratch\.\w+\[|\bnotes(?:\[buf\])?\.\w+\[|\bred\[|\bkeys\[",
    "residual_norm.cu": r"\bsh\.red\[|\bpart\[",
    "block128_quantize_kernel.cuh": r"\bcodes_t\[|\bpart\[|\binverse\[",
    "block128_rows_kernel.cuh": r"\bpart\[",
}
# the helpers, and the address of an asynchronous copy that is checked before it
CHECKED = r"\b(?:smem_load<\w+>|smem_store|smem_get|smem_put|smem_within|smem_u32|sizeof)\("


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


def test_every_unit_with_checked_accesses_has_its_status_read():
    check = re.search(r"int mxfp4_check\(.*?\n\}", source("libmxfp4.cu"), flags=re.S).group(0)
    for unit in ("block128", "residual_norm", "logprobs"):
        assert f"{unit}_take_status(" in check
        assert f"int {unit}_take_status(" in source(f"{unit}.cu")
