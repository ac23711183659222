"""Which status words mxfp4_check looks at goes by which parts of the library have launched a kernel: every launch of a
part has to note it, and every note has to be the part's own.  Read from the sources; no GPU needed."""
import os
import re

import pytest

from paper_2605_09825_b200 import api, build

UNITS = sorted(f for f in os.listdir(build.CSRC) if f.endswith(".cu"))
# the part that is looked at in any case, and whose self-tests and probe are launched without attributes
ALWAYS = "libmxfp4.cu"


def source(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def function(text, name):
    """A function's definition, from its name to the brace that ends it."""
    m = re.search(rf"^[^\n;]*\b{name}\([^;{{]*\{{.*?^\}}", text, flags=re.S | re.M)
    return m.group(0)


@pytest.mark.parametrize("unit", UNITS)
def test_kernels_are_launched_through_the_helper_that_notes_it(unit):
    if unit != ALWAYS:
        assert "<<<" not in source(unit) and "cudaLaunchKernel" not in source(unit)
    for header in build._depends(os.path.join(build.CSRC, unit)):
        if header.endswith((".cuh", ".h")) and os.path.basename(header) not in ("tma_host.cuh", "host_common.cuh"):
            assert "<<<" not in source(header) and "cudaLaunchKernel" not in source(header), header


def test_the_helper_notes_the_launch_in_its_own_unit():
    text = source("tma_host.cuh")
    assert "unit_used(" in function(text, "launch_kernel_pdl_cluster")
    # of internal linkage: one instantiation shared by two units would note one unit's launches for the other
    for name in ("launch_kernel_pdl_cluster", "launch_kernel_pdl"):
        assert re.search(rf"static inline cudaError_t {name}\(", text), name
    assert text.count("cudaLaunchKernelEx(") == 1


def test_unknown_parts_are_refused():
    build.build_library()
    lib = api.load_library()
    assert lib.mxfp4_selftest_unit_timeout(-1, None) == lib.mxfp4_selftest_unit_timeout(9, None) == -4
