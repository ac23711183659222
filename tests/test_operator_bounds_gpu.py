"""The small suites of the 128-block products, the residual norm and the log probabilities under the bounds-checking build:
any shared-memory address outside its buffer would be recorded in the status word and fail their `api.check()`."""
import os
import subprocess
import sys

import pytest

from paper_2605_09825_b200 import build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys
sys.path.insert(0, sys.argv[1])
from paper_2605_09825_b200 import api
assert api.bounds_checked(), "the child did not load the bounds-checking build"
import pytest
sys.exit(pytest.main(["-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_block128_gpu.py",
                      "tests/test_residual_norm_gpu.py", "tests/test_logprobs_gpu.py", "tests/test_block_step_gpu.py"]))
"""


def test_suites_pass_under_the_bounds_checking_build():
    lib = build.build_library(bounds=True)
    env = dict(os.environ, MXFP4_LIBRARY=lib)
    res = subprocess.run([sys.executable, "-c", CHILD, ROOT], cwd=ROOT, env=env, capture_output=True, text=True,
                         timeout=1800)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-3000:]
    assert " passed" in res.stdout and "failed" not in res.stdout
