"""The example that runs drafting, tree verification and the 4-bit cache together."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_passes_over_a_cache_that_is_never_cut(dtype):
    """What is left of the error is that of 4 bits.  A value of a group of 64 is off by at most half
    a step, a 30th of the group's range (about 5 of its standard deviations), so by 5 / 30 / sqrt(3) =
    0.1 of one at most in the mean square; keys shift a score of unit spread by as much, and with
    it the result's weights: 0.2 together, doubled for the worst of many positions."""
    import verify_passes
    got = verify_passes.run(requests=3, passes=12, budget=4096, dtype=dtype, prompt=60, log=lambda s: None)
    assert got["slots"] == got["positions"]
    assert got["worst_error"] < 0.4
    assert got["tokens_per_pass"] > 1      # more than the anchors: drafts were accepted


def test_passes_over_a_bounded_cache():
    """Sequences stay at the budget while positions go on; the checks inside are the test."""
    import verify_passes
    got = verify_passes.run(requests=2, passes=15, budget=64, prompt=100, log=lambda s: None)
    assert got["slots"] == [64, 64] and min(got["positions"]) > 115


def test_the_example_runs_as_a_command():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "verify_passes.py"), "--passes", "5", "--dtype", "f16"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "tokens a pass" in r.stdout, r.stdout + r.stderr
