"""The example with whole prompts: attention, weights and scores of the prompts before the first pass."""
import math
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_passes_after_whole_prompts(dtype):
    """What is stored is the same, so positions and slots are; the error's bound is that of the four bits (see
    test_gpu_verify_passes.py)."""
    import verify_passes
    common = dict(requests=3, passes=10, budget=4096, dtype=dtype, prompt=60, log=lambda s: None)
    old, got = verify_passes.run(**common), verify_passes.run(**common, whole_prompts=True)
    assert got["positions"] == old["positions"] and got["slots"] == old["slots"]
    assert got["worst_error"] == old["worst_error"] < 0.4
    s = got["scores"]
    assert old["scores"]["tokens"] == 0 and s["tokens"] > 3 * 59
    assert s["logp"] < 0 < s["entropy"] < s["tokens"] * math.log(2048)


def test_whole_prompts_over_a_bounded_cache():
    import verify_passes
    got = verify_passes.run(requests=2, passes=12, budget=64, prompt=100, log=lambda s: None, whole_prompts=True)
    assert got["slots"] == [64, 64] and min(got["positions"]) >= 112         # a pass commits one token at least


def test_the_command():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "verify_passes.py"), "--passes", "3", "--whole-prompts"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "tokens scored" in r.stdout, r.stdout + r.stderr
