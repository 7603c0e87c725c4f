"""Attention over prompts at the ends of the types: results, sums and scores that are large."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, attend, check_attend

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
# (sequences, key heads): with few items clusters share them, with many they do not
FEW, MANY = (1, 1), (24, 8)


def prompts(n, many, d, dtype):
    """q, k, v of zeros, all sequences n long, and the calls' arguments."""
    s = Side([n] * many[0], True)
    new = lambda: torch.zeros(s.rows, many[1], d, device="cuda")
    return s, new(), new(), new(), s.arguments(("first", "n_new"))


def check(q, k, v, s, how, dtype, scale, rows=None):
    q, k, v = (x.to(dtype) for x in (q, k, v))
    out, lse = B.prompt_attend(q, k, v, scale=scale, **how)
    assert B.prompt_status() == B.OK
    for i in {0, len(s.counts) - 1}:
        a = s.at(i)
        ref = attend(q[a], k[a], v[a], scale)
        assert bool(torch.isfinite(out[a]).all())
        check_attend(out[a], lse[a], ref, dtype, q.shape[-1])
    return out, lse


@pytest.mark.parametrize("many", [FEW, MANY])
@pytest.mark.parametrize("keys", ["equal", "rising"])
def test_sums_of_large_values(many, keys):
    """bf16 values up to 3e38: 2,000 equal keys, whose values' sum fp32 does not hold; keys that rise by less than
    2^8 in all, where the running maximum stays behind."""
    s, q, k, v, how = prompts(2000, many, 64, BF16)
    q[..., 0] = 1.0
    g = torch.Generator(device="cuda").manual_seed(1)
    v[:] = torch.rand(v.shape, generator=g, device="cuda") * 3.3e38
    v[..., 5] = -3.3e38
    v[..., 6] *= 1e-10
    if keys == "rising":
        for i in range(len(s.counts)):
            k[s.at(i)][..., 0] = torch.linspace(0, 7.9 * math.log(2), 2000, device="cuda")[:, None]
    check(q, k, v, s, how, BF16, 1.0)


@pytest.mark.parametrize("size", [1e-30, 2.0 ** -120])
def test_sums_of_small_values(size):
    """The other end: what bf16 holds with all its bits comes out so, off by a few of fp32's smallest steps times the
    2^-21 that a sum over 2,000 keys is taken down by."""
    s, q, k, v, how = prompts(2000, FEW, 64, BF16)
    g = torch.Generator(device="cuda").manual_seed(1)
    v[:] = (torch.rand(v.shape, generator=g, device="cuda") + 0.5) * size
    v = v.bfloat16()
    out, _ = B.prompt_attend(q.bfloat16(), k.bfloat16(), v, scale=1.0, **how)
    want = v.double().cumsum(0) / torch.arange(1, 2001, device="cuda")[:, None, None]
    assert bool(((out.double() - want).abs() <= 2.0 ** -7 * want + 2.0 ** -126).all())


@pytest.mark.parametrize("many", [FEW, MANY])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_results_next_to_the_types_largest_number(many, d, dtype):
    """Rounded probabilities over a sum that is not: all of them may be rounded up (one key at 0, the others
    where half a step is added), and the result lies above the values' size.  It ends at the type's largest number."""
    s, q, k, v, how = prompts(1000, many, d, dtype)
    half = 0.5 + 0.6 * torch.finfo(dtype).eps / 2          # (rounded to the next number up)
    first = torch.tensor(math.log(half)).to(dtype).float()
    q[..., :2] = 1.0
    k[..., 0], k[..., 1] = first, (math.log(half) - first).to(dtype).float()
    v[:] = torch.finfo(dtype).max
    v[..., 1::2] *= -1
    for i in range(len(s.counts)):
        k[s.at(i)][0] = 0.0
    out, _ = check(q, k, v, s, how, dtype, 1.0)
    for i in (0, len(s.counts) - 1):                       # what a row sees is not hidden
        v[s.at(i)][900, 0, 3] = math.inf
    out, _ = B.prompt_attend(*(x.to(dtype) for x in (q, k, v)), scale=1.0, **how)
    for i in (0, len(s.counts) - 1):
        x = out[s.at(i)]
        assert bool((x[900:, 0, 3] == math.inf).all()) and bool(torch.isfinite(x[:900]).all()) and bool(torch.isfinite(x[..., 4:]).all())
