"""The weight of a prompt's keys where rows that do not see a key hold what is not a number."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, check_weigh, weigh

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(s, hq, hkv, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return (new(*s.shape, hq, d) * 2).to(dtype), new(*s.shape, hkv, d).to(dtype)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("hq,hkv,d,dtype,n,row", [(4, 2, 64, BF16, 300, 100), (2, 2, 128, F16, 700, 300), (16, 2, 64, F16, 200, 3),
                                                   (6, 2, 128, BF16, 513, 512), (8, 8, 64, BF16, 1500, 777)])
def test_a_row_of_nan_reaches_the_keys_it_sees(packed, hq, hkv, d, dtype, n, row):
    """The calls in sequence: the row's logarithm is NaN too."""
    s = Side([n, 40], packed)
    q, k = make(s, hq, hkv, d, dtype)
    how = s.arguments(("first", "n_new"))
    q[s.at(0)][row, 0] = math.nan
    lse = B.prompt_attend(q, k, k, **how)[1]
    assert torch.isnan(lse[s.at(0)][row, 0])
    w = B.prompt_weigh(q, lse, k, **how)
    got = w[:, s.at(0)[0]] if packed else w[0][:, :n]
    assert bool(torch.isnan(got[0, :row + 1]).all())
    clean = q[s.at(0)].clone()
    clean[row, 0] = 0.0
    rl = lse[s.at(0)].clone()
    rl[row, 0] = -math.inf                                 # the row counts for nothing
    ref = weigh(clean, rl, k[s.at(0)], torch.ones(n, device="cuda"), d ** -0.5)
    check_weigh(got[0, row + 1:], [x[0, row + 1:] for x in ref], n * hq, d)
    check_weigh(got[1:], [x[1:] for x in ref], n * hq, d)
    ref = weigh(q[s.at(1)], lse[s.at(1)], k[s.at(1)], torch.ones(40, device="cuda"), d ** -0.5)
    check_weigh(w[:, s.at(1)[0]] if packed else w[1][:, :40], ref, 40 * hq, d)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("hq,hkv,n,row", [(4, 2, 300, 100), (8, 1, 700, 650), (1, 1, 200, 0)])
def test_a_weight_that_is_no_number_reaches_the_keys_its_row_sees(bad, hq, hkv, n, row):
    s = Side([n], True)
    q, k = make(s, hq, hkv, 64, BF16)
    how = s.arguments(("first", "n_new"))
    lse = B.prompt_attend(q, k, k, **how)[1]
    rw = torch.rand(n, device="cuda") + 0.5
    rw[row] = bad
    w = B.prompt_weigh(q, lse, k, row_weight=rw, **how)
    seen = w[:, :row + 1]
    assert bool(torch.isnan(seen).all() if math.isnan(bad) else (seen == bad).all())
    rw[row] = 0.0
    ref = weigh(q, lse, k, rw, 0.125)
    check_weigh(w[:, row + 1:], [x[:, row + 1:] for x in ref], n * hq, 64)


@pytest.mark.parametrize("row", [0, 100, 299])
def test_a_logarithm_of_infinity_counts_for_nothing(row):
    s = Side([300], True)
    q, k = make(s, 4, 2, 64, F16)
    how = s.arguments(("first", "n_new"))
    lse = B.prompt_attend(q, k, k, **how)[1]
    lse[row] = math.inf
    w = B.prompt_weigh(q, lse, k, **how)
    rw = torch.ones(300, device="cuda")
    rw[row] = 0.0
    lse[row] = 0.0
    check_weigh(w, weigh(q, lse, k, rw, 0.125), 1200, 64)
