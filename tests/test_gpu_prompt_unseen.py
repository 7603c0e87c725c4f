"""Attention over prompts where infinities and NaN lie among the values, at sizes that take every block
through several items (no clusters share them)."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, attend, check_attend, seen

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(s, hq, hkv, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return ((new(*s.shape, hq, d) * 2).to(dtype), new(*s.shape, hkv, d).to(dtype), new(*s.shape, hkv, d).to(dtype))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 16, 128, BF16), (16, 16, 64, F16), (32, 8, 64, BF16), (24, 8, 128, F16)])
def test_values_that_are_not_finite_in_whole_items(bad, packed, hq, hkv, d, dtype):
    """More items than twice the SMs: of sequence i, key j and what lies behind every sequence's last row."""
    s = Side([700, 300, 690, 513, 450, 64] * 2, packed, tail=5)
    q, k, v = make(s, hq, hkv, d, dtype)
    refs = {n: attend(q[s.at(n)], k[s.at(n)], v[s.at(n)], d ** -0.5) for n in (0, 1, 3, 9)}
    how = s.arguments(("first", "n_new"))
    for i, j in ((0, 5), (0, 699), (1, 250), (9, 511)):
        k2, v2 = k.clone(), v.clone()
        for x in (k2, v2):
            x[s.at(i)][j, :, 3] = bad
            if packed:
                x[s.rows - 5:] = bad
            else:
                for n, rows in enumerate(s.counts):
                    x[n, rows:] = bad
        out, lse = B.prompt_attend(q, k2, v2, **how)
        assert B.prompt_status() == B.OK
        for n, ref in refs.items():
            a, clean = s.at(n), slice(0, j if n == i else None)
            check_attend(out[a][clean], lse[a][clean], [x[clean] for x in ref], dtype, d)
            if n == i:
                assert not torch.isfinite(out[a][j:]).all(-1).any(), "what a row sees is not hidden"


@pytest.mark.parametrize("packed", [True, False])
def test_infinite_values_reach_the_rows_that_see_them(packed):
    """A channel with an infinity is infinite from that key on, one with both signs NaN; the others stay."""
    s = Side([600, 300, 500] * 4, packed)
    q, k, v = make(s, 16, 16, 64, BF16)
    how = s.arguments(("first", "n_new"))
    want, wl = B.prompt_attend(q, k, v, **how)
    v2 = v.clone()
    x = v2[s.at(4)]
    x[50, 3, 7], x[60, 3, 7], x[70, 3, 9], x[70, 4, 9] = math.inf, math.inf, -math.inf, math.nan
    x[75, 3, 9], x[299, 5, 63] = math.inf, -math.inf
    out, lse = B.prompt_attend(q, k, v2, **how)
    expect = want.clone()
    y = expect[s.at(4)]
    y[50:, 3, 7], y[70:75, 3, 9], y[75:, 3, 9], y[70:, 4, 9], y[299, 5, 63] = math.inf, -math.inf, math.nan, math.nan, -math.inf
    assert torch.equal(out.nan_to_num(2.0 ** 100), expect.nan_to_num(2.0 ** 100)) and torch.equal(lse, wl)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(48, 16, 64, BF16), (16, 16, 128, F16), (64, 8, 64, F16)])
@pytest.mark.parametrize("extra", [0, 2, 150])
def test_every_item_holds_values_that_are_not_finite(hq, hkv, d, dtype, extra):
    """One to three in every sequence and key head, so that items are done again one behind the other, long and short
    ones, some without rows in a group or (more rows than keys) with rows that see nothing: the rows that see such a value
    are infinite or NaN in its channel, the others right."""
    counts = [420, 1180, 108, 209, 1383, 64, 300, 900, 37, 128, 257]
    qs, ks = Side(counts, False), Side([max(1, n - extra) for n in counts], True, tail=3)
    g = torch.Generator(device="cuda").manual_seed(7)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k, v = new(*qs.shape, hq, d).to(dtype), new(*ks.shape, hkv, d).to(dtype), new(*ks.shape, hkv, d).to(dtype)
    clean, kind = v.clone(), torch.zeros(v.shape, device="cuda")
    at = torch.Generator().manual_seed(8)
    pick = lambda n: int(torch.randint(0, n, (1,), generator=at))
    for i, c in enumerate(ks.counts):
        for h in range(hkv):
            for _ in range(1 + pick(3)):
                j, ch, what = pick(c), pick(d), pick(3)
                v[ks.at(i)][j, h, ch], kind[ks.at(i)][j, h, ch] = (math.inf, -math.inf, math.nan)[what], 1 + what
                clean[ks.at(i)][j, h, ch] = 0.0
    out, lse = B.prompt_attend(q, k, v, **qs.arguments(("first", "n_new")), **ks.arguments(("first_k", "n_k")))
    assert B.prompt_status() == B.OK
    for i in range(len(counts)):
        a, b = qs.at(i), ks.at(i)
        see = seen(qs.counts[i], ks.counts[i]).double()
        which = kind[b].repeat_interleave(hq // hkv, 1)
        plus, minus, none = (torch.einsum("nc,chd->nhd", see, (which == x).double()) > 0 for x in (1, 2, 3))
        none = none | (plus & minus)
        odd = plus | minus | none
        want = torch.where(none, math.nan, torch.where(plus, math.inf, -math.inf))
        assert torch.equal(out[a].double().nan_to_num(2.0 ** 200)[odd], want.double().nan_to_num(2.0 ** 200)[odd])
        ref = attend(q[a], k[b], clean[b], d ** -0.5)
        calm = lambda x: torch.where(odd, torch.zeros_like(x), x)
        check_attend(calm(out[a]), lse[a], [calm(ref[0]), *ref[1:]], dtype, d)
