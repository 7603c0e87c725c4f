"""Attention over prompts at the ends of the types: results, sums and scores that are large."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, attend, check_attend, seen

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


@pytest.mark.parametrize("many", [FEW, MANY])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("dtype,size,scale", [(F16, 3e4, 1.0), (F16, 3e4, 0.7), (F16, 5e4, 3.3), (BF16, 1.3e6, 0.123), (BF16, 1e18, 0.9),
                                              (BF16, 7e18, 1.1), (F16, 4e3, 0.9)])
def test_scores_of_any_size(many, sign, dtype, size, scale):
    """Scores beside whose size a softmax's differences vanish: equal ones share, larger ones take all.  Each is one
    product, exact in fp32."""
    s, q, k, v, how = prompts(700, many, 64, dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    v[:] = torch.randn(v.shape, generator=g, device="cuda")
    q[..., 9], k[..., 9] = size, sign * size
    for i in range(len(s.counts)):
        k[s.at(i)][300:310, :, 9] = size * 1.125 * sign
        k[s.at(i)][400:, :, 9] = size * 0.5 * sign
        k[s.at(i)][500:505, :, 9] = size * 1.25 * sign
    q, k, v = (x.to(dtype) for x in (q, k, v))
    out, lse = B.prompt_attend(q, k, v, scale=scale, **how)
    half = torch.finfo(dtype).eps / 2
    for i in {0, len(s.counts) - 1}:
        x, y, z = (t[s.at(i)].double() for t in (q, k, v))
        scores = (torch.einsum("nhd,chd->hnc", x, y) * scale).masked_fill(~seen(700, 700), -math.inf)
        p, rl = scores.softmax(-1), scores.logsumexp(-1).T  # (exp(x - lse) would miss what 64 bits have no room for in lse)
        ref, mass = torch.einsum("hnc,chd->nhd", p, z), torch.einsum("hnc,chd->nhd", p, z.abs())
        # equal scores have equal probabilities, whatever they are rounded to: half a step of the result, and of fp32
        assert bool(((out[s.at(i)].double() - ref).abs() <= half * ref.abs() + (half + 2.0 ** -20) * mass).all())
        assert bool(((lse[s.at(i)].double() - rl).abs() <= 2.0 ** -21 * rl.abs() + 2.0 ** -20).all())


@pytest.mark.parametrize("many", [FEW, MANY])
def test_scores_that_fp32_does_not_hold(many):
    """scale q.k beyond 3e38, q.k itself not: the largest takes all, and the logarithm is infinite."""
    s, q, k, v, how = prompts(300, many, 64, BF16)
    g = torch.Generator(device="cuda").manual_seed(2)
    v[:] = torch.randn(v.shape, generator=g, device="cuda")
    q[..., 9], k[..., 9] = 1e15, 1e15
    for i in range(len(s.counts)):
        k[s.at(i)][40, :, 9] = 2e15
        k[s.at(i)][200, :, 9] = 4e15
    q, k, v = (x.to(BF16) for x in (q, k, v))
    out, lse = B.prompt_attend(q, k, v, scale=1e12, **how)
    for i in {0, len(s.counts) - 1}:
        x, y = out[s.at(i)], v[s.at(i)]
        assert torch.equal(x[40:200], y[40:41].expand(160, -1, -1)) and torch.equal(x[200:], y[200:201].expand(100, -1, -1))
    assert bool((lse == math.inf).all())
    k.neg_()
    out, lse = B.prompt_attend(q, k, v, scale=1e12, **how)
    for i in {0, len(s.counts) - 1}:                       # all but two are equal
        x, y = out[s.at(i)], v[s.at(i)].double()
        want = (y[:300].sum(0) - y[40] - y[200]) / 298
        assert bool(((x[299].double() - want).abs() <= 2.0 ** -8 * (want.abs() + y.abs().mean(0)) * 1.01).all())
    assert bool((lse == -math.inf).all())                  # (its value is below fp32's lowest)


def test_a_scale_of_zero_over_large_scores():
    s, q, k, v, how = prompts(300, FEW, 64, BF16)
    g = torch.Generator(device="cuda").manual_seed(2)
    v[:] = torch.randn(v.shape, generator=g, device="cuda")
    q[..., 0] = 1e18
    k[..., 0] = torch.linspace(-1e19, 1e19, 300, device="cuda")[:, None]
    for scale in (0.0, 1e-40):
        check(q, k, v, s, how, BF16, scale)


@pytest.mark.parametrize("where", ["padding", "inside", "everywhere"])
def test_values_that_are_not_finite_take_no_time(where):
    """8,192 keys with NaN behind a sequence's last row, at one key inside, at all of them: rows that do not see them are
    right, and no wait of five milliseconds runs out (the whole call takes less than one)."""
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda h: torch.randn(2, 8256, h, 64, generator=g, device="cuda").bfloat16()
    q, k, v = new(8), new(2), new(2)
    n = torch.tensor([8191, 8000], dtype=torch.int32, device="cuda")
    bad = {"padding": slice(8256, None), "inside": slice(8100, 8101), "everywhere": slice(0, None)}[where]
    want, wl = B.prompt_attend(q, k, v, n_new=n)
    dirty = v.clone()
    for i in range(2):
        dirty[i, int(n[i]):] = math.nan
        dirty[i, bad] = math.nan
    try:
        B.prompt_set_wait_limit(5_000_000)
        out, lse = B.prompt_attend(q, k, dirty, n_new=n)
        assert B.prompt_status() == B.OK
    finally:
        B.prompt_set_wait_limit(0)
    assert torch.equal(lse, wl)
    for i in range(2):
        clean = min(int(n[i]), bad.start)
        assert torch.equal(out[i, :clean], want[i, :clean]) and bool(torch.isnan(out[i, clean:int(n[i])]).all())
        assert bool((out[i, int(n[i]):] == 0).all())
