"""The attention weight that a prompt's keys receive against 64 bits."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, check_weigh, weigh

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(qs, ks, hq, hkv, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k = (new(*qs.shape, hq, d) * 2).to(dtype), new(*ks.shape, hkv, d).to(dtype)
    lse = B.prompt_attend(q, k, k, **arguments(qs, ks))[1]
    return q, lse, k


def arguments(qs, ks):
    return {**qs.arguments(("first", "n_new")), **ks.arguments(("first_k", "n_k"))}


def check(q, lse, k, qs, ks, row_weight=None, scale=None, **more):
    w = B.prompt_weigh(q, lse, k, row_weight=row_weight, scale=scale, **arguments(qs, ks), **more)
    assert B.prompt_status() == B.OK
    hq, d = q.shape[-2:]
    rw = torch.ones(qs.shape, device="cuda") if row_weight is None else row_weight
    for i in range(len(qs.counts)):
        a, b = qs.at(i), ks.at(i)
        got = w[:, b[0]] if ks.packed else w[i][:, b[1]]
        ref = weigh(q[a], lse[a], k[b], rw[a], d ** -0.5 if scale is None else scale)
        check_weigh(got, ref, qs.counts[i] * hq, d)
        if not ks.packed:
            assert bool((w[i][:, ks.counts[i]:] == 0).all())
    return w


LENGTHS = {"one": [1], "few": [3, 0, 37, 1], "tile edges": [127, 128, 129], "item edges": [255, 256, 257, 33, 31],
           "long": [1000, 0, 1537]}


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (6, 2), (16, 1)])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (128, F16), (64, F16)])
@pytest.mark.parametrize("packed", [True, False])
def test_prompts_over_themselves(lengths, hq, hkv, d, dtype, packed):
    s = Side(LENGTHS[lengths], packed)
    check(*make(s, s, hq, hkv, d, dtype), s, s)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F16)])
def test_pieces_of_prompts(packed, d, dtype):
    qs, ks = Side([1, 5, 200, 64, 0, 7, 300], packed), Side([900, 5, 333, 20, 50, 0, 2], packed)
    check(*make(qs, ks, 8, 2, d, dtype), qs, ks)


def test_packed_rows_over_padded_keys():
    for p in (True, False):
        qs, ks = Side([4, 1, 9], p), Side([40, 300, 9], not p)
        check(*make(qs, ks, 8, 2, 128, BF16), qs, ks)


@pytest.mark.parametrize("hq,hkv", [(64, 1), (7, 7), (12, 1), (10, 2), (1, 1)])
def test_groups(hq, hkv):
    s = Side([70, 300], True)
    check(*make(s, s, hq, hkv, 64, BF16), s, s)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30])
def test_scales(scale):
    s = Side([5, 150], True)
    q, lse, k = make(s, s, 4, 2, 64, F16)
    check(q, lse.abs() + 3, k, s, s, scale=scale)


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("kind", ["window", "first", "none", "some", "signed"])
def test_row_weights(packed, kind):
    s = Side([700, 3, 0, 513, 2000], packed, tail=3)
    q, lse, k = make(s, s, 8, 2, 64, BF16)
    g = torch.Generator(device="cuda").manual_seed(9)
    rw = torch.zeros(s.shape, device="cuda")
    for i, n in enumerate(s.counts):
        x = rw[s.at(i)]
        if kind == "window":
            x[max(0, n - 16):] = 1.0
        elif kind == "first":
            x[:2] = 0.5
        elif kind == "some":
            x.copy_((torch.rand(n, generator=g, device="cuda") < 0.02) * torch.rand(n, generator=g, device="cuda"))
        elif kind == "signed":
            x.copy_(torch.randn(n, generator=g, device="cuda"))
    w = check(q, lse, k, s, s, rw)
    if kind == "none":
        assert bool((w[:, :sum(s.counts)] if packed else w).eq(0).all())
    # what does not count may hold anything
    dead = (rw == 0)
    q[dead], lse[dead] = math.nan, math.nan
    if packed:
        q[s.rows - 3:], k[s.rows - 3:] = math.inf, math.nan
    again = B.prompt_weigh(q, lse, k, row_weight=rw, **arguments(s, s))
    for i in range(5):
        b = s.at(i)
        assert torch.equal(w[:, b[0]], again[:, b[0]]) if packed else torch.equal(w[i], again[i])


def test_weights_add_up():
    """A softmax adds up to one: each row's weight comes out again, whole."""
    s = Side([900, 77, 1200], True)
    q, lse, k = make(s, s, 16, 8, 128, BF16)
    w = B.prompt_weigh(q, lse, k, **arguments(s, s))
    for i, n in enumerate(s.counts):
        # (a row's sum is off by what exp is off where the score is: 128 products of 2^-24 of 100 at most)
        assert abs(w[:, s.at(i)[0]].double().sum().item() / (16 * n) - 1) < 128 * 2.0 ** -24 * 100


def test_long_sums_lose_nothing():
    """65,536 rows' equal weights on one key: an fp32 sum alone would drift."""
    n = 65536
    q, k = torch.zeros(n, 8, 64, dtype=F16, device="cuda"), torch.zeros(1, 1, 64, dtype=F16, device="cuda")
    first, first_k = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (n, 1))
    # only the last row sees the one key; with as many keys, the first is seen by all
    lse = torch.full((n, 8), 1.7, device="cuda")
    w = B.prompt_weigh(q, lse, k, first=first, first_k=first_k)
    one = math.exp(-torch.tensor(1.7).item())
    assert abs(w.item() / (8 * one) - 1) < 2.0 ** -20
    w = B.prompt_weigh(q, lse, k.expand(n, -1, -1).contiguous(), first=first)
    want = 8 * one * torch.arange(n, 0, -1, device="cuda", dtype=torch.float64)
    # exp is off by 2^-21 (its argument by half a step of 2.45, its result by two steps), the same for all
    assert ((w[0].double() / want - 1).abs().max().item()) < 2.0 ** -20


def test_strides():
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)
    s = Side([100, 170, 31], True)
    both = new(*s.shape, 10, 128)
    q, k = both[:, :8], both[:, 8:]
    lse = B.prompt_attend(q, k, k, **arguments(s, s))[1]
    a = check(q, lse, k, s, s)
    wide = torch.zeros(8, s.rows + 3, device="cuda").T[:s.rows]
    wide.copy_(lse)
    b = check(q.transpose(0, 1).contiguous().transpose(0, 1), wide, k, s, s)
    assert torch.equal(a, b)


def test_rows_of_no_sequence_stay():
    s = Side([50, 90], True, lead=7, tail=30)
    w = torch.full((2, s.rows), 5.0, device="cuda")
    check(*make(s, s, 4, 2, 64, BF16), s, s, weight=w)
    assert bool((w[:, :7] == 5.0).all()) and bool((w[:, 147:] == 5.0).all())


def test_rows_that_saw_nothing():
    """lse of -inf: more rows than keys."""
    qs, ks = Side([300], True), Side([40], True)
    check(*make(qs, ks, 8, 2, 128, F16), qs, ks)


def test_nothing_at_all():
    q = torch.zeros(0, 4, 64, dtype=BF16, device="cuda")
    first = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert B.prompt_weigh(q, q[..., 0].float(), q[:, :2], first=first).shape == (2, 0)
    k = torch.randn(5, 2, 64, device="cuda").to(BF16)
    w = B.prompt_weigh(q, q[..., 0].float(), k, first=first[:2], first_k=torch.tensor([0, 5], dtype=torch.int32, device="cuda"))
    assert bool((w == 0).all())


def test_streams_and_graphs():
    s = Side([300, 41], True)
    q, lse, k = make(s, s, 8, 2, 128, BF16)
    how = arguments(s, s)
    ref = B.prompt_weigh(q, lse, k, **how)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w = torch.empty_like(ref)
    B.prompt_weigh(q, lse, k, weight=w, stream=side, **how)
    side.synchronize()
    assert torch.equal(w, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.prompt_weigh(q, lse, k, weight=w, **how)
    for x, y in zip((q, lse, k), make(s, s, 8, 2, 128, BF16, 1)):
        x.copy_(y)
    graph.replay()
    assert torch.equal(w, B.prompt_weigh(q, lse, k, **how))
