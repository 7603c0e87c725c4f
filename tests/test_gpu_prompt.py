"""Attention over whole prompts against 64 bits."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, attend, check_attend

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(qs, ks, hq, hkv, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return ((new(*qs.shape, hq, d) * 2).to(dtype), new(*ks.shape, hkv, d).to(dtype), new(*ks.shape, hkv, d).to(dtype))


def run(q, k, v, qs, ks, scale=None, **more):
    return B.prompt_attend(q, k, v, scale=scale, **qs.arguments(("first", "n_new")), **ks.arguments(("first_k", "n_k")), **more)


def check(q, k, v, qs, ks, scale=None, **more):
    out, lse = run(q, k, v, qs, ks, scale, **more)
    assert B.prompt_status() == B.OK
    d = q.shape[-1]
    for i in range(len(qs.counts)):
        a, b = qs.at(i), ks.at(i)
        check_attend(out[a], lse[a], attend(q[a], k[b], v[b], d ** -0.5 if scale is None else scale), q.dtype, d)
        if not qs.packed:
            assert bool((out[i, qs.counts[i]:] == 0).all()) and bool((lse[i, qs.counts[i]:] == -math.inf).all())
    return out, lse


LENGTHS = {"one": [1], "few": [3, 0, 37, 1], "tile edges": [127, 128, 129], "item edges": [63, 64, 65, 255, 256, 257],
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
    """Fewer query rows than keys; more; no keys at all; no rows."""
    qs, ks = Side([1, 5, 200, 64, 0, 7, 300], packed), Side([900, 5, 333, 20, 50, 0, 2], packed)
    check(*make(qs, ks, 8, 2, d, dtype), qs, ks)


def test_packed_rows_over_padded_keys():
    qs, ks = Side([4, 1, 9], True), Side([40, 300, 9], False)
    check(*make(qs, ks, 8, 2, 128, BF16), qs, ks)
    qs, ks = Side([4, 1, 9], False), Side([40, 300, 9], True)
    check(*make(qs, ks, 8, 2, 128, BF16), qs, ks)


@pytest.mark.parametrize("hq,hkv", [(64, 1), (7, 7), (12, 1), (10, 2), (1, 1)])
def test_groups(hq, hkv):
    s = Side([70, 300], True)
    check(*make(s, s, hq, hkv, 64, BF16), s, s)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0, 1e-30, 3.0])
def test_scales(scale):
    s = Side([5, 150], True)
    check(*make(s, s, 4, 2, 64, F16), s, s, scale)


def test_many_sequences():
    g = torch.Generator().manual_seed(3)
    s = Side(torch.randint(0, 40, (1024,), generator=g).tolist(), True)
    q, k, v = make(s, s, 4, 2, 64, BF16)
    out, lse = run(q, k, v, s, s)
    for i in range(0, 1024, 41):
        a = s.at(i)
        check_attend(out[a], lse[a], attend(q[a], k[a], v[a], 0.125), BF16, 64)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_more_items_than_blocks(dtype):
    """Every block takes several items, of falling lengths."""
    s = Side([2000, 1, 1300, 700, 0, 2500], True)
    check(*make(s, s, 16, 8, 128, dtype), s, s)


def test_strides():
    """Slices of one projection; heads before rows; rows far apart; the same rows for all sequences."""
    g = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)
    s = Side([100, 170, 31], True)
    both = new(*s.shape, 12, 128)
    check(both[:, :8], both[:, 8:10], both[:, 10:], s, s)
    q, k, v = new(8, *s.shape, 128).transpose(0, 1), new(2, *s.shape, 128).transpose(0, 1), new(2, s.rows, 160)[..., 32:].transpose(0, 1)
    out = new(8, *s.shape, 128).transpose(0, 1)
    lse = torch.zeros(8, s.rows, device="cuda").T
    check(q, k, v, s, s, out=out, lse=lse)
    p = Side([90, 140], False)
    q, k = new(2, 8, 140, 128).transpose(1, 2), new(140, 2, 2, 64).transpose(0, 1)
    k = torch.cat((k, k), -1)
    check(q, k, new(140, 2, 128).expand(2, -1, -1, -1), p, p)


def test_rows_of_no_sequence_stay():
    s = Side([50, 90], True, lead=7, tail=30)
    q, k, v = make(s, s, 4, 2, 64, BF16)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 5.0, device="cuda")
    check(q, k, v, s, s, out=out, lse=lse)
    for x, was in ((out, 7.0), (lse, 5.0)):
        assert bool((x[:7] == was).all()) and bool((x[147:] == was).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("packed,dtype,d", [(True, BF16, 128), (False, F16, 64)])
def test_what_is_not_seen_may_hold_anything(bad, packed, dtype, d):
    """Keys and values behind a row's last one, of the next sequence, of padding: in tiles that the row's tile reads."""
    s = Side([100, 70, 200], packed, tail=5)
    q, k, v = make(s, s, 8, 2, d, dtype)
    refs = [attend(q[s.at(n)], k[s.at(n)], v[s.at(n)], d ** -0.5) for n in range(3)]
    for i, j in ((0, 60), (0, 99), (1, 69), (2, 130)):            # sequence i, key j
        k2, v2 = k.clone(), v.clone()
        for x in (k2, v2):
            x[s.at(i)][j, :, 3] = bad
        if packed:
            k2[370:], v2[370:] = bad, bad
        else:
            k2[0, 100:], v2[1, 70:] = bad, bad
        out, lse = run(q, k2, v2, s, s)
        for n in range(3):
            a, clean = s.at(n), slice(0, j if n == i else None)
            check_attend(out[a][clean], lse[a][clean], [x[clean] for x in refs[n]], dtype, d)
            if n == i:
                assert not torch.isfinite(out[a][j:]).all(-1).any(), "what a row sees is not hidden"


def test_masked_scores_of_infinity():
    """A key whose scores are all -inf counts for nothing; a row with nothing else is empty."""
    s = Side([3], True)
    q, k, v = make(s, s, 1, 1, 64, BF16)
    q.fill_(1.0)
    k[0] = -3e38
    out, lse = run(q, k, v, s, s, scale=1.0)
    assert lse[0, 0] == -math.inf and bool((out[0] == 0).all())
    ref = attend(q[1:], k[1:], v[1:], 1.0)
    check_attend(out[1:], lse[1:], ref, BF16, 64)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_many_keys_far_below_one(dtype):
    """2,000 keys 17 below one other (in exp's units) keep their part of the result, wherever the one lies."""
    s = Side([2048], True)
    d = 64
    q, k, v = torch.zeros(2048, 1, d, device="cuda"), torch.zeros(2048, 1, d, device="cuda"), torch.zeros(2048, 1, d, device="cuda")
    q[:, :, 0] = 1.0
    for top in (0, 100, 2000):
        k.zero_()
        k[top, :, 0] = 17.0
        v.fill_(1000.0)
        v[top] = 0.0
        check(q.to(dtype), k.to(dtype), v.to(dtype), s, s, 1.0)


def test_offsets_and_counts_outside_are_cut():
    s = Side([20, 30], True)
    q, k, v = make(s, s, 4, 2, 64, BF16)
    cut = lambda *at: torch.tensor(at, dtype=torch.int32, device="cuda")
    ref, _ = B.prompt_attend(q, k, v, first=cut(0, 20, 50))
    out, _ = B.prompt_attend(q, k, v, first=cut(-5, 20, 10 ** 9))
    assert torch.equal(out, ref)
    out = torch.zeros_like(q)
    B.prompt_attend(q, k, v, first=cut(20, 10, 50), out=out)       # the first one empty, the second from 10
    assert bool((out[:10] == 0).all())
    p = Side([50, 50], False)
    q, k, v = make(p, p, 4, 2, 64, BF16)
    ref, _ = B.prompt_attend(q, k, v)
    out, _ = B.prompt_attend(q, k, v, n_new=cut(50, 10 ** 9), n_k=cut(2 ** 31 - 1, 50))
    assert torch.equal(out, ref)
    out, lse = B.prompt_attend(q, k, v, n_new=cut(-1, -2 ** 31))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert B.prompt_status() == B.OK


def test_nothing_at_all():
    q = torch.zeros(0, 4, 64, dtype=BF16, device="cuda")
    first = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = B.prompt_attend(q, q[:, :2], q[:, :2], first=first)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    q = torch.randn(5, 4, 64, device="cuda").to(BF16)
    out, lse = B.prompt_attend(q, q[:0, :2], q[:0, :2], first=torch.tensor([0, 5], dtype=torch.int32, device="cuda"),
                               first_k=torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_streams_and_graphs():
    s = Side([300, 41], True)
    q, k, v = make(s, s, 8, 2, 128, BF16)
    ref, ref_lse = run(q, k, v, s, s)
    side = torch.cuda.Stream()
    first = s.arguments(("first", ""))["first"]
    side.wait_stream(torch.cuda.current_stream())
    out, lse = torch.empty_like(ref), torch.empty_like(ref_lse)
    B.prompt_attend(q, k, v, first=first, out=out, lse=lse, stream=side)
    side.synchronize()
    assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.prompt_attend(q, k, v, first=first, out=out, lse=lse)
    for seed in (1, 2):
        for x, y in zip((q, k, v), make(s, s, 8, 2, 128, BF16, seed)):
            x.copy_(y)
        first.copy_(torch.tensor([0, 300 - 50 * seed, 341], dtype=torch.int32))
        graph.replay()
        again = B.prompt_attend(q, k, v, first=first)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_the_same_call_gives_the_same_bits():
    s = Side([1500, 800], True)
    q, k, v = make(s, s, 16, 8, 128, BF16)
    a, b = run(q, k, v, s, s), run(q, k, v, s, s)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
