"""Prompt calls: what the binding refuses, waits that run out, threads, other streams, numbers at the ends of the types."""
import math
import threading

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, attend, check_attend, check_weigh, weigh

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(s, hq, hkv, d, dtype, seed=0, ks=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    ks = ks or s
    return ((new(*s.shape, hq, d) * 2).to(dtype), new(*ks.shape, hkv, d).to(dtype), new(*ks.shape, hkv, d).to(dtype))


def test_what_the_binding_refuses():
    s = Side([10, 20], True)
    q, k, v = make(s, 4, 2, 64, BF16)
    first = s.arguments(("first", ""))["first"]
    p = q.view(2, 15, 4, 64)
    n = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    ok = B.prompt_attend(q, k, v, first=first)
    for bad in (lambda: B.prompt_attend(q, k, v), lambda: B.prompt_attend(q, k, v, first=first.long()),
                lambda: B.prompt_attend(q, k, v, first=first.cpu()), lambda: B.prompt_attend(q, k, v, first=first, n_new=n),
                lambda: B.prompt_attend(q, k, v, first=first, n_k=n), lambda: B.prompt_attend(p, k, v),
                lambda: B.prompt_attend(p, p[:, :, :2], p[:, :, :2], first=first), lambda: B.prompt_attend(q, k[:20], v, first=first),
                lambda: B.prompt_attend(q, k, v[..., :32], first=first), lambda: B.prompt_attend(q, k.half(), v, first=first),
                lambda: B.prompt_attend(q.float(), k, v, first=first), lambda: B.prompt_attend(q.transpose(1, 2), k, v, first=first),
                lambda: B.prompt_attend(q, k, v, first=first, out=torch.empty_like(k)),
                lambda: B.prompt_attend(q, k, v, first=first, lse=torch.empty(30, 3, device="cuda")),
                lambda: B.prompt_attend(p, p[:, :, :2], p[:, :, :2], n_new=n[:1]),
                lambda: B.prompt_weigh(q, ok[1].half(), k, first=first),
                lambda: B.prompt_weigh(q, ok[1], k, first=first, row_weight=torch.ones(2, 15, device="cuda")),
                lambda: B.prompt_weigh(q, ok[1], k, first=first, weight=torch.ones(2, 29, device="cuda"))):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: B.prompt_attend(q[:, :3], k, v, first=first), lambda: B.prompt_attend(q, k, v, first=first, scale=math.nan),
                lambda: B.prompt_attend(q[..., :32].contiguous(), k[..., :32].contiguous(), v[..., :32].contiguous(), first=first),
                lambda: B.prompt_attend(torch.zeros(30 * 256 + 4, dtype=BF16, device="cuda")[4:].view(30, 4, 64), k, v, first=first),
                lambda: B.prompt_attend(torch.zeros(30 * 260, dtype=BF16, device="cuda").as_strided((30, 4, 64), (260, 64, 1)),
                                        k, v, first=first)):
        with pytest.raises(B.OilbirdError):
            bad()
    with pytest.raises(RuntimeError, match="backward"):
        B.prompt_attend(q.requires_grad_(), k, v, first=first)
    with torch.no_grad():
        assert torch.equal(B.prompt_attend(q, k, v, first=first)[0], ok[0])


@pytest.mark.parametrize("d,lengths", [(64, [3000, 300, 1]), (128, [700, 2000]), (128, [40])])
def test_waits_of_a_nanosecond_end_and_leave_everything_usable(d, lengths):
    """With next to no patience the kernels may give up anywhere: they say so or their results are right, and the
    next call with the usual limit is right again."""
    s = Side(lengths, True)
    q, k, v = make(s, 8, 2, d, BF16)
    how = s.arguments(("first", ""))
    want, lse = B.prompt_attend(q, k, v, **how)
    w = B.prompt_weigh(q, lse, k, **how)
    try:
        for _ in range(4):
            B.prompt_set_wait_limit(1)
            out = B.prompt_attend(q, k, v, **how)[0]
            if B.prompt_status() == B.OK:
                assert torch.equal(out, want)
            got = B.prompt_weigh(q, lse, k, **how)
            if B.prompt_status() == B.OK:
                assert torch.equal(got, w)
            B.prompt_set_wait_limit(0)
            assert torch.equal(B.prompt_attend(q, k, v, **how)[0], want) and torch.equal(B.prompt_weigh(q, lse, k, **how), w)
            assert B.prompt_status() == B.OK
    finally:
        B.prompt_set_wait_limit(0)


def test_calls_from_two_threads_on_two_streams():
    cases = []
    for seed in (0, 1):
        s = Side([1200, 300 + seed, 77], True)
        q, k, v = make(s, 8, 2, 128, BF16, seed)
        how = s.arguments(("first", ""))
        x = torch.randn(20, 40000, device="cuda")
        out, lse = B.prompt_attend(q, k, v, **how)
        cases.append((q, k, v, how, x, out, lse, B.prompt_weigh(q, lse, k, **how), B.token_scores(x, None, 5)))
    torch.cuda.synchronize()
    wrong = []

    def work(q, k, v, how, x, out, lse, w, sc):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                a, b = B.prompt_attend(q, k, v, **how)
                c, e = B.prompt_weigh(q, lse, k, **how), B.token_scores(x, None, 5)
                stream.synchronize()
                if not (torch.equal(a, out) and torch.equal(b, lse) and torch.equal(c, w) and torch.equal(e.top_id, sc.top_id) and
                        torch.equal(e.entropy, sc.entropy)):
                    wrong.append(1)
    threads = [threading.Thread(target=work, args=c) for c in cases]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_large_scores_and_values(dtype):
    """Scores of thousands, where one key takes all; values at the end of the type."""
    s = Side([200], True)
    q, k, v = make(s, 4, 2, 64, dtype)
    q, k = q * 20, k * 20
    v = v.sign() * torch.finfo(dtype).max * 0.5
    out, lse = B.prompt_attend(q, k, v, **s.arguments(("first", "")))
    ref = attend(q, k, v, 0.125)
    check_attend(out, lse, ref, dtype, 64)
    w = B.prompt_weigh(q, lse, k, **s.arguments(("first", "")))
    check_weigh(w, weigh(q, lse, k, torch.ones(200, device="cuda"), 0.125), 800, 64)


def test_what_a_row_sees_comes_through():
    """NaN and infinities in queries, keys and values reach the rows that see them, in attention and weights."""
    s = Side([300], True)
    how = s.arguments(("first", ""))
    q, k, v = make(s, 4, 2, 64, BF16)
    ref, rl = B.prompt_attend(q, k, v, **how)
    v2 = v.clone()
    v2[0, 0, 5] = math.inf
    out, lse = B.prompt_attend(q, k, v2, **how)
    assert bool((out[:, :2, 5] == math.inf).all()) and torch.equal(out[:, 2:], ref[:, 2:]) and torch.equal(lse, rl)
    assert torch.equal(out[:, :2, 6:], ref[:, :2, 6:])
    q2 = q.clone()
    q2[100, 1] = math.nan
    out, lse = B.prompt_attend(q2, k, v, **how)
    assert bool(torch.isnan(out[100, 1]).all()) and torch.isnan(lse[100, 1])
    out[100, 1], lse[100, 1] = ref[100, 1], rl[100, 1]
    assert torch.equal(out, ref) and torch.equal(lse, rl)
    w = B.prompt_weigh(q2, rl, k, **how)
    assert bool(torch.isnan(w[0, :101]).all()) and bool(torch.isfinite(w[0, 101:]).all()) and bool(torch.isfinite(w[1]).all())


@pytest.mark.parametrize("rows", [1, 3, 64, 65])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (4, 1, 128)])
def test_few_rows_over_many_keys(rows, hq, hkv, d):
    """Clusters share an item's keys: of rows that see many tiles, few and none; unseen values of infinity."""
    qs, ks = Side([rows, 1, min(rows, 2)], True), Side([5000 + rows, 1, 130], True, tail=3)
    q, k, v = make(qs, hq, hkv, d, BF16, 2, ks)
    how = {**qs.arguments(("first", "")), **ks.arguments(("first_k", ""))}
    v[ks.rows - 3:] = math.inf
    out, lse = B.prompt_attend(q, k, v, **how)
    w = B.prompt_weigh(q, lse, k, **how)
    for i in range(3):
        a, b = qs.at(i), ks.at(i)
        check_attend(out[a], lse[a], attend(q[a], k[b], v[b], d ** -0.5), BF16, d)
        check_weigh(w[:, b[0]], weigh(q[a], lse[a], k[b], torch.ones(qs.rows, device="cuda")[a], d ** -0.5), qs.counts[i] * hq, d)
    assert B.prompt_status() == B.OK


def test_rows_that_read_infinities_they_do_not_see_over_many_keys():
    """The same with the infinity among the keys of the rows' own last tile."""
    qs, ks = Side([40], True), Side([3000], True)
    q, k, v = make(qs, 4, 1, 64, F16, 3, ks)
    v[2990] = math.inf                                     # seen by the last ten rows alone
    how = {**qs.arguments(("first", "")), **ks.arguments(("first_k", ""))}
    out, lse = B.prompt_attend(q, k, v, **how)
    clean = v.clone()
    clean[2990] = 0.0
    ref = attend(q, k, clean, 0.125)
    check_attend(out[:30], lse[:30], [x[:30] for x in ref], F16, 64)
    assert bool((out[30:] == math.inf).all())


def test_many_short_sequences_with_weights_at_their_ends():
    s = Side([700, 3, 0] * 60, True)
    q, k, _ = make(s, 4, 2, 64, BF16)
    how = s.arguments(("first", ""))
    lse = B.prompt_attend(q, k, k, **how)[1]
    rw = torch.zeros(s.rows, device="cuda")
    for i, n in enumerate(s.counts):
        rw[s.at(i)][max(0, n - 5):] = 0.5
    w = B.prompt_weigh(q, lse, k, row_weight=rw, **how)
    for i in (0, 1, 2, 90, 177):
        a = s.at(i)
        check_weigh(w[:, a[0]], weigh(q[a], lse[a], k[a], rw[a], 0.125), s.counts[i] * 4, 64)
