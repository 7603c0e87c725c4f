"""From prompts to verdicts: the prompt calls, the 4-bit cache and token scores one after another."""
import math
import os
import sys

import pytest
import torch

from paper_2608_03839_b200 import binding as B
from tests.prompt_reference import Side, attend, check_attend, check_weigh, weigh

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype,d,page", [(BF16, 128, 64), (F16, 64, 16)])
def test_packed_rows_join_as_padded_ones_do(dtype, d, page):
    counts = [70, 0, 1, 133]
    s = Side(counts, True, lead=2, tail=9)
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    both = new(*s.shape, 6, d).to(dtype)
    k, v, w = both[:, :2], both[:, 3:5], new(2, s.rows).abs()
    a, b = (B.KVCache(4, 2, d, 900, page_size=page, dtype=dtype) for _ in range(2))
    first = s.arguments(("first", ""))["first"]
    rows = torch.zeros(4, 133, 2, d, dtype=dtype, device="cuda"), torch.zeros(4, 133, 2, d, dtype=dtype, device="cuda")
    weight = torch.zeros(4, 2, 133, device="cuda")
    for i, n in enumerate(counts):
        rows[0][i, :n], rows[1][i, :n], weight[i, :, :n] = k[s.at(i)], v[s.at(i)], w[:, s.at(i)[0]]
    for _ in range(2):                                     # the second time behind the first
        a.append(k, v, first=first, weight=w)
        b.append(*rows, n_new=torch.tensor(counts, dtype=torch.int32, device="cuda"), weight=weight)
        for name in ("pages", "weight", "pos", "seq_len", "n_pos"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
    a.append(k, v, first=first)                            # no weights: 0
    assert a.dropped() == 0 and a.seq_len.tolist() == [3 * n for n in counts]
    # what leaves the rows is cut
    a.append(k, v, first=torch.tensor([-4, 3, 2, 200, 10 ** 9], dtype=torch.int32, device="cuda"))
    assert a.seq_len.tolist() == [213, 0, 201, 399 + s.rows - 200] and a.dropped() == 0


def test_packed_refusals():
    c = B.KVCache(2, 2, 64, 100)
    k = torch.zeros(10, 2, 64, dtype=BF16, device="cuda")
    first = torch.tensor([0, 5, 10], dtype=torch.int32, device="cuda")
    for bad in (dict(first=first[:2]), dict(first=first.long()), dict(first=first, n_new=first[:2]),
                dict(first=first, weight=torch.zeros(2, 2, 10, device="cuda"))):
        with pytest.raises(AssertionError):
            c.append(k, k, **bad)
    with pytest.raises(AssertionError):
        c.append(k[:, :1], k, first=first)
    assert c.seq_len.tolist() == [0, 0]


@pytest.mark.parametrize("packed", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_prompts_to_verdicts(packed, dtype):
    """A prompt in two pieces, its weights, the cache cut to the heaviest slots, a draft tree over it, its logits'
    scores: each step against 64 bits on what the step before it gave."""
    counts, hq, hkv, d, vocab = [300, 41, 512], 8, 2, 64, 1000
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    s = Side(counts, packed)
    q, k, v = (new(*s.shape, hq, d) * 2).to(dtype), new(*s.shape, hkv, d).to(dtype), new(*s.shape, hkv, d).to(dtype)
    how = s.arguments(("first", "n_new"))
    out, lse = B.prompt_attend(q, k, v, **how)
    for i in range(3):
        check_attend(out[s.at(i)], lse[s.at(i)], attend(q[s.at(i)], k[s.at(i)], v[s.at(i)], d ** -0.5), dtype, d)
    # the last rows as a piece of their own, over all keys: the same rows
    tail = Side([min(n, 50) for n in counts], packed)
    q2 = torch.zeros(*tail.shape, hq, d, dtype=dtype, device="cuda")
    for i, n in enumerate(tail.counts):
        q2[tail.at(i)] = q[s.at(i)][-n:]
    piece, _ = B.prompt_attend(q2, k, v, **tail.arguments(("first", "n_new")), **s.arguments(("first_k", "n_k")))
    for i, n in enumerate(tail.counts):
        ref = attend(q[s.at(i)], k[s.at(i)], v[s.at(i)], d ** -0.5)
        check_attend(piece[tail.at(i)], lse[s.at(i)][-n:], [x[-n:] for x in ref], dtype, d)
    w = B.prompt_weigh(q, lse, k, **how)
    ones = torch.ones(s.shape, device="cuda")
    for i, n in enumerate(counts):
        check_weigh(w[:, s.at(i)[0]] if packed else w[i][:, :n],
                    weigh(q[s.at(i)], lse[s.at(i)], k[s.at(i)], ones[s.at(i)], d ** -0.5), n * hq, d)
    cache = B.KVCache(3, hkv, d, 600, dtype=dtype)
    cache.append(k, v, weight=w, **how)
    cache.evict(128, sink=4, recent=32)
    assert cache.seq_len.tolist() == [128, 41, 128] and cache.n_pos.tolist() == counts
    for i, n in enumerate(counts):                          # the heaviest stay, with their weights
        mine = (w[:, s.at(i)[0]] if packed else w[i][:, :n])
        for h in range(hkv):
            slots = cache.pos[cache.page_table[i].long(), h].flatten()[:min(n, 128)].long()
            heavy = mine[h].clone()
            heavy[:4] = heavy[n - 32:] = math.inf
            assert set(slots.tolist()) == set(heavy.topk(min(n, 128)).indices.tolist())
            assert torch.equal(cache.weight[cache.page_table[i].long(), h].flatten()[:min(n, 128)], mine[h][slots])
    nodes = new(3, 6, hq + 2 * hkv, d).to(dtype)
    got, _ = cache.attend(nodes[:, :, :hq], nodes[:, :, hq:hq + hkv], nodes[:, :, hq + hkv:])
    head = new(hq * d, vocab) / (hq * d) ** 0.5
    logits = (got.flatten(2).float() @ head).to(dtype).flatten(0, 1)
    drafted = torch.randint(0, vocab, (18, 3), generator=g, device="cuda", dtype=torch.int32)
    scores = B.token_scores(logits, drafted, 4)
    p = torch.log_softmax(logits.double(), -1)
    assert (scores.logp.double() - p.gather(1, drafted.long())).abs().max() < 1e-4
    assert torch.equal(scores.top_id.long(), torch.sort(logits, descending=True, stable=True).indices[:, :4])
    assert (scores.entropy.double() + (p.exp() * p).sum(-1)).abs().max() < 1e-4
    assert B.prompt_status() == B.OK
