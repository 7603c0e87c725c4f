"""Scores of tokens from logits against 64 bits."""
import math

import pytest
import torch

from paper_2608_03839_b200 import binding as B

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def make(rows, vocab, dtype, seed=0, width=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, width or vocab, generator=g, device="cuda") * 3).to(dtype)


def check(logits, tokens=None, top=0):
    got = B.token_scores(logits, tokens, top)
    rows, vocab = logits.shape
    for r in range(0, rows, max(1, rows // 40)):
        x = logits[r].double()
        lse = torch.logsumexp(x, 0)
        empty = lse == -math.inf
        z = torch.where(x > -math.inf, x - lse, 0.0)
        p = torch.where(x > -math.inf, z.exp(), 0.0)
        mean = (p * z.abs()).sum().item()                  # in exp's units
        # Each exponential: two steps of 2^-23, and half a step of its argument (of 1.45 |z| and twice the
        # distance of the threads' maxima, in the mean 2 of mean + 1); sums: 16 terms, one a load (64), trees of 16.
        rel = 2.0 ** -24 * (4 + 16 + vocab / 4096 + 16 + 4 * mean + 4)
        tol = rel + 2.0 ** -22 * (0 if empty else abs(lse.item()))
        assert empty and got.lse[r] == -math.inf or abs(got.lse[r].item() - lse.item()) <= tol
        entropy = -(p * z).sum().item()
        assert abs(got.entropy[r].item() - entropy) <= rel * (2 + 2 * mean), (got.entropy[r].item(), entropy)

        def same(name, out, ids):
            for y, t in zip(out.tolist(), ids.tolist()):
                if not 0 <= t < vocab or x[t] == -math.inf:
                    assert y == -math.inf
                else:
                    want = (x[t] - lse).item()
                    assert abs(y - want) <= rel + 2.0 ** -22 * (abs(want) + 1), (name, y, want)
        if tokens is not None:
            same("logp", got.logp[r], tokens[r])
        best = torch.sort(x, descending=True, stable=True).indices[:top]
        assert got.top_id[r].tolist()[:vocab] == best.tolist()
        assert got.top_id[r].tolist()[vocab:] == [-1] * max(0, top - vocab)
        same("top", got.top_logp[r], got.top_id[r])
    return got


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 31, 255, 257, 2047, 2049, 8193, 32003, 128256, 262143])
@pytest.mark.parametrize("rows", [1, 3])
def test_vocabularies(dtype, vocab, rows):
    tokens = torch.randint(-2, vocab + 2, (rows, 5), device="cuda", dtype=torch.int32)
    for top in (0, 1, 20, 64):
        check(make(rows, vocab, dtype, vocab), tokens, top)


@pytest.mark.parametrize("rows", [17, 64, 150, 700])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_numbers_of_rows(rows, dtype):
    x = make(rows, 32000, dtype, rows)
    tokens = torch.randint(0, 32000, (rows, 1), device="cuda", dtype=torch.int32)
    check(x, tokens, 5)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_rows_of_any_alignment(dtype):
    for off, width in ((1, 5003), (3, 5008), (7, 5001)):
        x = make(6, 4990, dtype, off, width)[:, off:off + 4990]
        check(x, torch.arange(30, device="cuda", dtype=torch.int32).view(6, 5) * 160, 9)
    x = make(1, 5000, dtype).expand(4, -1)                 # the same row again
    got = check(x, None, 3)
    assert torch.equal(got.top_id[0], got.top_id[3])


@pytest.mark.parametrize("vocab", [300, 8192, 50000, 152064])
@pytest.mark.parametrize("top", [1, 10, 64])
def test_ties_go_to_the_lowest_token(vocab, top):
    same = torch.full((3, vocab), 1.5, device="cuda", dtype=BF16)
    same[1] = torch.randint(0, 3, (vocab,), device="cuda").to(BF16)
    same[2, vocab // 2:] = 2.0
    check(same, None, top)
    zeros = torch.zeros(2, vocab, device="cuda")
    zeros[0, ::2] = -0.0                                   # equal to 0
    check(zeros, None, top)


@pytest.mark.parametrize("vocab", [5000, 40000, 152064])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top", [1, 33, 64])
def test_orders_that_fill_the_list(vocab, dtype, top):
    """Ascending, descending, and everything of weight at the end."""
    up = torch.arange(vocab, device="cuda") * (20.0 / vocab)
    rows = torch.stack((up, -up, torch.where(up > 15, up, -math.inf), torch.where(up > 19.9, 0.0, -math.inf), up ** 2 / 3))
    check(rows.to(dtype), None, top)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [40, 9000, 128256])
def test_masked_tokens(dtype, vocab):
    x = make(5, vocab, dtype)
    x[0, 1:] = -math.inf                                   # one token is left: the first,
    x[1, :-1] = -math.inf                                  # the last
    x[2] = -math.inf                                       # none
    x[3, ::2] = -math.inf
    x[4] = torch.finfo(dtype).min                          # the type's lowest value is a number like any other
    tokens = torch.tensor([[0, 1, vocab - 1, -1]] * 5, device="cuda", dtype=torch.int32)
    got = check(x[:4], tokens[:4], 8)
    assert got.lse[2] == -math.inf and got.entropy[2] == 0 and got.top_id[2].tolist() == list(range(8))
    assert got.entropy[0] == 0 and got.logp[0, 0] == 0     # (x - m is 0, whatever x is)
    low = B.token_scores(x[4:], tokens[4:], 4)
    # (all equal: logp is the difference of two sums of 3e38's size only if somebody forms them)
    assert abs(low.logp[0, 0].item() + math.log(vocab)) < 1e-4 and abs(low.entropy[0].item() - math.log(vocab)) < 1e-4
    assert low.top_id[0].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_hold_no_numbers(bad):
    x = make(3, 33000, F32)
    ref = B.token_scores(x, torch.zeros(3, 1, device="cuda", dtype=torch.int32), 4)
    x[1, 20000] = bad
    got = B.token_scores(x, torch.zeros(3, 1, device="cuda", dtype=torch.int32), 4)
    for name in ("lse", "entropy", "logp", "top_logp"):
        a, b = getattr(got, name), getattr(ref, name)
        assert bool(torch.isnan(a[1]).all()) and torch.equal(a[::2], b[::2]), name
    if math.isnan(bad):                                    # no alternative
        x[1, 20000] = -math.inf
        assert got.top_id[1].tolist() == B.token_scores(x, None, 4).top_id[1].tolist()
    else:
        assert got.top_id[1, 0] == 20000
    x[0] = math.nan
    assert B.token_scores(x, None, 3).top_id[0].tolist() == [-1] * 3


def test_large_logits():
    """Distances count, not sizes."""
    x = make(4, 10000, F32)
    x += torch.tensor([1000.0, -1000.0, 30000.0, 0.0], device="cuda")[:, None]
    check(x, torch.arange(8, device="cuda", dtype=torch.int32).view(4, 2), 5)


def test_streams_graphs_and_bits():
    x = make(64, 50000, BF16)
    t = torch.randint(0, 50000, (64, 3), device="cuda", dtype=torch.int32)
    ref = B.token_scores(x, t, 7)
    fields = ("logp", "lse", "entropy", "top_id", "top_logp")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.token_scores(x, t, 7, stream=side)
    side.synchronize()
    assert all(torch.equal(getattr(ref, f), getattr(got, f)) for f in fields)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = B.token_scores(x, t, 7)
    x.copy_(make(64, 50000, BF16, 1))
    graph.replay()
    again = B.token_scores(x, t, 7)
    assert all(torch.equal(getattr(held, f), getattr(again, f)) for f in fields)


def test_nothing_at_all():
    got = B.token_scores(torch.zeros(0, 100, device="cuda"), torch.zeros(0, 2, device="cuda", dtype=torch.int32), 5)
    assert got.logp.shape == (0, 2) and got.top_id.shape == (0, 5) and got.lse.shape == (0,)
    got = B.token_scores(torch.zeros(2, 100, device="cuda"), torch.zeros(2, 0, device="cuda", dtype=torch.int32))
    assert got.logp.shape == (2, 0) and abs(got.lse[0].item() - math.log(100)) < 1e-5


def test_refusals():
    x = torch.zeros(2, 100, device="cuda")
    for call in (lambda: B.token_scores(x, top=65), lambda: B.token_scores(x, top=-1), lambda: B.token_scores(x, top=2 ** 32 + 1),
                 lambda: B.token_scores(x[:, :0])):
        with pytest.raises(B.OilbirdError):
            call()
    for call in (lambda: B.token_scores(x.T), lambda: B.token_scores(x.double()), lambda: B.token_scores(x.cpu()),
                 lambda: B.token_scores(x[0]), lambda: B.token_scores(x, torch.zeros(2, 1, device="cuda")),
                 lambda: B.token_scores(x, torch.zeros(3, 1, device="cuda", dtype=torch.int32))):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(RuntimeError, match="backward"):
        B.token_scores(x.requires_grad_())
