"""What the binding does around the prompt calls and token scores: gradients and streams."""
import pytest
import torch

from paper_2608_03839_b200 import binding as B

pytestmark = pytest.mark.gpu


def made(n=300):
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda h: torch.randn(n, h, 64, generator=g, device="cuda").bfloat16()
    return new(8), new(2), new(2), torch.tensor([0, n], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("which", ["lse", "row_weight", "q", "k"])
def test_weights_of_what_wants_a_gradient_are_refused(which):
    q, k, v, first = made()
    t = {"lse": B.prompt_attend(q, k, v, first=first)[1], "row_weight": torch.ones(300, device="cuda"), "q": q, "k": k}
    want = B.prompt_weigh(first=first, **t)
    t[which].requires_grad_()
    with pytest.raises(RuntimeError, match="backward"):
        B.prompt_weigh(first=first, **t)
    with torch.no_grad():
        assert torch.equal(B.prompt_weigh(first=first, **t), want)


@pytest.mark.parametrize("which", ["out", "lse"])
def test_results_that_want_a_gradient_are_refused(which):
    q, k, v, first = made()
    t = {"out": torch.zeros_like(q), "lse": torch.zeros(300, 8, device="cuda")}[which].requires_grad_()
    with pytest.raises(RuntimeError, match="backward"):
        B.prompt_attend(q, k, v, first=first, **{which: t})


def test_the_cache_refuses_logarithms_and_weights_that_want_a_gradient():
    q, k, v, first = made()
    c = B.KVCache(1, 2, 64, 400)
    with pytest.raises(RuntimeError, match="backward"):
        c.append(k, v, first=first, weight=torch.ones(2, 300, device="cuda", requires_grad=True))
    assert c.seq_len.tolist() == [0]
    c.append(k, v, first=first)
    row = q[None, :1]
    lse = c.attend(row)[1].requires_grad_()
    with pytest.raises(RuntimeError, match="backward"):
        c.weigh(row, lse)
    with torch.no_grad():
        c.weigh(row, lse)


CALLS = {
    "attend": lambda m, stream: list(B.prompt_attend(m.q, m.k, m.v, first=m.first, stream=stream)),
    "weigh": lambda m, stream: [B.prompt_weigh(m.q, m.lse, m.k, first=m.first, stream=stream)],
    "scores": lambda m, stream: [t for t in vars(B.token_scores(m.x, None, 3, stream=stream)).values() if t is not None],
    "cache attend": lambda m, stream: list(m.cache.attend(m.q[None, :40], m.k[None, :40], m.v[None, :40], stream=stream)),
    "cache weigh": lambda m, stream: [m.cache.weigh(m.q[None, :40], m.tree[1], m.k[None, :40], stream=stream)],
    "cache read": lambda m, stream: list(m.cache.read(300, stream=stream)),
    "pool query": lambda m, stream: [t for t in vars(m.pool.query(m.keys[:40], B.QueryParams(k=8), stream=stream)).values()
                                     if isinstance(t, torch.Tensor)],
    "ring query": lambda m, stream: list(vars(m.ring.query(m.keys[:40], m.anchors[:40], stream=stream)).values()),
}


class Made:
    def __init__(self):
        self.q, self.k, self.v, self.first = made()
        self.lse = B.prompt_attend(self.q, self.k, self.v, first=self.first)[1]
        self.x = torch.randn(70, 5000, device="cuda")
        self.cache = B.KVCache(1, 2, 64, 400)
        self.cache.append(self.k, self.v, first=self.first)
        self.tree = self.cache.attend(self.q[None, :40], self.k[None, :40], self.v[None, :40])
        self.keys = torch.randn(64, 128, device="cuda").bfloat16()
        self.anchors = torch.arange(64, device="cuda", dtype=torch.int32)
        self.pool = B.Pool(128, 1024)
        self.pool.append(self.keys, self.anchors)
        self.ring = B.Ring(128, 64, 8)
        self.ring.append(self.keys, self.anchors, torch.zeros(64, 8, device="cuda", dtype=torch.int32))


@pytest.fixture(scope="module")
def m():
    return Made()


def busy(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(400_000_000)                     # some 200 ms


@pytest.mark.parametrize("call", CALLS)
def test_results_of_another_stream_are_not_used_again_too_early(m, call):
    """A result dropped while the stream that fills it is still busy: its memory goes to nobody meanwhile."""
    CALLS[call](m, None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(side)
    got = CALLS[call](m, side)
    at = {t.data_ptr(): (t.shape, t.dtype) for t in got if t.numel()}
    del got
    again = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in at.values() for _ in range(3)]
    assert not side.query(), "the stream was to be busy"
    assert not {t.data_ptr() for t in again} & set(at)
    torch.cuda.synchronize()


@pytest.mark.parametrize("call", CALLS)
def test_results_of_another_stream_do_not_lie_where_the_current_one_is_at_work(m, call):
    """The current stream is busy on tensors that have been dropped: their memory is its own until it is through."""
    side = torch.cuda.Stream()
    got = CALLS[call](m, None)
    like = [(t.shape, t.dtype) for t in got]
    del got
    torch.cuda.synchronize()
    busy(torch.cuda.current_stream())
    mine = [torch.zeros(shape, dtype=dtype, device="cuda") for shape, dtype in like for _ in range(3)]
    ends = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in mine]
    del mine
    got = CALLS[call](m, side)
    assert not torch.cuda.current_stream().query(), "the stream was to be busy"
    for t in got:
        lo, hi = t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()
        assert not any(a < hi and lo < b for a, b in ends)
    torch.cuda.synchronize()
