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
