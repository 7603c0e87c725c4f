"""The 4-bit key/value cache where its operators can go wrong: rows and tiles of zeros, what a row
does not see, probabilities far below the largest, extreme values, slots without content.

Every case runs on both attention kernels: up to 16 rows (nodes x query heads of a key head), and more.
"""
import numpy as np
import pytest
import torch

from oracle import kv as O
from paper_2608_03839_b200 import binding as B
from test_gpu_kv import KIND, UNIT, Made, check_attend, f64, sees_of, tree_mask

pytestmark = pytest.mark.gpu


def custom(keys, values, d=128, page=64, dtype="bf16"):
    """A cache of the given [n_seq, n, hkv, d] keys and values (16-bit elements)."""
    n_seq, n, hkv, _ = keys.shape
    per = max(1, -(-n // page))
    c = Made([0] * n_seq, hkv, d, page, dtype, max_pages=per, spare=n_seq * per + 1)
    c.table.copy_(torch.randperm(n_seq * per + 1)[:n_seq * per].int().view(n_seq, per))
    if n:
        c.cache.append(keys.to(KIND[dtype]), values.to(KIND[dtype]))
    return c


# ---------------------------------------------------------------- rows and keys of zeros ----

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,hq", [(1, 4), (4, 4), (30, 4), (60, 8)])
def test_zero_queries_over_zero_keys(m, hq, d, dtype):
    """Every score is 0: the result is the mean of the values the row sees, lse the logarithm of
    their number.  (A new nodes' tile always has slots that a row does not see.)"""
    for held in (0, 5, 130, 300):
        zero = torch.zeros(2, held, 1, d, device="cuda")
        c = custom(zero, torch.randn(2, held, 1, d, device="cuda"), d, 16, dtype)
        q, kn = (torch.zeros(2, m, h, d, device="cuda").to(KIND[dtype]) for h in (hq, 1))
        vn = c.rand(2, m, 1, d).to(KIND[dtype])
        mask = tree_mask(2, m, 3)
        out, lse = c.cache.attend(q, kn, vn, mask=mask)
        check_attend(c, q, kn, vn, mask, None, out, lse, d ** -0.5)


@pytest.mark.parametrize("m,hq", [(1, 4), (30, 4)])
def test_zero_queries_over_pages_that_name_nothing(m, hq):
    """Whole tiles without a page in front of, between and behind slots that exist."""
    c = Made([700, 300, 300], 1, 128, 64)
    c.table[0, 0:3], c.table[0, 6:9] = -1, 1 << 30
    c.table[1, :4], c.table[2, :] = -1, -1
    q = torch.zeros(3, m, hq, 128, device="cuda").bfloat16()
    out, lse = c.cache.attend(q)
    check_attend(c, q, None, None, None, None, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-30])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,hq", [(1, 4), (3, 4), (30, 4)])
def test_scale_of_zero_and_below(m, hq, dtype, scale):
    c = Made([300, 0, 140], 1, 128, 64, dtype)
    q, kn, vn = (c.rand(3, m, h, 128).to(KIND[dtype]) for h in (hq, 1, 1))
    mask = tree_mask(3, m, 5)
    out, lse = c.cache.attend(q, kn, vn, mask=mask, scale=scale)
    # (the checker's bounds take a positive scale: the sign goes to the queries, exactly)
    check_attend(c, q if scale >= 0 else -q, kn, vn, mask, None, out, lse, abs(scale))
    q, kn = q * 0, kn * 0
    out, lse = c.cache.attend(q, kn, vn, mask=mask, scale=scale)
    check_attend(c, q, kn, vn, mask, None, out, lse, abs(scale))


# ---------------------------------------------------------- what a row does not see ----

@pytest.mark.parametrize("dtype,big", [("bf16", 3e38), ("f16", 6e4)])
@pytest.mark.parametrize("m,hq", [(3, 4), (40, 4), (40, 8)])
@pytest.mark.parametrize("held", [0, 70])
def test_large_hidden_nodes_change_nothing(m, hq, held, dtype, big):
    """Rows are bit for bit the same whatever finite keys and values the nodes they do not see hold."""
    c = Made([held, held // 2], 1, 128, 64, dtype)
    q, kn, vn = (c.rand(2, m, h, 128).to(KIND[dtype]) for h in (hq, 1, 1))
    mask = torch.ones(2, m, dtype=torch.int64, device="cuda") << torch.arange(m, device="cuda")
    mask[:, 2:] |= 2                                             # most rows also see node 1
    want, wl = c.cache.attend(q, kn, vn, mask=mask)
    check_attend(c, q, kn, vn, mask, None, want, wl, 128 ** -0.5)
    kn[:, 0], vn[:, 0] = big, -big                               # row 0 alone sees node 0
    got, gl = c.cache.attend(q, kn, vn, mask=mask)
    assert torch.equal(gl[:, 1:], wl[:, 1:]) and torch.equal(got[:, 1:], want[:, 1:])
