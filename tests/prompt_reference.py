"""Attention over whole prompts and the weight of their keys in 64 bits, with the bounds that the
library's roundings stay within."""
import math

import torch


class Side:
    """Rows of a batch of sequences, packed or padded: where they lie in a tensor."""

    def __init__(self, counts, packed, rows=None, lead=0, tail=0):
        self.counts, self.packed, self.lead = list(counts), packed, lead
        self.rows = rows or (lead + sum(counts) + tail if packed else max(counts))
        self.shape = (self.rows,) if packed else (len(counts), self.rows)

    def at(self, i):
        if not self.packed:
            return (i, slice(0, self.counts[i]))
        first = self.lead + sum(self.counts[:i])
        return (slice(first, first + self.counts[i]),)

    def arguments(self, names):
        """first (packed) or counts (padded) as the calls take them."""
        if self.packed:
            at = [self.lead + sum(self.counts[:i]) for i in range(len(self.counts) + 1)]
            return {names[0]: torch.tensor(at, dtype=torch.int32, device="cuda")}
        return {names[1]: torch.tensor(self.counts, dtype=torch.int32, device="cuda")}


def seen(n, c):
    """[n, c]: which keys a row sees."""
    return torch.arange(c, device="cuda") <= torch.arange(n, device="cuda")[:, None] + (c - n)


def attend(q, k, v, scale):
    """One sequence, in 64 bits: q [n, hq, d], k, v [c, hkv, d] -> out [n, hq, d], lse [n, hq], and for each
    row and channel the sums of p |v| and of |v|, for each row the largest sum of |scale q k| of a key it sees."""
    n, hq, d = q.shape
    c, hkv, _ = k.shape
    q, k, v = (x.double() for x in (q, k, v))
    k, v = (x.repeat_interleave(hq // hkv, 1) if c else x.new_zeros(0, hq, d) for x in (k, v))
    see = seen(n, c)
    x = (torch.einsum("nhd,chd->hnc", q, k) * scale).masked_fill(~see, -math.inf)
    size = (torch.einsum("nhd,chd->hnc", q.abs(), k.abs()) * abs(scale)).masked_fill(~see, 0.0)
    lse = torch.logsumexp(x, -1) if c else x.new_full((hq, n), -math.inf)
    p = torch.where(see, (x - torch.where(lse > -math.inf, lse, 0.0)[..., None]).exp(), 0.0)
    reach = size.amax(-1) if c else x.new_zeros(hq, n)
    return (torch.einsum("hnc,chd->nhd", p, v), lse.T, torch.einsum("hnc,chd->nhd", p, v.abs()),
            torch.einsum("nc,chd->nhd", see.double(), v.abs()), reach.T)


def check_attend(got, lse, ref, dtype, d):
    """Half a step of the type for the probabilities (as often as they count) and one for the result; what the
    fp32 sum of d products may be off by, in the exponent."""
    out, rl, mass, whole, reach = ref
    half = torch.finfo(dtype).eps / 2
    drift = d * 2.0 ** -24 * reach + 2.0 ** -20
    tol = (half + drift[..., None]) * mass * 1.01 + half * out.abs()
    if dtype is torch.float16:
        # Below 2^-14 half a step is 2^-25: of the result, and of each probability in units in which the row's
        # largest is 2^7 at least (so 2^-32 of the largest, whose probability is 1 at most).
        tol = tol + 2.0 ** -25 + 2.0 ** -32 * whole
    err = (got.double() - out).abs()
    assert bool((err <= tol).all()), f"off by {err.max().item():.3g}, {(err / tol.clamp(min=1e-30)).max().item():.3g} of the bound"
    there = rl > -math.inf
    assert torch.equal(lse > -math.inf, there)
    e = (lse.double() - rl)[there].abs()
    assert bool((e <= (drift + 2.0 ** -21 * rl.abs())[there]).all()), f"lse off by {e.max().item():.3g}"


def weigh(q, lse, k, row_weight, scale):
    """One sequence, in 64 bits: what each key receives, [hkv, c]; the same with |row_weight|, and the largest
    of the sums |scale q k| + |lse| of what goes into it."""
    n, hq, d = q.shape
    c, hkv, _ = k.shape
    q, lse, w = q.double(), lse.double(), row_weight.double()
    k = k.double().repeat_interleave(hq // hkv, 1)
    use = seen(n, c) & (w != 0)[:, None] & (lse.T > -math.inf)[..., None]
    x = torch.einsum("nhd,chd->hnc", q, k) * scale - lse.T[..., None]
    p = torch.where(use, x.exp() * w[:, None], 0.0)
    size = torch.einsum("nhd,chd->hnc", q.abs(), k.abs()) * abs(scale) + lse.abs().T[..., None]
    per = lambda y: y.unflatten(0, (hkv, -1)).sum((1, 2))
    reach = torch.where(use, size, 0.0).unflatten(0, (hkv, -1)).amax((1, 2)) if n else p.new_zeros(hkv, c)
    return per(p), per(p.abs()), reach


def check_weigh(got, ref, n_terms, d):
    """What the fp32 sums of d products and of a tile's 32 terms each may be off by; the sum over the tiles keeps what
    it loses (two steps and a half in all)."""
    w, mass, reach = ref
    tol = ((d + 8) * 2.0 ** -24 * reach + (32 + 8) * 2.0 ** -24 + n_terms * 2.0 ** -46) * mass * 1.01 + 1e-37
    err = (got.double() - w).abs()
    assert bool((err <= tol).all()), f"off by {err.max().item():.3g}, {(err / tol).max().item():.3g} of the bound"
