"""Speculative decoding passes over a 4-bit key/value cache of bounded length, on one GPU.

A small synthetic verifier (one attention layer with grouped query heads, random weights, texts
that repeat phrases) runs the draft path and the cache together, as a serving loop would:

    Pool.query      drafts continuations for every request's current state
    merge_chains    makes each request's draft tree and its attention mask
    KVCache.attend  verifies all nodes of all trees against the cache, with that mask
    KVCache.weigh   adds the weight the accepted path gave each slot
    KVCache.append  stores the accepted path's keys and values, chosen from the tree's rows
    KVCache.evict   cuts every sequence back to its budget, lightest slots first
    Pool.append     remembers the accepted positions for later drafts

and compares each pass's attention with attention in 64 bits over the exact 16-bit keys and
values of the whole text, which shows what four bits and eviction cost together.

    python examples/verify_passes.py [--requests 4] [--passes 40] [--budget 256] [--dtype bf16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_03839_b200 import binding as B  # noqa: E402


class Verifier:
    """Random projections of token and position: what a layer's attention gets and returns."""

    def __init__(self, vocab, width, q_heads, kv_heads, head_dim, dtype, gen):
        new = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        self.embed = new(vocab, width)
        self.wq = new(width, q_heads * head_dim) / width ** 0.5
        self.wk = new(width, kv_heads * head_dim) / width ** 0.5
        self.wv = new(width, kv_heads * head_dim) / width ** 0.5
        self.heads, self.kv_heads, self.d, self.dtype = q_heads, kv_heads, head_dim, dtype

    def state(self, tok, prev):
        """The hidden state the pool keys on: a token in the context of the one before it."""
        return (self.embed[tok] + 0.5 * self.embed[prev]).to(torch.bfloat16)

    def qkv(self, tok, prev):
        x = self.state(tok, prev).float()
        cut = lambda w, h: (x @ w).view(*tok.shape, h, self.d).to(self.dtype)
        return cut(self.wq, self.heads), cut(self.wk, self.kv_heads), cut(self.wv, self.kv_heads)


def make_texts(n, length, vocab, gen):
    """[n, length] tokens: phrases of 12 drawn again and again from a small common stock."""
    stock = torch.randint(0, vocab, (24, 12), generator=gen, device="cuda")
    return stock[torch.randint(0, 24, (n, -(-length // 12)), generator=gen, device="cuda")].reshape(n, -1)[:, :length]


def exact_attention(q, k, v):
    """q [rows, heads, d] over k and v [len, kv_heads, d], all seen, in 64 bits."""
    g = q.shape[1] // k.shape[1]
    k, v = (x.double().repeat_interleave(g, 1) for x in (k, v))
    p = torch.softmax(torch.einsum("mhd,nhd->hmn", q.double(), k) * q.shape[2] ** -0.5, -1)
    return torch.einsum("hmn,nhd->mhd", p, v)


def accepted_path(tok, parent, n_nodes, text, at):
    """Nodes of one tree along the text: the root (the token at `at`), then child by child."""
    path, node = [0], 0
    while at + len(path) < len(text):
        step = [j for j in range(1, n_nodes) if parent[j] == node and tok[j] == text[at + len(path)]]
        if not step:
            break
        node = step[0]
        path.append(node)
    return path


def run(requests=4, passes=40, budget=256, dtype=torch.bfloat16, prompt=200, max_nodes=32, seed=0,
        log=print):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ver = Verifier(2048, 256, 8, 2, 64, dtype, gen)
    length = prompt + passes * max_nodes + 1
    texts = make_texts(requests, length, 2048, gen)
    prev = torch.cat([texts[:, :1], texts[:, :-1]], 1)
    text_host = texts.tolist()
    everything = ver.qkv(texts, prev)                        # for the comparison alone

    pool = B.Pool(256, requests * length, device=0)
    cache = B.KVCache(requests, ver.kv_heads, ver.d, max(prompt, budget) + max_nodes, dtype=dtype)
    params = B.QueryParams(k=4, theta=0.5, depth_mode=B.DEPTH_FIXED, cont_len=8)

    # The prompts: stored, then weighed by the last positions' own queries, as any later pass is.
    q, k, v = (x[:, :prompt] for x in everything)
    cache.append(k, v)
    look = q[:, prompt - 16:prompt]
    cache.weigh(look, cache.attend(look)[1])
    cache.evict(budget)
    for s in range(requests):
        pool.append(ver.state(texts[s, :prompt], prev[s, :prompt]), texts[s, :prompt].int())

    at = [prompt] * requests                                 # each request's anchor: committed, not stored
    pooled = [prompt] * requests                             # how far the pool knows each text
    taken, worst = 0, 0.0
    for _ in range(passes):
        pos = torch.tensor(at, device="cuda")
        rows = torch.arange(requests, device="cuda")
        anchor, before = texts[rows, pos], texts[rows, pos - 1]
        # the last verified state chose the anchor; what follows in the past begins two rows on
        hit = pool.query(ver.state(before, texts[rows, pos - 2]), params)

        tok = torch.full((requests, max_nodes), -1, dtype=torch.int32, device="cuda")
        parent = torch.full_like(tok, -1)
        tok[:, 0] = anchor
        n_nodes = torch.ones(requests, dtype=torch.int32, device="cuda")
        tree = B.merge_chains(tok, parent, n_nodes, hit.cont_tok, hit.cont_len)

        node = tok.clamp(min=0).long()
        up = torch.where(parent >= 0, node.gather(1, parent.clamp(min=0).long()), before[:, None])
        q, k, v = ver.qkv(node, up)
        out, lse = cache.attend(q, k, v, tree.mask, n_nodes)

        # Which nodes the verifier agrees with: here, those that follow the request's text.
        path = [accepted_path(t, p, n, text_host[s], at[s]) for s, (t, p, n) in
                enumerate(zip(tok.tolist(), parent.tolist(), n_nodes.tolist()))]
        n_new = torch.tensor([len(p) for p in path], dtype=torch.int32, device="cuda")
        select = torch.tensor([p + [0] * (max_nodes - len(p)) for p in path], dtype=torch.int32, device="cuda")
        on_path = torch.zeros(requests, max_nodes, device="cuda")
        for s, p in enumerate(path):
            on_path[s, p] = 1.0

        for s, p in enumerate(path):                         # the last accepted node sees all before it
            end = at[s] + len(p)
            full = exact_attention(q[s, p[-1]:p[-1] + 1], everything[1][s, :end], everything[2][s, :end])
            err = (out[s, p[-1]].double() - full[0]).norm() / full.norm()
            worst = max(worst, err.item())

        weight = cache.weigh(q, lse, k, tree.mask, n_nodes, row_weight=on_path)
        cache.append(k, v, n_new, select, weight)
        cache.evict(budget)
        for s, p in enumerate(path):
            at[s] += len(p)
            taken += len(p)
            if at[s] - pooled[s] >= 24:                      # a trace a piece: continuations stay in one text
                new = slice(pooled[s], at[s])
                pool.append(ver.state(texts[s, new], prev[s, new]), texts[s, new].int())
                pooled[s] = at[s]

    assert cache.n_pos.tolist() == at, "every accepted position was stored once"
    assert cache.seq_len.tolist() == [min(budget, n) for n in at] and cache.dropped() == 0
    result = {"tokens_per_pass": taken / (passes * requests), "positions": at,
              "slots": cache.seq_len.tolist(), "worst_error": worst}
    log(f"{requests} requests, {passes} passes: {result['tokens_per_pass']:.2f} tokens a pass; positions {at} in "
        f"{result['slots']} slots of 4 bits; attention off by at most {worst:.3f} of its norm")
    pool.close()
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--passes", type=int, default=40)
    ap.add_argument("--budget", type=int, default=256)
    ap.add_argument("--dtype", choices=("bf16", "f16"), default="bf16")
    a = ap.parse_args()
    run(a.requests, a.passes, a.budget, {"bf16": torch.bfloat16, "f16": torch.float16}[a.dtype])
