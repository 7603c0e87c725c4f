"""Cases for the verifier's 4-bit key/value cache: attention over it, accumulated attention
weight, storing into it and evicting from it.

A cache keeps, for every (slot, key/value head), the key and the value as 4-bit codes with a
16-bit scale and offset for each group of 64 channels, and beside them the attention weight
the slot has received (fp32) and the position it stands for (int32).  Pages hold 16, 32 or 64
slots; a table names the pages of each sequence.
"""
import math

import numpy as np
import torch

own = False

GROUP = 64
BF16, FP16 = "bfloat16", "float16"


def listed():
    return [
        # one request decoding, short context: a call's latency
        dict(name="attend one", op="attend", n_seq=1, length=517, ragged=False, nodes=1, hq=32, hkv=8, d=128, page=64, dtype=BF16),
        # a full batch decoding, contexts of all lengths
        dict(name="attend batch", op="attend", n_seq=64, length=8192, ragged=True, nodes=1, hq=32, hkv=8, d=128, page=64, dtype=BF16),
        # one request with a very long document
        dict(name="attend long", op="attend", n_seq=1, length=131085, ragged=False, nodes=1, hq=64, hkv=8, d=128, page=64, dtype=FP16),
        # verification of full draft trees (60 nodes) for a small batch
        dict(name="attend trees", op="attend", n_seq=8, length=4096, ragged=True, nodes=60, hq=32, hkv=8, d=128, page=64, dtype=BF16),
        # one draft tree over a long context
        dict(name="attend tree long", op="attend", n_seq=1, length=65541, ragged=False, nodes=60, hq=32, hkv=8, d=128, page=32, dtype=BF16),
        # a small model: narrow heads, three query heads to a key head, small pages, an empty sequence
        dict(name="attend odd", op="attend", n_seq=5, length=777, ragged=True, nodes=7, hq=12, hkv=4, d=64, page=16, dtype=FP16),
        # the weight a batch's decoding step adds
        dict(name="weigh batch", op="weigh", n_seq=64, length=8192, ragged=True, nodes=1, hq=32, hkv=8, d=128, page=64, dtype=BF16),
        # the weight of the accepted paths of a batch of draft trees
        dict(name="weigh trees", op="weigh", n_seq=8, length=4096, ragged=True, nodes=60, hq=32, hkv=8, d=128, page=32, dtype=FP16),
        # the accepted paths join the cache
        dict(name="append paths", op="append", n_seq=16, length=1000, ragged=True, nodes=60, take=7, hq=32, hkv=8, d=128, page=64, dtype=BF16),
        # prompts join the cache
        dict(name="append prompts", op="append", n_seq=4, length=100, ragged=True, nodes=4096, take=0, hq=32, hkv=8, d=128, page=64, dtype=FP16),
        # a bounded cache after a verification step: a few slots over the budget
        dict(name="evict step", op="evict", n_seq=16, length=1031, ragged=True, budget=1024, hq=32, hkv=8, d=128, page=64, dtype=BF16),
        # prompts cut to the budget before decoding begins
        dict(name="evict prompts", op="evict", n_seq=8, length=32768, ragged=True, budget=4096, hq=32, hkv=8, d=128, page=32, dtype=FP16),
    ]


def draw(rng):
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)

    def spread(low, high):
        return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))

    while True:
        hq, hkv = rng.choice([(32, 8), (64, 8), (16, 16), (12, 4), (8, 1), (32, 4)])
        c = dict(op=rng.choice(["attend", "attend", "attend", "weigh", "append", "evict"]), n_seq=spread(1, 64),
                 length=spread(1, 131072), ragged=rng.random() < 0.7, hq=hq, hkv=hkv, d=rng.choice([64, 128, 128]),
                 page=rng.choice([16, 32, 64, 64]), dtype=rng.choice([BF16, BF16, FP16]))
        if c["op"] in ("attend", "weigh"):
            c["nodes"] = rng.choice([1, 1, spread(2, 64), spread(2, 64)])
        elif c["op"] == "append":
            c["take"] = rng.choice([0, spread(1, 16)])
            c["nodes"] = rng.randint(c["take"], 64) if c["take"] else spread(1, 4096)
        else:
            c["budget"] = max(8, int(c["length"] * rng.uniform(0.1, 1.0)))
        w = work(c)
        held = c["n_seq"] * (c["length"] + c.get("nodes", 0)) * c["hkv"] * c["d"]
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops and held <= 64 * 8192 * 8 * 128:
            return c


def lengths(case):
    """Slots that each sequence holds before the pass: all alike, or spread from nothing (with
    three sequences or more) or half to the whole.  Sequences to be cut are spread down to the
    budget where that is less than half."""
    n, top = case["n_seq"], case["length"]
    if not case["ragged"]:
        return [top] * n
    low = min(top, case["budget"]) if case["op"] == "evict" else top // 2
    got = [top - (i * 7 % n) * (top - low) // max(1, n - 1) for i in range(n)]
    if n >= 3 and case["op"] != "evict":
        got[1] = 0
    return got


def taken(case):
    """Rows that join each sequence in an append, or nodes of each draft tree."""
    n, top = case["n_seq"], case.get("take") or case.get("nodes", 0)
    return [top - (i * 5 % n) * (top // 2) // max(1, n - 1) if case["ragged"] else top for i in range(n)]


def accepted(case):
    """Nodes of each draft tree that verification accepted: a path of seven at most."""
    return [min(7, t, 1 + i * 3 % 7) for i, t in enumerate(taken(case))]


def work(case):
    groups, slots, new = case["d"] // GROUP, sum(lengths(case)), sum(taken(case))
    row = groups * 36                       # bytes of one key or one value: 32 of codes, 4 of scale and offset, each group
    wide = 2 * case["d"]                    # the same in 16 bits
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "attend":
        pairs = sum(n * (m + t / 2) for n, m, t in zip(taken(case), lengths(case), taken(case)))
        return {"bytes": slots * hkv * 2 * row + new * (2 * hq * wide + 2 * hkv * wide + 4 * hq + 8), "flops": 4.0 * d * hq * pairs}
    if case["op"] == "weigh":
        pairs = sum(a * (m + a / 2) for a, m in zip(accepted(case), lengths(case)))
        rows = sum(accepted(case))
        return {"bytes": slots * hkv * (row + 8) + rows * (hq * wide + 4 * hq + 12) + new * hkv * (wide + 4), "flops": 2.0 * d * hq * pairs}
    if case["op"] == "append":
        return {"bytes": new * hkv * (2 * wide + 2 * row + 12) + new * hkv * (2 * row + 2 * wide), "flops": 12.0 * new * hkv * d}
    moved = sum(max(0, m - case["budget"]) * min(m, case["budget"]) / m for m in lengths(case))
    kept = sum(min(m, case["budget"]) for m in lengths(case))
    return {"bytes": hkv * (slots * 8 + moved * 2 * (2 * row + 8) + kept * (2 * row + 2 * wide)), "flops": 8.0 * slots * hkv}


# ------------------------------------------------------------------ inputs ----

def quantise(x, kind):
    """x [..., d] in 32 bits -> codes [..., d], scale and offset [..., d / 64] in 16 bits."""
    g = x.unflatten(-1, (-1, GROUP))
    low, high = g.amin(-1), g.amax(-1)
    scale = ((high * 0.5 - low * 0.5) / 7.5).to(kind)
    half = scale.float().unsqueeze(-1) * 0.5
    code = torch.round((g * 0.5 - low.unsqueeze(-1) * 0.5) / half).clamp(0, 15)
    code = torch.where(half > 0, code, torch.zeros_like(code))
    return code.flatten(-2).to(torch.int32), scale, low.to(kind)


def packed(x, kind):
    """x [pages, heads, slots, d] -> the bytes of its codes and of its scales and offsets, each [pages, heads, ...]."""
    code, scale, low = quantise(x, kind)
    w = code.unflatten(-1, (-1, GROUP // 8, 4, 2))                  # word, channel pair, even / odd
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device=x.device)
    w = (w << shift).sum((-1, -2)).to(torch.int32)                  # [.., slots, groups, 8]
    codes = w.transpose(-2, -3).contiguous().view(torch.uint8).flatten(2)
    meta = torch.stack((scale, low), -1).contiguous().view(torch.uint8).flatten(2)
    return codes, meta


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    kind = getattr(torch, case["dtype"])
    n_seq, hq, hkv, d, page = case["n_seq"], case["hq"], case["hkv"], case["d"], case["page"]
    held, new = lengths(case), taken(case)
    room = [m + (t if case["op"] == "append" else 0) for m, t in zip(held, new)]
    need = [-(-r // page) for r in room]
    most = max(1, max(need))
    n_pages = sum(need) + 3

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    # the pages of a sequence are scattered; entries behind its last page name no page
    table = torch.full((n_seq, most), -1, dtype=torch.int32)
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32).cpu()
    at = 0
    for i, c in enumerate(need):
        table[i, :c] = order[at:at + c]
        at += c
    table = table.to(dev)

    # keys with some channels off centre, as a model's are; values around zero
    lean = normal(hkv, 1, d) * (torch.rand(hkv, 1, d, generator=gen, device=dev) < 0.1) * 3
    kc, km = packed((normal(n_pages, hkv, page, d) + lean).to(kind).float(), kind)
    vc, vm = packed((normal(n_pages, hkv, page, d) * 0.5).to(kind).float(), kind)
    pages = torch.cat((kc, km, vc, vm), -1)
    del kc, km, vc, vm

    # weights, positions, lengths and counts of positions in one buffer
    cells = n_pages * hkv * page
    book = torch.zeros(2 * cells + 2 * n_seq, dtype=torch.int32, device=dev)
    shape = (n_pages, hkv, page)
    weight, pos = book[:cells].view(torch.float32).view(shape), book[cells:2 * cells].view(shape)
    seq_len, n_pos = book[2 * cells:2 * cells + n_seq], book[2 * cells + n_seq:]
    weight.copy_((normal(*shape) * 2).exp() * (torch.rand(shape, generator=gen, device=dev) < 0.9))
    seq_len.copy_(torch.tensor(held, dtype=torch.int32))
    first = torch.rand(n_seq, hkv, most * page, generator=gen, device=dev).argsort(-1)
    first = first if case["op"] == "evict" and case["length"] <= case["budget"] + 64 else torch.arange(most * page, device=dev).expand_as(first)
    spread = (first * 3 + torch.randint(0, 3, first.shape, generator=gen, device=dev)).to(torch.int32)
    spread = spread.view(n_seq, hkv, most, page).transpose(1, 2)
    pos[table[table >= 0].long()] = spread[table >= 0]
    n_pos.copy_(3 * torch.tensor(held, dtype=torch.int32) + 3)

    state = dict(case=case, kind=kind, pages=pages, book0=book.clone(), book=book, weight=weight, pos=pos, table=table,
                 seq_len=seq_len, n_pos=n_pos, most=most * page, scale=1.0 / math.sqrt(d))
    if case["op"] == "append":
        width = case["nodes"]
        state["k"] = (normal(n_seq, width, hkv, d) + lean.transpose(0, 1)).to(kind)
        state["v"] = (normal(n_seq, width, hkv, d) * 0.5).to(kind)
        state["n_new"] = torch.tensor(new, dtype=torch.int32, device=dev)
        state["gain"] = torch.rand(n_seq, hkv, width, generator=gen, device=dev)
        state["select"], state["rows"] = None, width
        if case["take"]:
            some = torch.rand(n_seq, width, generator=gen, device=dev).argsort(-1)[:, :case["take"]].sort(-1).values
            state["select"], state["rows"] = some.to(torch.int32).contiguous(), case["take"]
    elif case["op"] in ("attend", "weigh"):
        m = case["nodes"]
        # queries, keys and values as slices of one projection
        both = normal(n_seq, m, (hq + 2 * hkv), d).to(kind)
        both[:, :, :hq] *= 2
        state["q"], state["k"], state["v"] = both[:, :, :hq], both[:, :, hq:hq + hkv], both[:, :, hq + hkv:]
        state["n_new"] = torch.tensor(new, dtype=torch.int32, device=dev)
        # each node's parent is an earlier node; a node sees itself and its ancestors
        parent = (torch.rand(n_seq, m, generator=gen, device=dev) * torch.arange(m, device=dev)).long()
        sees = torch.eye(m, device=dev).repeat(n_seq, 1, 1)
        sees.scatter_(-1, parent.unsqueeze(-1), 1.0)
        for _ in range(6):
            sees = (sees @ sees > 0).float()
        bits = torch.ones(m, dtype=torch.int64, device=dev) << torch.arange(m, device=dev)
        state["mask"] = (sees.long() * bits).sum(-1)
        if case["op"] == "weigh":
            state["lse"] = plain_attend(state)["lse"]
            ok = torch.zeros(n_seq, m)
            for i, a in enumerate(accepted(case)):
                ok[i, :a] = 1.0
            state["accepted"] = ok.to(dev)
    return state


# -------------------------------------------------------------- plain forms ----

def opened(s):
    """The cache's keys and values in 32 bits, in the order of their slots: [sequence, head, slot, d]."""
    case, kind = s["case"], s["kind"]
    page, groups = case["page"], case["d"] // GROUP
    blocks = s["pages"][s["table"].clamp(min=0).long()]              # [sequence, page, head, bytes]
    return tuple(values(b, page, groups, kind) for b in blocks.chunk(2, -1))


def values(block, page, groups, kind):
    codes, meta = block.split([groups * page * 32, groups * page * 4], -1)
    w = codes.contiguous().view(torch.int32).unflatten(-1, (groups, page, 8))
    shift = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=w.device, dtype=torch.int32)
    c = ((w.unsqueeze(-1) >> shift) & 15).flatten(-2)                # [.., groups, slots, 64]
    meta = meta.contiguous().view(kind).unflatten(-1, (page, groups, 2)).transpose(-2, -3).float()
    x = c * meta[..., 0:1] + meta[..., 1:2]
    return x.transpose(-2, -3).flatten(-2).transpose(1, 2).flatten(2, 3)   # [sequence, head, slot, d]


def scores(s):
    """Scaled products of every query row with the slots and with the new nodes, -inf where it does
    not look: [sequence, key head, query head of the group, node, slot or node]; and the values."""
    case = s["case"]
    hkv, m = case["hkv"], case["nodes"]
    k, v = opened(s)
    q = s["q"].float().unflatten(2, (hkv, -1)).permute(0, 2, 3, 1, 4)        # [sequence, key head, group, node, d]
    k = torch.cat((k, s["k"].float().transpose(1, 2)), 2)
    v = torch.cat((v, s["v"].float().transpose(1, 2)), 2)
    x = (q.flatten(2, 3) @ k.transpose(-1, -2)).unflatten(2, (-1, m)) * s["scale"]
    node = torch.arange(m, device=q.device)
    sees = ((s["mask"].unsqueeze(-1) >> node) & 1).bool() & (node < s["n_new"].unsqueeze(-1)).unsqueeze(1)
    sees = sees & (node < s["n_new"].unsqueeze(-1)).unsqueeze(-1)
    slot = torch.arange(s["most"], device=q.device) < s["seq_len"].unsqueeze(-1)
    slot = slot.unsqueeze(1) & (node < s["n_new"].unsqueeze(-1)).unsqueeze(-1)
    return x.masked_fill(~torch.cat((slot, sees), -1)[:, None, None], -math.inf), v


def plain_attend(s):
    x, v = scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = (x - top).exp()
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v).unflatten(2, p.shape[2:4]) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (total.log() + top).squeeze(-1)
    return {"out": o.permute(0, 3, 1, 2, 4).flatten(2, 3).to(s["kind"]), "lse": lse.permute(0, 3, 1, 2).flatten(2, 3)}


def spread_to_pages(s, at, whole, part):
    """`whole` [pages, heads, slots] with part [sequence, head, slot] in the places where `at` holds."""
    case = s["case"]
    seq, head, slot = at.nonzero(as_tuple=True)
    whole = whole.clone()
    whole[s["table"][seq, slot // case["page"]].long(), head, slot % case["page"]] = part[at]
    return whole


def per_slot(s, whole):
    """[pages, heads, slots] -> [sequence, head, slot]."""
    return whole[s["table"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)


def plain_weigh(s):
    x, _ = scores(s)
    lse = s["lse"].unflatten(2, (s["case"]["hkv"], -1)).permute(0, 2, 3, 1).unsqueeze(-1)
    p = torch.where(x > -math.inf, (x - lse).exp(), torch.zeros_like(x)) * s["accepted"][:, None, None, :, None]
    got = p.sum((2, 3))
    slots, nodes = got.split([s["most"], s["case"]["nodes"]], -1)
    at = (torch.arange(s["most"], device=x.device) < s["seq_len"].unsqueeze(-1)).unsqueeze(1).expand_as(slots)
    return {"weight": spread_to_pages(s, at, s["weight"], per_slot(s, s["weight"]) + slots), "nodes": nodes}


def plain_append(s):
    case = s["case"]
    rows = s["rows"]
    take = torch.arange(rows, device="cuda").expand(case["n_seq"], -1) if s["select"] is None else s["select"].long()
    fits = torch.arange(rows, device="cuda") < s["n_new"].unsqueeze(-1)             # [sequence, row]

    def stored(x):
        x = x.gather(1, take[:, :, None, None].expand(-1, -1, *x.shape[2:])).float()
        code, scale, low = quantise(x, s["kind"])
        y = code.unflatten(-1, (-1, GROUP)) * scale.float().unsqueeze(-1) + low.float().unsqueeze(-1)
        return torch.where(fits[:, :, None, None], y.flatten(-2), torch.zeros_like(x)).to(s["kind"])

    slot = s["seq_len"].unsqueeze(-1) + torch.arange(rows, device="cuda")
    seq, row = fits.nonzero(as_tuple=True)
    page, cell = s["table"][seq, slot[seq, row] // case["page"]].long(), slot[seq, row] % case["page"]
    weight, pos = s["weight"].clone(), s["pos"].clone()
    weight[page, :, cell] = s["gain"].transpose(1, 2)[seq, take[seq, row]]
    pos[page, :, cell] = (s["n_pos"][seq] + row).to(torch.int32).unsqueeze(-1).expand(-1, case["hkv"])
    return {"k": stored(s["k"]), "v": stored(s["v"]), "weight": weight, "pos": pos,
            "seq_len": s["seq_len"] + s["n_new"], "n_pos": s["n_pos"] + s["n_new"]}


def bounds(case):
    """Positions that are never evicted: the first ones, and the newest."""
    return min(4, case["budget"] // 4), case["budget"] // 4


def plain_evict(s):
    case = s["case"]
    budget, (sink, recent) = case["budget"], bounds(case)
    weight, pos = per_slot(s, s["weight"]), per_slot(s, s["pos"])
    slot = torch.arange(s["most"], device="cuda").expand_as(pos)
    size = s["seq_len"][:, None, None]
    after = size.clamp(max=budget)
    safe = (pos < sink) | (pos >= s["n_pos"][:, None, None] - recent)
    value = torch.where(safe, torch.full_like(weight, math.inf), weight)
    value = torch.where(slot < size, value, torch.full_like(weight, -math.inf))
    order = torch.where(slot < size, pos, torch.full_like(pos, 2 ** 31 - 1)).sort(dim=-1, stable=True).indices
    order = order.gather(-1, value.gather(-1, order).sort(dim=-1, descending=True, stable=True).indices)
    rank = torch.zeros_like(order).scatter(-1, order, slot)
    keep = rank < after
    hole, mover = ~keep & (slot < after), keep & (slot >= after)
    # the i-th free slot takes the i-th kept slot behind the budget
    nth = torch.where(mover, mover.cumsum(-1) - 1, torch.full_like(slot, s["most"]))
    source = torch.zeros(*slot.shape[:2], s["most"] + 1, dtype=torch.int64, device="cuda").scatter(-1, nth, slot)
    source = torch.where(hole, source.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), slot)

    def kept(x):
        x = x.gather(2, source[:, :, :budget, None].expand(-1, -1, -1, x.shape[-1]))
        x = torch.where((slot < after)[:, :, :budget, None], x, torch.zeros_like(x))
        short = budget - x.shape[2]
        x = torch.cat((x, x.new_zeros(*x.shape[:2], short, x.shape[3])), 2) if short > 0 else x
        return x.transpose(1, 2).to(s["kind"])

    k, v = opened(s)
    return {"k": kept(k), "v": kept(v), "weight": spread_to_pages(s, hole, s["weight"], weight.gather(-1, source)),
            "pos": spread_to_pages(s, hole, s["pos"], pos.gather(-1, source)), "seq_len": after.flatten().to(torch.int32)}


# ------------------------------------------------------------------ passes ----

def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"attend": plain_attend, "weigh": plain_weigh, "append": plain_append, "evict": plain_evict}[op](s)
    cache = s.get("cache")
    if cache is None:
        from paper_2608_03839_b200 import binding
        cache = s["cache"] = binding.KVCache.over(s["pages"], s["weight"], s["pos"], s["table"], s["seq_len"], s["n_pos"],
                                                  dtype=s["kind"])
    if op == "attend":
        out, lse = cache.attend(s["q"], s["k"], s["v"], mask=s["mask"], n_new=s["n_new"], scale=s["scale"])
        return {"out": out, "lse": lse}
    s["book"].copy_(s["book0"])              # what the calls below update, as it was
    if op == "weigh":
        nodes = cache.weigh(s["q"], s["lse"], s["k"], mask=s["mask"], n_new=s["n_new"], row_weight=s["accepted"], scale=s["scale"])
        return {"weight": s["weight"], "nodes": nodes}
    if op == "append":
        start = s["book0"][-2 * s["case"]["n_seq"]:-s["case"]["n_seq"]]
        cache.append(s["k"], s["v"], n_new=s["n_new"], select=s["select"], weight=s["gain"])
        k, v = cache.read(s["rows"], start=start)
        return {"k": k, "v": v, "weight": s["weight"], "pos": s["pos"], "seq_len": s["seq_len"], "n_pos": s["n_pos"]}
    sink, recent = bounds(s["case"])
    cache.evict(s["case"]["budget"], sink=sink, recent=recent)
    k, v = cache.read(s["case"]["budget"])
    return {"k": k, "v": v, "weight": s["weight"], "pos": s["pos"], "seq_len": s["seq_len"]}


# ------------------------------------------------------------------- exact ----

def exact(case, seed):
    """The definitions in 64 bits, one sequence at a time."""
    s = prepare(case, seed)
    op, dev, kind = case["op"], "cuda", s["kind"]
    page, hkv, hq, d, groups = case["page"], case["hkv"], case["hq"], case["d"], case["d"] // GROUP
    held, new = lengths(case), taken(case)
    table = s["table"].cpu().numpy()
    # byte and shift of every channel's code inside the 32 bytes of a group
    channel = np.arange(GROUP)
    bit = 32 * (channel // 8) + 4 * (channel % 8 // 2) + 16 * (channel % 2)
    byte, shift = torch.from_numpy(bit // 8).to(dev), torch.from_numpy(bit % 8).to(dev)

    def cached(i, which):
        """Keys (0) or values (1) that sequence i holds: [head, slot, d]."""
        n = -(-held[i] // page)
        b = s["pages"][torch.from_numpy(table[i, :n]).long().to(dev)]
        half = b.shape[-1] // 2
        b = b[..., which * half:(which + 1) * half]
        x = torch.zeros(n, hkv, page, d, dtype=torch.float64, device=dev)
        meta = b[..., groups * page * 32:].contiguous().view(kind).double().view(n, hkv, page, groups, 2)
        for g in range(groups):
            raw = b[..., g * page * 32:(g + 1) * page * 32].reshape(n, hkv, page, 32)
            code = torch.bitwise_right_shift(raw[..., byte].int(), shift.int()) & 15
            x[..., g * GROUP:(g + 1) * GROUP] = meta[..., g, 1:] + code.double() * meta[..., g, :1]
        return x.permute(1, 0, 2, 3).reshape(hkv, n * page, d)[:, :held[i]]

    def looks(i):
        """Which of its new nodes each node of sequence i sees."""
        words = s["mask"][i].cpu().numpy().astype(np.int64).view(np.uint64)
        m = new[i]
        return torch.tensor([[bool(int(words[a]) >> b & 1) for b in range(m)] for a in range(m)], device=dev).view(m, m)

    def logits(i, h):
        """For query head h of sequence i, in 64 bits: nodes x (slots, then nodes)."""
        t, g = new[i], h // (hq // hkv)
        q = s["q"][i, :t, h].double()
        x = torch.cat((q @ keys[g].T, q @ s["k"][i, :t, g].double().T), 1) / math.sqrt(d)
        x[:, held[i]:][~looks(i)] = -math.inf
        return x

    if op == "attend":
        out = torch.zeros(case["n_seq"], case["nodes"], hq, d, dtype=torch.float64, device=dev)
        lse = torch.full((case["n_seq"], case["nodes"], hq), -math.inf, dtype=torch.float64, device=dev)
        for i in range(case["n_seq"]):
            keys, vals = cached(i, 0), cached(i, 1)
            for h in range(hq):
                t, g = new[i], h // (hq // hkv)
                x = logits(i, h)
                lse[i, :t, h] = torch.logsumexp(x, 1)
                out[i, :t, h] = torch.softmax(x, 1) @ torch.cat((vals[g], s["v"][i, :t, g].double()), 0)
        return {"out": out, "lse": lse}
    if op == "weigh":
        weight = s["weight"].double()
        nodes = torch.zeros(case["n_seq"], hkv, case["nodes"], dtype=torch.float64, device=dev)
        for i in range(case["n_seq"]):
            keys = cached(i, 0)
            got = torch.zeros(hkv, held[i] + new[i], dtype=torch.float64, device=dev)
            for h in range(hq):
                x = logits(i, h) - s["lse"][i, :new[i], h].double()[:, None]
                got[h // (hq // hkv)] += (x.exp() * s["accepted"][i, :new[i]].double()[:, None]).sum(0)
            nodes[i, :, :new[i]] = got[:, held[i]:]
            at = np.arange(held[i])
            weight[torch.from_numpy(table[i, at // page]).long().to(dev), :, torch.from_numpy(at % page).to(dev)] += got[:, :held[i]].T
        return {"weight": weight, "nodes": nodes}
    if op == "append":
        weight, pos = s["weight"].double(), s["pos"].clone()
        kept = {"k": torch.zeros(case["n_seq"], s["rows"], hkv, d, dtype=torch.float64, device=dev)}
        kept["v"] = torch.zeros_like(kept["k"])
        for i in range(case["n_seq"]):
            rows = torch.arange(new[i], device=dev) if s["select"] is None else s["select"][i, :new[i]].long()
            for name in ("k", "v"):
                x = s[name][i, rows].double().view(new[i], hkv, groups, GROUP)
                low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
                scale = ((high - low) / 15).to(kind).double()
                code = torch.where(scale > 0, torch.round((x - low) / scale).clamp(0, 15), 0.0)
                kept[name][i, :new[i]] = (low + code * scale).view(new[i], hkv, d)
            at = held[i] + np.arange(new[i])
            p, c = torch.from_numpy(table[i, at // page]).long().to(dev), torch.from_numpy(at % page).to(dev)
            weight[p, :, c] = s["gain"][i].T[rows].double()
            pos[p, :, c] = (int(s["n_pos"][i]) + torch.arange(new[i], device=dev)).int()[:, None]
        return {**kept, "weight": weight, "pos": pos, "seq_len": s["seq_len"] + s["n_new"], "n_pos": s["n_pos"] + s["n_new"]}
    budget, (sink, recent) = case["budget"], bounds(case)
    weight, pos = s["weight"].cpu().numpy().copy(), s["pos"].cpu().numpy().copy()
    got = torch.zeros(2, case["n_seq"], budget, hkv, d, dtype=torch.float64, device=dev)
    for i in range(case["n_seq"]):
        at, fit = np.arange(held[i]), min(held[i], budget)
        p, c = table[i, at // page], at % page
        kv = [cached(i, 0), cached(i, 1)]
        for h in range(hkv):
            w, x = weight[p, h, c], pos[p, h, c]
            safe = (x < sink) | (x >= int(s["n_pos"][i]) - recent)
            keep = np.zeros(held[i], bool)
            keep[np.lexsort((x, -w, ~safe))[:fit]] = True
            src = at[:fit].copy()
            src[~keep[:fit]] = at[fit:][keep[fit:]]
            weight[p[:fit], h, c[:fit]], pos[p[:fit], h, c[:fit]] = w[src], x[src]
            for n in (0, 1):
                got[n, i, :fit, h] = kv[n][h][torch.from_numpy(src).to(dev)]
    return {"k": got[0], "v": got[1], "weight": torch.from_numpy(weight).double().to(dev), "pos": torch.from_numpy(pos).to(dev),
            "seq_len": torch.tensor([min(m, budget) for m in held], dtype=torch.int32, device=dev)}
