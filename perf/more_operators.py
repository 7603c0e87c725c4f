"""Cases for the verifier's prompts and verdicts: attention over whole prompts, the attention
weight that a prompt's keys receive, and scores of tokens from logits.

Prompts come packed (all sequences' rows one after another, with the offsets where each begins)
or padded (a fixed number of rows for each sequence, with the number that counts).  A sequence
may bring fewer query rows than key rows: its last rows, over all of its keys.
"""
import math

import torch

own = False

BF16, FP16, FP32 = "bfloat16", "float16", "float32"
AT_ONCE = 1 << 28          # elements of a plain form's widest intermediate


def listed():
    return [
        # one short question: a call's latency
        dict(name="prompt one", op="attend", n_seq=1, length=37, past=0, ragged=False, packed=True, hq=32, hkv=8, d=128, dtype=BF16),
        # a batch of prompts of all lengths
        dict(name="prompt batch", op="attend", n_seq=16, length=2048, past=0, ragged=True, packed=True, hq=32, hkv=8, d=128, dtype=BF16),
        # one very long document
        dict(name="prompt long", op="attend", n_seq=1, length=32768, past=0, ragged=False, packed=True, hq=32, hkv=8, d=128, dtype=BF16),
        # the next piece of long prompts, over the keys of all pieces so far
        dict(name="prompt piece", op="attend", n_seq=4, length=1024, past=15360, ragged=True, packed=False, hq=64, hkv=8, d=128, dtype=FP16),
        # a small model: narrow heads, three query heads to a key head, an empty sequence, rows behind the sequences
        dict(name="prompt odd", op="attend", n_seq=5, length=777, past=0, ragged=True, packed=False, hq=12, hkv=4, d=64, dtype=FP16),
        # what every row of a batch of prompts gave the keys
        dict(name="weigh batch", op="weigh", n_seq=16, length=2048, past=0, ragged=True, packed=True, window=0, hq=32, hkv=8, d=128, dtype=BF16),
        # what the last 64 rows of long prompts gave the keys
        dict(name="weigh window", op="weigh", n_seq=4, length=16384, past=0, ragged=True, packed=False, window=64, hq=32, hkv=8, d=128, dtype=FP16),
        # one prompt of a small model
        dict(name="weigh one", op="weigh", n_seq=1, length=1000, past=0, ragged=False, packed=True, window=0, hq=12, hkv=4, d=64, dtype=BF16),
        # one request's next token, with alternatives
        dict(name="score one", op="score", rows=1, vocab=128256, tokens=1, top=20, dtype=FP32),
        # the next tokens of a full batch
        dict(name="score batch", op="score", rows=64, vocab=128256, tokens=1, top=1, dtype=BF16),
        # the nodes of a draft tree with their drafted children; rows that begin anywhere
        dict(name="score tree", op="score", rows=60, vocab=32003, tokens=8, top=8, dtype=FP16),
        # every token of a prompt
        dict(name="score prompt", op="score", rows=2048, vocab=152064, tokens=1, top=5, dtype=BF16),
    ]


def draw(rng):
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)

    def spread(low, high):
        return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))

    while True:
        op = rng.choice(["attend", "attend", "weigh", "score"])
        if op == "score":
            c = dict(op=op, rows=spread(1, 4096), vocab=rng.choice([32000, 128256, 152064, spread(17, 262144), spread(17, 262144)]),
                     tokens=spread(1, 16), dtype=rng.choice([BF16, BF16, FP16, FP32]))
            c["top"] = rng.choice([0, 1, spread(2, min(64, c["vocab"]))])
        else:
            hq, hkv = rng.choice([(32, 8), (64, 8), (16, 16), (12, 4), (8, 1), (32, 4)])
            c = dict(op=op, n_seq=spread(1, 64), length=spread(1, 32768), past=rng.choice([0, 0, spread(1, 32768)]),
                     ragged=rng.random() < 0.7, packed=rng.random() < 0.6, hq=hq, hkv=hkv, d=rng.choice([64, 128, 128]),
                     dtype=rng.choice([BF16, BF16, FP16]))
            if op == "weigh":
                c["window"] = rng.choice([0, spread(1, 256)])
            n, top = c["n_seq"], c["length"] + c["past"]
            if n * max(c["length"] * c["hq"], top * c["hkv"]) * c["d"] > 32768 * 64 * 128:
                continue
        w = work(c)
        if w["bytes"] <= most_bytes and w["flops"] <= most_flops:
            return c


def counts(case):
    """Query rows and key rows of each sequence: all alike, or spread from an eighth to the whole,
    one of them empty where there are three or more."""
    n, top = case["n_seq"], case["length"]
    new = [top - (i * 7 % n) * (top - top // 8) // max(1, n - 1) if case["ragged"] else top for i in range(n)]
    if case["ragged"] and n >= 3:
        new[1] = 0
    return new, [t + (case["past"] - (i * 5 % n) * case["past"] // n if case["ragged"] and t else case["past"] * (t > 0))
                 for i, t in enumerate(new)]


def work(case):
    if case["op"] == "score":
        size = 4 if case["dtype"] == FP32 else 2
        cells = case["rows"] * case["vocab"]
        return {"bytes": cells * size + case["rows"] * (8 + 8 * case["tokens"] + 8 * case["top"]), "flops": 5.0 * cells}
    (new, keys), hq, hkv, d = counts(case), case["hq"], case["hkv"], case["d"]
    if case["op"] == "attend":
        pairs = sum(n * (c - n) + n * (n + 1) / 2 for n, c in zip(new, keys))
        return {"bytes": sum(new) * (4 * hq * d + 4 * hq) + sum(keys) * 4 * hkv * d, "flops": 4.0 * d * hq * pairs}
    live = [min(n, case["window"]) if case["window"] else n for n in new]      # the last rows of each sequence count
    pairs = sum(n * (c - n) + n * (n + 1) / 2 for n, c in zip(live, keys))
    return {"bytes": sum(live) * (2 * hq * d + 4 * hq + 4) + sum(keys) * hkv * (2 * d + 4), "flops": 2.0 * d * hq * pairs}


# ------------------------------------------------------------------ inputs ----

def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    kind = getattr(torch, case["dtype"])

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    if case["op"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        logits = torch.empty(rows, vocab, dtype=kind, device=dev)
        for r in range(0, rows, 256):
            part = normal(min(256, rows - r), vocab) * 2.5
            # some tokens are likely, and what a grammar forbids or no token has is out
            likely = torch.randint(0, vocab, (part.shape[0], 6), generator=gen, device=dev)
            part.scatter_add_(1, likely, 8 * torch.rand(likely.shape, generator=gen, device=dev) + 4)
            part[:, vocab - vocab // 64:] = -math.inf
            logits[r:r + 256] = part.to(kind)
        tokens = torch.randint(0, vocab - vocab // 64, (rows, case["tokens"]), generator=gen, device=dev, dtype=torch.int32)
        return dict(case=case, kind=kind, logits=logits, tokens=tokens)

    n_seq, hq, hkv, d = case["n_seq"], case["hq"], case["hkv"], case["d"]
    new, keys = counts(case)

    def offsets(n):
        return torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=dev)

    lead = lambda n, top: (max(1, sum(n)),) if case["packed"] else (n_seq, top)
    s = dict(case=case, kind=kind, new=new, keys=keys, scale=1.0 / math.sqrt(d))
    rows = lead(new, case["length"])
    if case["past"]:
        wide = lead(keys, case["length"] + case["past"])
        s["q"], s["k"], s["v"] = (normal(*rows, hq, d) * 2).to(kind), normal(*wide, hkv, d).to(kind), normal(*wide, hkv, d).to(kind)
    else:
        # queries, keys and values as slices of one projection
        both = torch.empty(*rows, hq + 2 * hkv, d, dtype=kind, device=dev)
        both[..., :hq, :] = (normal(*rows, hq, d) * 2).to(kind)
        both[..., hq:, :] = normal(*rows, 2 * hkv, d).to(kind)
        s["q"], s["k"], s["v"] = both[..., :hq, :], both[..., hq:hq + hkv, :], both[..., hq + hkv:, :]
    if case["packed"]:
        s["how"] = dict(first=offsets(new), first_k=offsets(keys))
    else:
        s["how"] = dict(n_new=torch.tensor(new, dtype=torch.int32, device=dev), n_k=torch.tensor(keys, dtype=torch.int32, device=dev))
    if case["op"] == "weigh":
        s["lse"] = plain_attend(s)["lse"]
        s["row_weight"] = None
        if case["window"]:
            s["row_weight"] = torch.zeros(rows, device=dev)
            for i in range(n_seq):
                part = sequence(s, s["row_weight"], i, new)
                part[max(0, new[i] - case["window"]):] = 1.0
    return s


def sequence(s, x, i, n):
    """The rows of x that are sequence i's."""
    if s["case"]["packed"]:
        return x[sum(n[:i]):sum(n[:i + 1])]
    return x[i, :n[i]]


# -------------------------------------------------------------- plain forms ----

def blocks(s, i):
    """Sequence i some rows at a time: where they begin, and their scaled products with its keys, -inf
    behind what each sees: [key head, query head of the group, row, key]."""
    case = s["case"]
    n, c, hkv = s["new"][i], s["keys"][i], case["hkv"]
    q = sequence(s, s["q"], i, s["new"]).float().unflatten(1, (hkv, -1)).permute(1, 2, 0, 3)     # [key head, group, row, d]
    k = sequence(s, s["k"], i, s["keys"]).float().transpose(0, 1).unsqueeze(1)
    step = max(1, AT_ONCE // max(1, case["hq"] * c))
    at = torch.arange(c, device=q.device)
    for r in range(0, n, step):
        part = q[:, :, r:r + step]
        x = (part.flatten(1, 2) @ k.squeeze(1).transpose(-1, -2)).unflatten(1, part.shape[1:3]) * s["scale"]
        row = torch.arange(r, r + part.shape[2], device=q.device) + (c - n)
        yield r, x.masked_fill_(at > row.unsqueeze(-1), -math.inf)


def plain_attend(s):
    case = s["case"]
    out = torch.zeros(s["q"].shape, dtype=s["kind"], device=s["q"].device)
    lse = torch.full(s["q"].shape[:-1], -math.inf, device=s["q"].device)
    for i in range(case["n_seq"]):
        if s["new"][i] == 0:
            continue
        v = sequence(s, s["v"], i, s["keys"]).float().transpose(0, 1)
        o, l = sequence(s, out, i, s["new"]), sequence(s, lse, i, s["new"])
        for r, x in blocks(s, i):
            rows = x.shape[2]
            top = x.amax(-1, keepdim=True)
            p = x.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            y = (p.flatten(1, 2) @ v).unflatten(1, p.shape[1:3]) / total
            o[r:r + rows] = y.permute(2, 0, 1, 3).flatten(1, 2).to(s["kind"])
            l[r:r + rows] = (total.log() + top).squeeze(-1).permute(2, 0, 1).flatten(1, 2)
    return {"out": out, "lse": lse}


def plain_weigh(s):
    case = s["case"]
    hkv = case["hkv"]
    lead = s["k"].shape[:-2]
    weight = torch.zeros(*lead[:-1], hkv, lead[-1], device=s["k"].device)
    for i in range(case["n_seq"]):
        if s["new"][i] == 0:
            continue
        w = sequence(s, weight.transpose(-1, -2), i, s["keys"])                # [key, key head]
        lse = sequence(s, s["lse"], i, s["new"]).unflatten(1, (hkv, -1)).permute(1, 2, 0).unsqueeze(-1)
        for r, x in blocks(s, i):
            rows = x.shape[2]
            p = x.sub_(lse[:, :, r:r + rows]).exp_()
            if s["row_weight"] is not None:
                p *= sequence(s, s["row_weight"], i, s["new"])[r:r + rows].unsqueeze(-1)
            w += p.sum((1, 2)).transpose(0, 1)
    return {"weight": weight}


def plain_score(s):
    case, logits = s["case"], s["logits"]
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    got = {"logp": [], "lse": [], "entropy": [], "top_id": [], "top_logp": []}
    at = torch.arange(vocab, device=logits.device)
    step = max(1, AT_ONCE // vocab)
    for r in range(0, rows, step):
        x = logits[r:r + step].float()
        high = x.amax(-1, keepdim=True)
        z = x - high
        e = z.exp()
        total = e.sum(-1, keepdim=True)
        lse = total.log() + high
        got["lse"].append(lse.squeeze(-1))
        got["entropy"].append((total.log() - (e * z.masked_fill_(e == 0, 0.0)).sum(-1, keepdim=True) / total).squeeze(-1))
        got["logp"].append(x.gather(-1, s["tokens"][r:r + step].long()) - lse)
        # one integer that orders by value, then by lowest index
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -1 - (bits & 0x7fffffff), bits) * (1 << 20) + (vocab - 1 - at)
        best = vocab - 1 - (order.topk(top, dim=-1).values & ((1 << 20) - 1))
        got["top_id"].append(best.to(torch.int32))
        got["top_logp"].append(x.gather(-1, best) - lse)
    return {name: torch.cat(parts) for name, parts in got.items()}


# ------------------------------------------------------------------ passes ----

def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"attend": plain_attend, "weigh": plain_weigh, "score": plain_score}[op](s)
    from paper_2608_03839_b200 import binding
    if op == "attend":
        out, lse = binding.prompt_attend(s["q"], s["k"], s["v"], scale=s["scale"], **s["how"])
        return {"out": out, "lse": lse}
    if op == "weigh":
        return {"weight": binding.prompt_weigh(s["q"], s["lse"], s["k"], row_weight=s["row_weight"], scale=s["scale"], **s["how"])}
    got = binding.token_scores(s["logits"], s["tokens"], top=s["case"]["top"])
    return {"logp": got.logp, "lse": got.lse, "entropy": got.entropy, "top_id": got.top_id, "top_logp": got.top_logp}


# ------------------------------------------------------------------- exact ----

def exact(case, seed):
    """The definitions in 64 bits: attention one sequence and one query head at a time, scores one row at a time."""
    s = prepare(case, seed)
    if case["op"] == "score":
        rows, top = case["rows"], case["top"]
        names = ("logp", "lse", "entropy", "top_id", "top_logp")
        got = {name: [] for name in names}
        for r in range(rows):
            x = s["logits"][r].double()
            lse = torch.logsumexp(x, 0)
            logp = x - lse
            ids = torch.sort(x, descending=True, stable=True).indices[:top]
            for name, y in zip(names, (logp[s["tokens"][r].long()], lse, -torch.special.xlogy(logp.exp(), logp.exp()).sum(),
                                       ids.to(torch.int32), logp[ids])):
                got[name].append(y)
        return {name: torch.stack(y) for name, y in got.items()}

    packed, hq, hkv = case["packed"], case["hq"], case["hkv"]
    new, keys = counts(case)
    dev = s["q"].device
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.full(s["q"].shape[:-1], -math.inf, dtype=torch.float64, device=dev)
    lead = s["k"].shape[:-2]
    weight = torch.zeros(*lead[:-1], hkv, lead[-1], dtype=torch.float64, device=dev)
    q0 = k0 = 0
    for i, (n, c) in enumerate(zip(new, keys)):
        a = (slice(q0, q0 + n),) if packed else (i, slice(0, n))
        b = (slice(k0, k0 + c),) if packed else (i, slice(0, c))
        q0, k0 = q0 + n, k0 + c
        for h in range(hq if n else 0):
            g = h // (hq // hkv)
            kd, vd = s["k"][b][:, g].double(), s["v"][b][:, g].double()
            for r in range(0, n, 4096):
                rows, see = min(4096, n - r), min(c, c - n + r + 4096)       # what the last of these rows sees
                if case["op"] == "weigh" and case["window"] and r + rows <= n - case["window"]:
                    continue
                x = s["q"][a][r:r + rows, h].double() @ kd[:see].T / math.sqrt(case["d"])
                x += torch.full((rows, see), -math.inf, dtype=torch.float64, device=dev).triu_(c - n + r + 1)
                if case["op"] == "attend":
                    total = torch.logsumexp(x, 1)
                    lse[a][r:r + rows, h] = total
                    out[a][r:r + rows, h] = (x - total[:, None]).exp() @ vd[:see]
                else:
                    p = (x - s["lse"][a][r:r + rows, h].double()[:, None]).exp()
                    if case["window"]:
                        p = p[max(0, n - case["window"] - r):]
                    (weight[g] if packed else weight[i, g])[b[-1]][:see] += p.sum(0)
    return {"out": out, "lse": lse} if case["op"] == "attend" else {"weight": weight}
