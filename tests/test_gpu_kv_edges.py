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


# ------------------------------------------- probabilities far below the largest ----

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,hq", [(1, 8), (2, 8), (10, 8), (40, 8)])
@pytest.mark.parametrize("nats", [12.0, 17.5])
def test_one_slot_far_above_the_others(nats, m, hq, dtype):
    """An attention sink: one slot with a value of zero, `nats` above 32,768 others whose values
    are alike, so that what each adds is small but all of it counts.  (As many sequences, over the
    same pages, as leave every one whole to a block.)

    A probability is an f16 operand: off by 2^-11 of itself, or, where it is small, by 2^-25 of
    an operand of one.  Operands go up to 2^15, so that the largest probability is one of at least
    2^7: 2^-32 absolute for each slot.  Values are rounded by 2^-11 of themselves at most."""
    n, d, n_seq = 32768, 128, 320
    gen = torch.Generator(device="cuda").manual_seed(4)
    u = torch.randn(d, generator=gen, device="cuda")
    u /= u.norm()
    like = torch.linspace(0.5, 1.0, d, device="cuda")[torch.randperm(d, generator=gen, device="cuda")]
    keys = torch.randn(1, n + 1, 1, d, generator=gen, device="cuda") * 0.05
    values = like + 0.01 * torch.randn(1, n + 1, 1, d, generator=gen, device="cuda")
    keys[0, 777, 0], values[0, 777, 0] = u * 16, 0.0
    c = custom(keys, values, d, 64, dtype)
    many = B.KVCache.over(c.pages, c.weight, c.pos, c.table.repeat(n_seq, 1), c.seq_len.repeat(n_seq),
                          c.n_pos.repeat(n_seq), dtype=KIND[dtype], workspace=c.cache.workspace)
    q = (u * nats / 16 * d ** 0.5 + 0.01 * torch.randn(n_seq, m, hq, d, generator=gen, device="cuda")).to(KIND[dtype])
    out, lse = many.attend(q)
    k, v, _ = c.dense(0, 0)
    top, step = np.abs(v).max(), np.ptp(k, -1).max() / 15
    for s in (0, 131, 319):
        row = f64(q[s], dtype).reshape(-1, d)
        x = (row @ k.T) * d ** -0.5
        p = np.exp(x - x.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        want, got = p @ v, f64(out[s], dtype).reshape(-1, d)
        mag = d ** -0.5 * (np.abs(row) @ (np.abs(k).T + 2 * np.abs(k).max())).max()
        # (the last term of e: keys as the sum of two f16 numbers, off by 2^-13 of the scale)
        e = 2.0 ** -24 * (2 * d + 12) * mag + 2.0 ** -21 + 2.0 ** -13 * d ** -0.5 * np.abs(row).sum(-1).max() * step
        tol = UNIT[dtype] * np.abs(want) + (p @ np.abs(v)) * (2 * 2.0 ** -11 + 2 * e) + n * 2.0 ** -32 * 2 * top + 2.0 ** -25
        assert np.all(np.abs(got - want) <= tol), (np.abs(got - want).max(), tol.min(), np.abs(want).max())


# ------------------------------------------------------------------- extreme values ----

@pytest.mark.parametrize("m,hq", [(1, 4), (4, 4), (30, 4)])
def test_values_near_the_largest_number(m, hq):
    c = Made([200, 17], 1, 128, 64, "bf16", v_gain=2e35)
    q = (c.rand(2, m, hq, 128) * 0.5).bfloat16()
    out, lse = c.cache.attend(q)
    check_attend(c, q, None, None, None, None, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("m,hq", [(1, 4), (30, 4)])
def test_keys_near_the_largest_number(m, hq):
    """Keys of 1e35 under queries of 1e-35: ordinary scores."""
    c = Made([0, 0], 1, 64, 64, max_pages=3, spare=6)
    c.table.copy_(torch.arange(6).int().view(2, 3))
    c.cache.append((c.rand(2, 150, 1, 64) * 2e35).bfloat16(), c.rand(2, 150, 1, 64).bfloat16())
    q = (c.rand(2, m, hq, 64) * 2e-35).bfloat16()
    out, lse = c.cache.attend(q)
    check_attend(c, q, None, None, None, None, out, lse, 64 ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_read_of_the_largest_numbers_is_finite(dtype):
    """15 * scale + lo may pass the type's largest number, as the scale was rounded up: the largest
    number it is then."""
    top = float(torch.finfo(KIND[dtype]).max)
    d = 128
    k = torch.zeros(1, 6, 1, d, device="cuda")
    k[0, 0, 0, 3] = top
    k[0, 1, 0, 70] = -top
    k[0, 2, 0, 0], k[0, 2, 0, 1] = top, -top
    k[0, 3] = top
    k[0, 4, 0, :64] = torch.linspace(0, 1, 64, device="cuda") * top
    k[0, 5, 0, 5] = float("inf")
    c = custom(k, -k, d, 16, dtype)
    for got, want in zip(c.cache.read(6), (k, -k)):
        got, want = got[0, :, 0].double(), want[0, :, 0].double()
        assert torch.isfinite(got[:5]).all() and torch.isfinite(got[5, 64:]).all() and torch.isnan(got[5, :64]).all()
        # half a step of 2 top / 15 at most, the scale's rounding over fifteen codes, the result's own
        assert float((got[:5] - want[:5]).abs().max()) <= top * (1 / 15 + 15 * UNIT[dtype] + UNIT[dtype])


# ---------------------------------------------------------- slots without content ----

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_rows_that_do_not_exist_leaves_nothing_stale(d, dtype):
    """A select entry outside the rows: the slot counts, so it has content of its own: NaN, weight 0
    and its position; what lay there before does not come back."""
    c = custom(torch.randn(2, 20, 3, d, device="cuda"), torch.randn(2, 20, 3, d, device="cuda"), d, 16, dtype)
    c.weight.fill_(9.0)
    c.seq_len.fill_(10)
    c.n_pos.copy_(torch.tensor([50, 10]))
    k, v = (c.rand(2, 4, 3, d).to(KIND[dtype]) for _ in range(2))
    sel = torch.tensor([[-1, 2, 4], [3, 99, -5]], dtype=torch.int32, device="cuda")
    w = torch.full((2, 3, 4), 5.0, device="cuda")
    c.cache.append(k, v, select=sel, weight=w)
    assert c.seq_len.tolist() == [13, 13] and c.n_pos.tolist() == [53, 13] and c.cache.dropped() == 4
    rk, rv = c.cache.read(3, start=torch.full((2,), 10, dtype=torch.int32, device="cuda"))
    bad = torch.tensor([[True, False, True], [False, True, True]], device="cuda")
    for r in (rk, rv):
        assert torch.isnan(r[bad]).all() and torch.isfinite(r[~bad]).all()
    for s in range(2):
        for j in range(3):
            page, cell = int(c.table[s, (10 + j) // 16]), (10 + j) % 16
            assert c.pos[page, :, cell].tolist() == [[50, 10][s] + j] * 3
            assert c.weight[page, :, cell].tolist() == [0.0 if bad[s, j] else 5.0] * 3


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,budget,none", [([100, 90], 64, [1]), ([70, 66], 64, [0, 3]), ([5000, 300], 128, [0, 2, 7]),
                                              ([100, 100], 64, [1, 5]), ([64 + 16, 200], 64, [1, 2, 3])])
def test_evict_moves_nothing_to_pages_that_name_nothing(lens, budget, none, d):
    """Slots without a page hold their places, for nothing is stored there; the slots that are kept
    are the best of the others, and all of them are still there afterwards."""
    page, hkv = 16, 2
    c = Made(lens, hkv, d, page, spare=2)
    c.weight.copy_(torch.rand(c.weight.shape, generator=c.g, device="cuda"))
    c.table[:, none] = -1
    sink, recent = 2, 8
    table = c.table.cpu().numpy()
    before = [t.cpu().numpy().copy() for t in (c.pages, c.weight, c.pos)]
    c.cache.evict(budget, sink=sink, recent=recent)
    after = [t.cpu().numpy() for t in (c.pages, c.weight, c.pos)]
    assert c.seq_len.tolist() == [min(n, budget) for n in lens]
    for s, n in enumerate(lens):
        here = [j for j in range(n) if table[s, j // page] >= 0]
        room = [j for j in range(min(n, budget)) if table[s, j // page] >= 0]
        for h in range(hkv):
            cell = lambda arr, j: arr[table[s, j // page], h, j % page]
            rank = sorted(here, key=lambda j: (not (cell(before[2], j) < sink or cell(before[2], j) >= n - recent),
                                               -cell(before[1], j) if sink <= cell(before[2], j) < n - recent else 0.0,
                                               cell(before[2], j)))
            keep = set(rank[:len(room)]) if n > budget else set(here)
            movers = [j for j in sorted(keep) if j >= budget]
            old, new = ({name: {} for name in ("k_code", "v_code", "k_low", "v_scale")} for _ in range(2))
            for j in here:
                for store, arr in ((old, before[0]), (new, after[0])):
                    blk = O.decode_block(arr[table[s, j // page], h], page, d, "bf16")
                    for name in store:
                        store[name][j] = blk[name][j % page]
            for j in room:
                src = j if j in keep else movers.pop(0)
                assert cell(after[1], j) == cell(before[1], src) and cell(after[2], j) == cell(before[2], src), (s, h, j)
                assert all(np.array_equal(new[name][j], old[name][src]) for name in old), (s, h, j)
            assert not movers


# ------------------------------------------------------------- waits that run out ----

def test_a_stall_is_reported():
    """The flag that a bounded wait raises when it gives up, set here by hand."""
    c = Made([40, 3], 1, 64, 16)
    stalled = c.cache.workspace[16:20].view(torch.int32)
    assert c.cache.dropped() == 0
    stalled.fill_(1)
    with pytest.raises(B.OilbirdError) as e:
        c.cache.dropped()
    assert e.value.code == B.ESTALL
    stalled.zero_()
    assert c.cache.dropped() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_waits_of_a_nanosecond_end_and_leave_everything_usable(d):
    """With next to no patience the kernel may give up anywhere: it says so or its result is right,
    and the next call with the usual limit is right again."""
    c = Made([3000, 300, 1], 2, d, 32)
    q, kn, vn = (c.rand(3, 40, h, d).bfloat16() for h in (8, 2, 2))
    want, wl = c.cache.attend(q, kn, vn)
    stalled, limit = c.cache.workspace[16:20].view(torch.int32), c.cache.workspace[24:32].view(torch.int64)
    for _ in range(5):
        limit.fill_(1)
        out, lse = c.cache.attend(q, kn, vn)
        if int(stalled) == 0:
            assert torch.equal(out, want) and torch.equal(lse, wl)
        limit.zero_()
        stalled.zero_()
        out, lse = c.cache.attend(q, kn, vn)
        assert torch.equal(out, want) and torch.equal(lse, wl) and c.cache.dropped() == 0


# ------------------------------------------------------------- what the binding takes ----

def test_workspaces_are_checked():
    """What goes to the kernels as a device address is one: of the cache's device, large enough."""
    c = Made([40, 3], 1, 64, 16)
    need = B.lib().oilbird_kv_workspace_bytes(64)
    dev = c.pages.device
    over = lambda w: B.KVCache.over(c.pages, c.weight, c.pos, c.table, c.seq_len, c.n_pos, workspace=w)
    for bad in (torch.zeros(need, dtype=torch.uint8), torch.zeros(need, dtype=torch.int8, device=dev),
                torch.zeros(need - 1, dtype=torch.uint8, device=dev),
                torch.zeros(need, 2, dtype=torch.uint8, device=dev)[:, 0],
                torch.zeros(need + 16, dtype=torch.uint8, device=dev)[8:]):
        with pytest.raises(ValueError, match="workspace"):
            over(bad)
    assert over(torch.zeros(need, dtype=torch.uint8, device=dev)).dropped() == 0


def test_tensors_of_another_device_are_refused():
    c = Made([40, 3], 1, 64, 16)
    q, kn = c.rand(2, 2, 4, 64).bfloat16(), c.rand(2, 2, 1, 64).bfloat16()
    out, lse = c.cache.attend(q, kn, kn)
    ints = torch.ones(2, dtype=torch.int32, device="cuda")
    words = torch.ones(2, 2, dtype=torch.int64, device="cuda")
    calls = [lambda d: c.cache._rows(d(q), 4, 2), lambda d: c.cache._vec(d(ints), torch.int32, (2,)),
             lambda d: c.cache._lse(d(lse), 2, 4), lambda d: c.cache._mask(d(words), 2)]
    for call in calls:
        call(lambda t: t)
        with pytest.raises(AssertionError):
            call(lambda t: t.cpu())
    c.cache._index = 1                                           # as if the cache lay on the second GPU
    for call in calls:
        with pytest.raises(AssertionError):
            call(lambda t: t)


def test_tensors_that_want_a_gradient_are_refused():
    c = Made([40, 3], 1, 64, 16)
    q, kn = c.rand(2, 2, 4, 64).bfloat16().requires_grad_(), c.rand(2, 2, 1, 64).bfloat16()
    with pytest.raises(RuntimeError, match="no backward"):
        c.cache.attend(q, kn, kn)
    with pytest.raises(RuntimeError, match="no backward"):
        c.cache.append(kn, kn.clone().requires_grad_())
    with torch.no_grad():
        out, lse = c.cache.attend(q, kn, kn)
    a, b = c.cache.attend(q.detach(), kn, kn)
    assert torch.equal(out, a) and torch.equal(lse, b) and c.seq_len.tolist() == [40, 3]


def test_an_owned_cache_takes_a_workspace():
    """Caches of one stream (a model's layers) share one."""
    one = B.KVCache(2, 1, 64, 100, page_size=16)
    two = B.KVCache(2, 1, 64, 100, page_size=16, workspace=one.workspace)
    assert two.workspace.data_ptr() == one.workspace.data_ptr()
    k = torch.randn(2, 90, 1, 64, device="cuda").bfloat16()
    q = torch.randn(2, 1, 4, 64, device="cuda").bfloat16()
    for c in (one, two, one, two):
        c.append(k[:, :45], k[:, 45:])
        c.attend(q)
    a, b = one.attend(q), two.attend(q)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and one.seq_len.tolist() == [90, 90]
    with pytest.raises(ValueError, match="workspace"):
        B.KVCache(2, 1, 128, 100, workspace=one.workspace)       # smaller than heads of 128 need


def test_strides_of_dimensions_of_one_do_not_matter():
    """One sequence, one node: its row of a wider buffer whose rows are no multiple of 16 bytes."""
    c = Made([40], 1, 64, 16)
    wide = c.rand(1, 1, 4 * 64 + 2 * 64 + 4).bfloat16()
    q, kn, vn = (torch.as_strided(wide, (1, 1, h, 64), (388, 388, 64, 1), at) for h, at in ((4, 0), (1, 256), (1, 320)))
    assert q.stride()[:2] == (388, 388)
    mask = torch.ones(1, 1, dtype=torch.int64, device="cuda")
    out, lse = c.cache.attend(q, kn, vn, mask=mask)
    a, b = c.cache.attend(q.contiguous(), kn.contiguous(), vn.contiguous(), mask=mask)
    assert torch.equal(out, a) and torch.equal(lse, b)
    nodes = c.cache.weigh(q, lse, kn, mask=mask)
    c.cache.append(kn, vn, weight=nodes)
    # masks: one request's as a column, every request's alike
    m = 3
    q, kn = c.rand(1, m, 4, 64).bfloat16(), c.rand(1, m, 1, 64).bfloat16()
    column = torch.tensor([[1], [3], [5]], dtype=torch.int64, device="cuda").t()
    assert column.stride() == (1, 1)
    a, b = c.cache.attend(q, kn, kn, mask=column), c.cache.attend(q, kn, kn, mask=column.clone(memory_format=torch.contiguous_format))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c = Made([40, 3, 0], 1, 64, 16)
    q, kn = c.rand(3, m, 4, 64).bfloat16(), c.rand(3, m, 1, 64).bfloat16()
    alike = column.expand(3, m)
    assert alike.stride(0) == 0
    a, b = c.cache.attend(q, kn, kn, mask=alike), c.cache.attend(q, kn, kn, mask=alike.contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ further ranges ----

def score_error(row, k, d, scale, many):
    """How far a score may be off.  Few rows: fp32 sums of the codes' products and the offsets' (see
    test_gpu_kv).  Many: sums of 2 D products, 16 a step, each step cut off at 2^-23 of the sum; the
    exponential's argument; keys as the sum of two f16 numbers, off by 2^-13 of their group's scale
    (independent in the channels: five standard deviations) and 2^-23 of the largest element."""
    size = scale * (np.abs(row) @ np.abs(k).T).max(initial=0)
    top = np.abs(k).max(initial=0) * scale * np.abs(row).sum(-1).max()
    if not many:
        return 2.0 ** -24 * (d + 12) * (size + 2 * top) + 2.0 ** -21
    step = np.ptp(k.reshape(-1, 64), -1).max(initial=0) / 15
    return (2.0 ** -23 * (2 * d / 16 + 4) * size + 2.0 ** -21 + 5 * 2.0 ** -13 / 3 ** 0.5 * step * scale * np.sqrt((row ** 2).sum(-1)).max()
            + 2.0 ** -23 * top)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (128, "f16"), (64, "bf16"), (64, "f16")])
@pytest.mark.parametrize("m,hq", [(5, 4), (20, 8), (60, 4)])
def test_scores_of_many_rows(m, hq, d, dtype):
    """lse and out to what two-part keys give.  (f16 keys rounded once are off by three times the bound
    on the short sequences; bf16 ones, whose scales have eight bits, mostly fit f16 as they are.)"""
    lens = [1, 2, 3, 5, 40, 130, 3000, 0]
    c = Made(lens, 1, d, 64, dtype, seed=11)
    q, kn, vn = (c.rand(len(lens), m, h, d).to(KIND[dtype]) for h in (hq, 1, 1))
    scale = d ** -0.5
    for nodes in (False, True):
        mask = tree_mask(len(lens), m, 2) if nodes else None
        out, lse = c.cache.attend(q, kn if nodes else None, vn if nodes else None, mask=mask)
        for s, n in enumerate(lens):
            k, v, _ = c.dense(s, 0)
            sees = np.ones((m, n), bool)
            if nodes:
                k, v = (np.concatenate([x, f64(y, dtype)[s, :, 0]]) for x, y in ((k, kn), (v, vn)))
                sees = np.concatenate([sees, sees_of(mask, s, m, m)], 1)
            for h in range(hq):
                row = f64(q, dtype)[s, :, h]
                want, wl = O.attend(row, k, v, sees, scale)
                got, gl = f64(out, dtype)[s, :, h], lse[s, :, h].cpu().numpy().astype(np.float64)
                if len(k) == 0:
                    assert np.all(got == 0) and np.all(gl == -np.inf)
                    continue
                e, vmax = score_error(row, k, d, scale, True), np.abs(v).max()
                assert np.all(np.abs(gl - wl) <= e + 2.0 ** -22 * (np.abs(wl) + 1)), (s, h, np.abs(gl - wl).max(), e)
                assert np.all(np.abs(got - want) <= UNIT[dtype] * np.abs(want) + (2 * e + 2 * 2.0 ** -11) * vmax + len(k) * 2.0 ** -32 * 2 * vmax)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,hq", [(1, 8), (2, 8), (20, 8)])
def test_a_long_sequence(m, hq, dtype):
    """131,085 slots.  Roundings of different slots are independent, so eight standard deviations of
    their sum are 8 |p| (2-norm) times one slot's: R 2^-11 and 2^-11 max |v| for the operands, 2 e max |v| for
    the score.  Beside them 2^-31 R for each slot (operands below f16's normal range) and 2^-23 R for
    each of 64 sums that the tensor cores cut off."""
    n, d = 131085, 128
    c = Made([n], 1, d, 64, dtype, seed=8, v_gain=1.0)
    q = (c.rand(1, m, hq, d) * 2).to(KIND[dtype])
    out, lse = c.cache.attend(q)
    k, v, _ = c.dense(0, 0)
    vmax, rng = np.abs(v).max(), np.ptp(v.reshape(-1, 64), -1).max()
    for h in range(hq):
        row = f64(q, dtype)[0, :, h]
        x = (row @ k.T) * d ** -0.5
        p = np.exp(x - x.max(-1, keepdims=True))
        total = p.sum(-1, keepdims=True)
        wl = np.log(total[:, 0]) + x.max(-1)
        p /= total
        want, got, gl = p @ v, f64(out, dtype)[0, :, h], lse[0, :, h].cpu().numpy().astype(np.float64)
        e = score_error(row, k, d, d ** -0.5, m * hq > 16)
        norm = np.sqrt((p ** 2).sum(-1, keepdims=True))
        tol = UNIT[dtype] * np.abs(want) + 8 * norm * (2.0 ** -11 * (rng + vmax) + 2 * e * vmax) + n * 2.0 ** -31 * rng + 64 * 2.0 ** -23 * rng
        assert np.all(np.abs(got - want) <= tol), (h, np.abs(got - want).max(), tol.min(), np.abs(want).max())
        assert np.all(np.abs(gl - wl) <= e + 2.0 ** -22 * (np.abs(wl) + 1))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,hq,hkv", [(16, 1, 1), (8, 2, 1), (5, 3, 1), (9, 1, 1), (16, 2, 2), (17, 1, 1), (3, 12, 2)])
def test_rows_up_to_the_change_of_kernels(m, hq, hkv, dtype):
    c = Made([0, 1, 63, 200, 900], hkv, 128, 64, dtype)
    q, kn, vn = (c.rand(5, m, h, 128).to(KIND[dtype]) for h in (hq, hkv, hkv))
    mask = tree_mask(5, m, 6)
    n_new = torch.tensor([m, 0, m - 1, 1, m], dtype=torch.int32, device="cuda")
    out, lse = c.cache.attend(q, kn, vn, mask=mask, n_new=n_new)
    check_attend(c, q, kn, vn, mask, n_new, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("lens", [[700, 1300, 129], [4000]])
def test_f16_trees_over_long_heads(lens):
    c = Made(lens, 2, 128, 32, "f16")
    n = len(lens)
    q, kn, vn = (c.rand(n, 60, h, 128).half() for h in (8, 2, 2))
    mask = tree_mask(n, 60, 6)
    out, lse = c.cache.attend(q, kn, vn, mask=mask)
    check_attend(c, q, kn, vn, mask, None, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("n_seq", [300, 1024])
def test_as_many_sequences_as_there_may_be(n_seq):
    """attend (both kernels), weigh, append and evict over all of them."""
    lens = [(7 * i) % 23 for i in range(n_seq)]
    c = Made(lens, 1, 64, 16, "bf16", max_pages=2)
    for m, hq in ((1, 2), (6, 4)):
        q, kn, vn = (c.rand(n_seq, m, h, 64).bfloat16() for h in (hq, 1, 1))
        out, lse = c.cache.attend(q, kn, vn)
        check_attend(c, q, kn, vn, None, None, out, lse, 64 ** -0.5)
        c.weight.zero_()
        nodes = c.cache.weigh(q, lse, kn)
        page, hold = c.table.clamp(min=0).long(), (c.table >= 0)
        got = (c.weight[page, 0].sum(-1) * hold).sum(-1) + nodes.sum((1, 2))
        assert torch.allclose(got, torch.full_like(got, float(m * hq)), rtol=1e-4)    # a softmax adds up to 1
    weight = c.weight[:, 0].cpu().numpy()
    table = c.table.cpu().numpy()
    c.cache.evict(9, sink=1, recent=2)
    after = c.weight[:, 0].cpu().numpy()
    assert c.seq_len.tolist() == [min(n, 9) for n in lens]
    for s, n in enumerate(lens):
        if n > 9:
            at = np.arange(n)
            w = weight[table[s, at // 16], at % 16]
            src = O.evict(w, at, n, 9, 1, 2)
            assert np.array_equal(after[table[s, at[:9] // 16], at[:9] % 16], w[src])
    k = c.rand(n_seq, 2, 1, 64).bfloat16()
    before = c.seq_len.tolist()
    c.cache.append(k, k, n_new=torch.arange(n_seq, device="cuda").int() % 3)
    room = [16 if 0 < n <= 16 else 0 if n == 0 else 32 for n in lens]
    lost = sum(max(0, b + i % 3 - r) for i, (b, r) in enumerate(zip(before, room)))
    assert c.seq_len.tolist() == [b + i % 3 for i, b in enumerate(before)] and c.cache.dropped() == lost


@pytest.mark.parametrize("m,hq", [(1, 4), (3, 4), (30, 4)])
def test_a_negative_scale_is_the_queries_sign(m, hq):
    c = Made([300, 0, 40], 1, 128, 64)
    q, kn, vn = (c.rand(3, m, h, 128).bfloat16() for h in (hq, 1, 1))
    a, b = c.cache.attend(q, kn, vn, scale=-0.1), c.cache.attend(-q, kn, vn, scale=0.1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.weight.zero_()
    na = c.cache.weigh(q, a[1], kn, scale=-0.1)
    wa = c.weight.clone()
    c.weight.zero_()
    nb = c.cache.weigh(-q, b[1], kn, scale=0.1)
    assert torch.equal(na, nb) and torch.equal(wa, c.weight) and float(wa.sum()) > 0


# ------------------------------------------------------------------ large budgets ----

def test_budgets_beyond_32_bits_cut_nothing():
    c = Made([40, 7], 1, 64, 16)
    for budget in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 40):
        c.cache.evict(budget)
        c.cache.evict(budget, sink=2 ** 30, recent=3)
        assert c.seq_len.tolist() == [40, 7]
    for sink, recent in ((2 ** 32, 0), (0, 2 ** 32), (-2 ** 32, 0)):
        with pytest.raises(B.OilbirdError):
            c.cache.evict(30, sink=sink, recent=recent)
    c.cache.evict(8)
    assert c.seq_len.tolist() == [8, 7]
