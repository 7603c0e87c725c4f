"""The 4-bit key/value cache on the GPU against its 64-bit implementation.

Tolerances.  u = 2^-8 (bf16) or 2^-11 (f16) is the unit roundoff of a result's type; every
output gets u * |result| for its last rounding.  What comes before it:
  scores      fp32 sums of D products: 2^-24 (D + 12) times the sum of the products' magnitudes
              (codes and offsets apart), called S below, and 2^-21 for the exponential; so a
              probability is off by the factor 1 + e, e = 2^-24 (D + 12) S + 2^-21.
              Where a call multiplies more than 16 rows with each key head, keys may be rounded to
              f16 first: eight standard deviations of that, 8 * 2^-11 / sqrt(3) |q k| (2-norm over
              the channels), join e.
  values      a probability times a scale is rounded to f16: 2^-11 of each term, and where it is
              small 2^-25 in units of the largest scale's power of two, times a code of 15: for N
              slots R (2^-11 + N 2^-24), R = the largest 15 * scale; f16 values: 2^-11 of max |v|.
  together    |out error| <= u |out| + R (2^-11 + N 2^-24) + (2 e + 2^-11) max |v|,
              |lse error| <= e + 2^-22 (|lse| + 1).
"""
import numpy as np
import pytest
import torch

from oracle import kv as O
from paper_2608_03839_b200 import binding as B

pytestmark = pytest.mark.gpu

KIND = {"bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def f64(t, dtype):
    return O.from16(bits(t), dtype)


class Made:
    """A cache with scattered pages whose unused slots and pages hold NaN, filled by append."""

    def __init__(self, lens, hkv=2, d=128, page=64, dtype="bf16", seed=0, v_gain=0.5, spare=2, max_pages=None):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.hkv, self.d, self.page, self.dtype = list(lens), hkv, d, page, dtype
        n_seq, need = len(lens), [-(-n // page) for n in lens]
        most = max(1, max(need)) if max_pages is None else max_pages
        n_pages = sum(need) + spare
        table = torch.full((n_seq, most), -1, dtype=torch.int32)
        order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int()
        at = 0
        for i, c in enumerate(need):
            table[i, :c] = order[at:at + c]
            at += c
        block = B.lib().oilbird_kv_block_bytes(d, page)
        self.pages = torch.full((n_pages, hkv, block), 0xFF, dtype=torch.uint8, device="cuda")
        self.weight = torch.full((n_pages, hkv, page), float("nan"), device="cuda")
        self.pos = torch.full((n_pages, hkv, page), -7, dtype=torch.int32, device="cuda")
        self.table = table.cuda()
        self.seq_len = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
        self.n_pos = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
        self.cache = B.KVCache.over(self.pages, self.weight, self.pos, self.table, self.seq_len, self.n_pos,
                                    dtype=KIND[dtype])
        m = max(lens)
        if m:
            lean = self.rand(1, 1, hkv, d) * 2
            self.k_in = (self.rand(n_seq, m, hkv, d) + lean).to(KIND[dtype])
            self.v_in = (self.rand(n_seq, m, hkv, d) * v_gain).to(KIND[dtype])
            self.cache.append(self.k_in, self.v_in, n_new=torch.tensor(lens, dtype=torch.int32, device="cuda"))

    def rand(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def dense(self, s, h):
        n = int(self.seq_len[s])
        return O.gather(self.pages.cpu().numpy(), self.table[s].cpu().numpy(), n, h, self.page, self.d, self.dtype)


def tree_mask(n_seq, m, seed):
    rng = np.random.default_rng(seed)
    out = np.zeros((n_seq, m), np.uint64)
    for s in range(n_seq):
        for i in range(m):
            out[s, i] = np.uint64(1) << np.uint64(i)
            if i:
                out[s, i] |= out[s, rng.integers(0, i)]
    return torch.from_numpy(out.view(np.int64)).cuda()


def sees_of(mask, s, nodes, m):
    words = mask[s].cpu().numpy().view(np.uint64) if mask is not None else [(2 << i) - 1 for i in range(m)]
    return np.array([[bool(int(words[i]) >> j & 1) for j in range(nodes)] for i in range(m)],
                    dtype=bool).reshape(m, nodes)


def check_attend(c, q, kn, vn, mask, n_new, out, lse, scale):
    n_seq, m, hq, d = q.shape
    group, dt = hq // c.hkv, c.dtype
    qf, of = f64(q, dt), f64(out, dt)
    lf = lse.cpu().numpy().astype(np.float64)
    counts = [m] * n_seq if n_new is None else n_new.cpu().tolist()
    for s in range(n_seq):
        nodes = max(0, min(m, counts[s]))
        for h in range(c.hkv):
            k, v, has = c.dense(s, h)
            sees = np.repeat(has[None, :], m, 0)
            n_nodes = 0
            if kn is not None:
                n_nodes = nodes
                k = np.concatenate([k, f64(kn, dt)[s, :nodes, h]])
                v = np.concatenate([v, f64(vn, dt)[s, :nodes, h]])
                sees = np.concatenate([sees, sees_of(mask, s, nodes, m)], 1)
            sees[nodes:] = False
            k, v = np.where(sees.any(0)[:, None], k, 0), np.where(sees.any(0)[:, None], v, 0)
            vmax = np.abs(v).max(initial=0)
            rng = 2 * vmax                       # hi - lo of a group, at most
            for g in range(group):
                row = qf[s, :, h * group + g]
                want, wlse = O.attend(row, k, v, sees, scale)
                mag = scale * (np.abs(row) @ (np.abs(k).T + 2 * np.abs(k).max(initial=0))).max(initial=0)
                e = 2.0 ** -24 * (d + 12) * mag + 2.0 ** -21
                if m * group > 16:
                    e += 8 * 2.0 ** -11 / 3 ** 0.5 * scale * np.sqrt((row ** 2 @ (k ** 2).T).max(initial=0))
                got, glse = of[s, :, h * group + g], lf[s, :, h * group + g]
                tol = UNIT[dt] * np.abs(want) + rng * (2.0 ** -11 + len(k) * 2.0 ** -24) + (2 * e + 2.0 ** -11) * vmax
                assert np.all(np.abs(got - want) <= tol), (s, h, g, np.abs(got - want).max(), tol.min())
                none = ~sees.any(1)
                assert np.all(got[none] == 0) and np.all(glse[none] == -np.inf)
                assert np.all(np.abs(glse - wlse)[~none] <= e + 2.0 ** -22 * (np.abs(wlse[~none]) + 1))


def attend_case(lens, m, hq=8, hkv=2, d=128, page=64, dtype="bf16", ragged=True, tree=True, nodes_kv=True, seed=1,
                **more):
    c = Made(lens, hkv, d, page, dtype, seed, **more)
    n_seq = len(lens)
    both = c.rand(n_seq, m, hq + 2 * hkv, d).to(KIND[dtype])
    q, kn, vn = both[:, :, :hq], both[:, :, hq:hq + hkv], both[:, :, hq + hkv:]
    mask = tree_mask(n_seq, m, seed) if tree else None
    n_new = None
    if ragged:
        n_new = torch.tensor([max(0, m - 3 * i) for i in range(n_seq)], dtype=torch.int32, device="cuda")
    if not nodes_kv:
        kn = vn = None
    out, lse = c.cache.attend(q, kn, vn, mask=mask if nodes_kv else None, n_new=n_new)
    check_attend(c, q, kn, vn, mask, n_new, out, lse, d ** -0.5)
    return c, q, kn, vn, mask, n_new, out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,page", [(128, 64), (128, 16), (64, 32), (64, 64)])
@pytest.mark.parametrize("m,hq,hkv", [(1, 8, 2), (1, 2, 2), (7, 6, 2), (33, 4, 1), (64, 8, 1), (2, 16, 1)])
def test_attend_lengths_around_tiles(dtype, d, page, m, hq, hkv):
    attend_case([0, 1, 15, 16, 17, 31, 32, 33, 64, 65, 130], m, hq, hkv, d, page, dtype)


@pytest.mark.parametrize("m", [1, 3, 60])
def test_attend_long_and_short_together(m):
    """One long sequence among short ones: its items are cut between blocks."""
    attend_case([9000, 3, 0, 700, 2049], m, 8, 2, ragged=False)


def test_attend_many_sequences():
    attend_case([(37 * i) % 200 for i in range(70)], 1, 4, 4, 64, 16, "f16", ragged=False)


@pytest.mark.parametrize("m,hq", [(1, 4), (12, 16)])
def test_attend_cache_alone(m, hq):
    """Without new keys: every node sees the slots only; an empty sequence gives nothing."""
    attend_case([0, 5, 100, 640], m, hq, 2, nodes_kv=False, ragged=False, tree=False)


@pytest.mark.parametrize("m,hq", [(1, 4), (20, 16)])
def test_attend_masks_that_leave_rows_empty(m, hq):
    c = Made([0, 0, 40], 2, 128)
    q, kn, vn = (c.rand(3, m, h, 128).bfloat16() for h in (hq, 2, 2))
    mask = torch.zeros(3, m, dtype=torch.int64, device="cuda")
    mask[1, m - 1] = 1                      # a row that sees node 0 alone
    out, lse = c.cache.attend(q, kn, vn, mask=mask)
    check_attend(c, q, kn, vn, mask, None, out, lse, 128 ** -0.5)
    assert torch.all(out[0] == 0) and torch.all(lse[0] == float("-inf"))


@pytest.mark.parametrize("m,hq", [(1, 4), (24, 8)])
def test_attend_pages_that_name_nothing(m, hq):
    c = Made([200, 64, 130], 2, 128, 32)
    c.table[0, 1], c.table[0, 6], c.table[1, :] = -1, 1 << 30, -5
    q = c.rand(3, m, hq, 128).bfloat16()
    out, lse = c.cache.attend(q)
    check_attend(c, q, None, None, None, None, out, lse, 128 ** -0.5)
    assert torch.all(out[1] == 0)


@pytest.mark.parametrize("dtype,gain", [("bf16", 1e-30), ("bf16", 1e25), ("f16", 3e-4), ("f16", 9e3)])
@pytest.mark.parametrize("m,hq", [(1, 4), (30, 4)])
def test_attend_values_of_any_size(dtype, gain, m, hq):
    """Values far from one: the products' 16-bit operands are scaled by powers of two."""
    c = Made([300, 17], 1, 128, 64, dtype, v_gain=gain)
    q = c.rand(2, m, hq, 128).to(KIND[dtype])
    out, lse = c.cache.attend(q)
    check_attend(c, q, None, None, None, None, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("m,hq", [(1, 4), (30, 4)])
def test_attend_large_and_small_queries(m, hq):
    c = Made([300, 17], 1, 64, 64, "bf16")
    q = (c.rand(2, m, hq, 64) * 1e20).bfloat16()
    out, lse = c.cache.attend(q, scale=1e-21)
    check_attend(c, q, None, None, None, None, out, lse, 1e-21)
    q = (c.rand(2, m, hq, 64) * 1e-25).bfloat16()
    out, lse = c.cache.attend(q, scale=1e25)
    check_attend(c, q, None, None, None, None, out, lse, 1e25)


@pytest.mark.parametrize("m,hq", [(1, 4), (40, 4)])
def test_attend_a_nan_reaches_only_its_rows_and_channels(m, hq):
    c = Made([100, 100], 1, 128, 64)
    k, v = c.k_in[:, :1].clone(), c.v_in[:, :1].clone()
    v[0, 0, 0, 70] = float("inf")
    c2 = Made([0, 0], 1, 128, 64, max_pages=2, spare=4)
    c2.table.copy_(torch.tensor([[0, 1], [2, 3]]))
    c2.cache.append(k, v)
    q = c2.rand(2, m, hq, 128).bfloat16()
    out, lse = c2.cache.attend(q)
    assert torch.isnan(out[0, :, :, 64:]).all() and torch.isfinite(out[0, :, :, :64]).all()
    assert torch.isfinite(out[1]).all() and torch.isfinite(lse).all()
    q[1, 0, 0, 5] = float("nan")
    out, lse = c2.cache.attend(q)
    assert torch.isnan(out[1, 0, 0]).all() and torch.isnan(lse[1, 0, 0])
    assert torch.isfinite(out[1, 0, 1:]).all() and torch.isfinite(out[1, 1:]).all()


def test_attend_strides_and_given_outputs():
    c = Made([90, 33], 2, 64, 16, "f16")
    q = c.rand(8, 3, 2, 64).half().permute(2, 1, 0, 3)          # [2, 3, 8, 64], heads outermost
    out = torch.zeros(3, 2, 8, 80, dtype=torch.float16, device="cuda")[..., :64].transpose(0, 1)
    lse = torch.zeros(8, 2, 3, device="cuda").permute(1, 2, 0)
    got, l2 = c.cache.attend(q, out=out, lse=lse)
    assert got is out and l2 is lse
    check_attend(c, q, None, None, None, None, out, lse, 64 ** -0.5)


@pytest.mark.parametrize("m,hq", [(1, 8), (48, 8)])
def test_attend_repeats_bit_for_bit(m, hq):
    """Splits and joins are a function of the lengths alone; the workspace carries nothing over."""
    c = Made([5000, 1, 800], 2, 128, 64)
    other = Made([64, 900, 0], 2, 128, 64, seed=5)
    q = c.rand(3, m, hq, 128).bfloat16()
    a, la = c.cache.attend(q)
    shared = B.KVCache.over(other.pages, other.weight, other.pos, other.table, other.seq_len, other.n_pos,
                            workspace=c.cache.workspace)
    for _ in range(5):
        shared.attend(q)
        b, lb = c.cache.attend(q)
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_long_cache_offsets_pass_32_bits():
    hkv, d, page = 8, 128, 64
    block = B.lib().oilbird_kv_block_bytes(d, page)
    n_pages = (5 << 30) // (block * hkv)
    pages = torch.empty(n_pages * hkv * block, dtype=torch.uint8, device="cuda")
    c = Made([0, 0], hkv, d, page, max_pages=3)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7], [n_pages - 2, n_pages // 2, 0]], dtype=torch.int32).cuda()
    weight = torch.zeros(n_pages, hkv, page, device="cuda")
    pos = torch.zeros(n_pages, hkv, page, dtype=torch.int32, device="cuda")
    cache = B.KVCache.over(pages, weight, pos, table, c.seq_len, c.n_pos)
    k, v = c.rand(2, 150, hkv, d).bfloat16(), c.rand(2, 150, hkv, d).bfloat16()
    cache.append(k, v)
    q = c.rand(2, 2, 16, d).bfloat16()
    out, lse = cache.attend(q)
    view = pages.view(n_pages, hkv, block)
    c.pages = torch.stack([view[int(t)] for t in table.flatten()])
    c.table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    check_attend(c, q, None, None, None, None, out, lse, d ** -0.5)
    rk, rv = cache.read(150)
    assert float((rk.float() - k.float()).abs().max()) < 0.3 and float((rv.float() - v.float()).abs().max()) < 0.3


def test_on_another_stream_and_in_a_graph():
    c = Made([500, 77], 2, 128, 64)
    q = c.rand(2, 4, 8, 128).bfloat16()
    kn, vn = c.rand(2, 4, 2, 128).bfloat16(), c.rand(2, 4, 2, 128).bfloat16()
    want, wl = c.cache.attend(q, kn, vn)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, gl = c.cache.attend(q, kn, vn, stream=side)
    side.synchronize()
    assert torch.equal(want, got) and torch.equal(wl, gl)
    out, lse = torch.zeros_like(want), torch.zeros_like(wl)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.attend(q, kn, vn, out=out, lse=lse)
    for _ in range(3):
        out.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want, out) and torch.equal(wl, lse)


# ------------------------------------------------------------------------- append / read ----

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,page", [(128, 64), (128, 16), (64, 32)])
def test_append_stores_the_format(dtype, d, page):
    """Meta: correctly rounded.  Codes: equal but where the quotient is within 2^-20 of a tie."""
    c = Made([70, 0, 1, 64, 33], 3, d, page, dtype)
    host = c.pages.cpu().numpy()
    table, slots = c.table.cpu().numpy(), 0
    for s, n in enumerate(c.lens):
        for j in range(n):
            for h in range(c.hkv):
                blk = O.decode_block(host[table[s, j // page], h], page, d, dtype) if j % page == 0 or h >= 0 else None
                for name, x in (("k", c.k_in), ("v", c.v_in)):
                    row = f64(x[s, j, h], dtype).reshape(-1, 64)
                    code, scale, low = O.quantise(row, dtype)
                    got_scale = O.from16(blk[name + "_scale"][j % page], dtype)
                    assert np.array_equal(O.from16(blk[name + "_low"][j % page], dtype), low)
                    exact = (row.max(-1) - row.min(-1)) / 15
                    assert np.all(np.abs(got_scale - exact) <= UNIT[dtype] * exact * (1 + 2.0 ** -12))
                    quo = (row - low[:, None]) / got_scale[:, None]
                    tie = np.abs(quo - np.floor(quo) - 0.5) < 2.0 ** -20
                    got = blk[name + "_code"][j % page].reshape(-1, 64)
                    assert np.all((got == np.clip(np.rint(quo), 0, 15)) | tie)
                slots += 1
            if slots > 60:
                break
    assert c.seq_len.tolist() == c.lens and c.n_pos.tolist() == c.lens


def test_append_select_counts_weights_and_positions():
    c = Made([10, 0, 63], 2, 128, 64, max_pages=2, spare=6)
    c.table.copy_(torch.tensor([[4, 5], [0, 7], [6, 2]]))
    c.seq_len.copy_(torch.tensor([10, 0, 63]))
    c.n_pos.copy_(torch.tensor([100, 5, 63]))
    k, v = c.rand(3, 9, 2, 128).bfloat16(), c.rand(3, 9, 2, 128).bfloat16()
    w = torch.rand(3, 2, 9, device="cuda")
    sel = torch.tensor([[8, 0, 3, 3], [1, 2, 5, 7], [7, 6, 5, 4]], dtype=torch.int32, device="cuda")
    n = torch.tensor([3, 0, 4], dtype=torch.int32, device="cuda")
    c.cache.append(k, v, n_new=n, select=sel, weight=w)
    assert c.seq_len.tolist() == [13, 0, 67] and c.n_pos.tolist() == [103, 5, 67]
    rk, rv = c.cache.read(4, start=torch.tensor([10, 0, 63], dtype=torch.int32, device="cuda"))
    for s, cnt in enumerate([3, 0, 4]):
        for j in range(4):
            if j >= cnt:
                assert torch.all(rk[s, j] == 0) and torch.all(rv[s, j] == 0)
                continue
            src = int(sel[s, j])
            for got, x in ((rk, k), (rv, v)):
                step = (x[s, src].float().unflatten(-1, (2, 64)).amax(-1) - x[s, src].float().unflatten(-1, (2, 64)).amin(-1)) / 15
                off = (got[s, j].float() - x[s, src].float()).unflatten(-1, (2, 64)).abs().amax(-1)
                assert torch.all(off <= step * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -8 * x[s, src].float().abs().max())
            slot = [10, 0, 63][s] + j
            p, cell = int(c.table[s, slot // 64]), slot % 64
            assert torch.equal(c.weight[p, :, cell], w[s, :, src])
            assert c.pos[p, :, cell].tolist() == [[100, 5, 63][s] + j] * 2


def test_read_gives_the_stored_values():
    """One rounding of scale * code + low to 16 bits; a fused multiply-add may differ from the
    64-bit value's rounding by nothing but a double rounding, one unit in the last place."""
    for dtype in ("bf16", "f16"):
        c = Made([70, 3, 0], 2, 64, 16, dtype)
        k, v = c.cache.read(75)
        for s in range(3):
            for h in range(2):
                dk, dv, _ = c.dense(s, h)
                n = c.lens[s]
                for got, want in ((k, dk), (v, dv)):
                    x = f64(got[s, :, h], dtype)
                    assert np.all(x[n:] == 0)
                    assert np.all(np.abs(x[:n] - want) <= UNIT[dtype] * np.abs(want) * (1 + 2.0 ** -10) + 2.0 ** -25)


def test_append_constants_extremes_and_non_finite_groups():
    c = Made([0], 1, 128, 16, max_pages=1)
    c.table.zero_()
    big = 3.0e38
    k = torch.zeros(1, 6, 1, 128, device="cuda")
    k[0, 0] = 2.5                                                # constant group
    k[0, 1, 0, 0], k[0, 1, 0, 1] = big, -big                     # the range itself overflows fp32
    k[0, 2, 0, 64] = float("nan")
    k[0, 3, 0, 3] = float("-inf")
    k[0, 4, 0, 1] = 1e-40                                        # a scale that rounds to nothing
    k = k.bfloat16()
    c.cache.append(k, k)
    rk, rv = c.cache.read(6)
    for r in (rk, rv):
        r = r.float()
        assert torch.all(r[0, 0] == 2.5)
        assert abs(float(r[0, 1, 0, 0]) / big - 1) < 0.02 and abs(float(r[0, 1, 0, 1]) / -big - 1) < 0.02
        assert torch.isfinite(r[0, 1]).all() and float(r[0, 1, 0, 2].abs()) <= 2 * big / 15 * 0.52
        assert torch.isnan(r[0, 2, 0, 64:]).all() and torch.all(r[0, 2, 0, :64] == 0)
        assert torch.isnan(r[0, 3, 0, :64]).all() and torch.all(r[0, 3, 0, 64:] == 0)
        assert torch.all(r[0, 4].abs() < 2e-40) and torch.all(r[0, 5] == 0)


def test_append_past_the_table_is_dropped_and_counted():
    c = Made([30, 5], 2, 64, 16, max_pages=3)
    before = c.pages.clone()
    c.table[1, 0] = -1
    k = c.rand(2, 40, 2, 64).bfloat16()
    c.cache.append(k, k, n_new=torch.tensor([40, 3], dtype=torch.int32, device="cuda"))
    # sequence 0: pages 0 and 1 exist, so slots 30 and 31 fit; sequence 1 has no page at all
    assert c.seq_len.tolist() == [48, 8]
    assert c.cache.dropped() == 38 + 3
    changed = (c.pages != before).any(-1).any(-1).nonzero().flatten().tolist()
    assert changed == [int(c.table[0, 1])]
    c.cache.append(k, k, select=torch.full((2, 1), 99, dtype=torch.int32, device="cuda"))
    assert c.cache.dropped() == 38 + 3 + 2


# --------------------------------------------------------------------------------- weigh ----

@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 64), ("f16", 128, 16), ("bf16", 64, 32)])
@pytest.mark.parametrize("m,hq,hkv,accept", [(1, 8, 2, None), (13, 6, 2, 4), (64, 8, 1, None), (60, 8, 2, 7), (5, 40, 2, None)])
def test_weigh(dtype, d, page, m, hq, hkv, accept):
    """Tolerance: a term's factor is 1 + e with e as for attend (no f16 keys here) and the lse's
    rounding, 2^-22 (|lse| + 1); the sum over r rows adds 2^-23 r, the slot's sum 2^-23 of itself."""
    lens = [0, 1, 33, 64, 300, 2000]
    c = Made(lens, hkv, d, page, dtype, seed=3)
    n_seq, group = len(lens), hq // hkv
    q, kn = c.rand(n_seq, m, hq, d).to(KIND[dtype]), c.rand(n_seq, m, hkv, d).to(KIND[dtype])
    mask = tree_mask(n_seq, m, 9)
    n_new = torch.tensor([max(0, m - i) for i in range(n_seq)], dtype=torch.int32, device="cuda")
    rw = None
    if accept is not None:
        rw = torch.zeros(n_seq, m, device="cuda")
        for s in range(n_seq):
            rw[s, torch.randperm(m, generator=c.g, device="cuda")[:accept]] = 0.25 + s
    scale = d ** -0.5
    _, lse = c.cache.attend(q, kn, kn, mask=mask, n_new=n_new)
    lse = lse.transpose(1, 2).contiguous().transpose(1, 2)       # other strides
    c.weight.copy_(torch.rand(c.weight.shape, generator=c.g, device="cuda"))
    before = c.weight.clone()
    nodes_w = c.cache.weigh(q, lse, kn, mask=mask, n_new=n_new, row_weight=rw)
    untouched = torch.ones_like(before, dtype=torch.bool)
    for s in range(n_seq):
        nodes = int(n_new[s])
        for h in range(hkv):
            k, _, _ = c.dense(s, h)
            keys = np.concatenate([k, f64(kn, dtype)[s, :nodes, h]])
            sees = np.concatenate([np.ones((m, len(k)), bool), sees_of(mask, s, nodes, m)], 1)[:nodes]
            got = np.zeros(len(keys))
            e = 0.0
            for g in range(group):
                row, l = f64(q, dtype)[s, :nodes, h * group + g], lse[s, :nodes, h * group + g].cpu().numpy().astype(np.float64)
                r = np.ones(nodes) if rw is None else rw[s, :nodes].cpu().numpy().astype(np.float64)
                x = (row @ keys.T) * scale
                ok = sees & np.isfinite(l)[:, None]
                got += (np.where(ok, np.exp(np.where(ok, x - l[:, None], 0)), 0) * r[:, None]).sum(0)
                mag = scale * (np.abs(row) @ (np.abs(keys).T + 2 * np.abs(keys).max(initial=0))).max(initial=0)
                lmax = np.abs(l[np.isfinite(l)]).max(initial=0)
                e = max(e, 2.0 ** -24 * (d + 12) * mag + 2.0 ** -21 + 2.0 ** -22 * (lmax + 1) + 2.0 ** -23 * nodes * group)
            n = len(k)
            at = np.arange(n)
            p = c.table[s].cpu().numpy()[at // page]
            w0 = before[p, h, at % page].cpu().numpy().astype(np.float64)
            w1 = c.weight[p, h, at % page].cpu().numpy().astype(np.float64)
            untouched[p, h, at % page] = False
            assert np.all(np.abs(w1 - w0 - got[:n]) <= e * got[:n] + 2.0 ** -23 * np.abs(w0 + got[:n]))
            nw = nodes_w[s, h].cpu().numpy().astype(np.float64)
            assert np.all(nw[nodes:] == 0)
            assert np.all(np.abs(nw[:nodes] - got[n:]) <= e * got[n:] + 2.0 ** -23 * got[n:])
    assert torch.equal(c.weight[untouched], before[untouched])


def test_weigh_probabilities_of_a_row_sum_to_one():
    c = Made([777, 5], 2, 128, 32)
    q, kn = c.rand(2, 6, 8, 128).bfloat16(), c.rand(2, 6, 2, 128).bfloat16()
    c.weight.zero_()
    _, lse = c.cache.attend(q, kn, kn)
    nodes = c.cache.weigh(q, lse, kn)
    total = [float(c.weight[c.table[s][c.table[s] >= 0].long()].sum() + nodes[s].sum()) for s in range(2)]
    assert np.allclose(total, 6 * 8, rtol=1e-4)
    before = c.weight.clone()
    assert c.cache.weigh(q, lse, row_weight=torch.zeros(2, 6, device="cuda")) is None
    assert torch.equal(before, c.weight)


# --------------------------------------------------------------------------------- evict ----

def evict_case(lens, budget, sink, recent, weights, d=128, page=32, dtype="bf16", hkv=2, pos=None, seed=2):
    c = Made(lens, hkv, d, page, dtype, seed)
    c.weight.copy_(weights(c, c.weight.shape))
    if pos is not None:
        c.pos.copy_(pos(c, c.pos.shape))
    pages, weight, where, npos = (t.clone().cpu().numpy() for t in (c.pages, c.weight, c.pos, c.n_pos))
    table = c.table.cpu().numpy()
    c.cache.evict(budget, sink=sink, recent=recent)
    after, w2, p2 = c.pages.cpu().numpy(), c.weight.cpu().numpy(), c.pos.cpu().numpy()
    assert c.seq_len.tolist() == [min(n, budget) for n in lens]
    for s, n in enumerate(lens):
        at = np.arange(n)
        p, cell = table[s, at // page], at % page
        for h in range(hkv):
            src = np.arange(n) if n <= budget else O.evict(weight[p, h, cell], where[p, h, cell], int(npos[s]), budget, sink, recent)
            assert np.array_equal(w2[p, h, cell][:len(src)], weight[p, h, cell][src], equal_nan=True)
            assert np.array_equal(p2[p, h, cell][:len(src)], where[p, h, cell][src])
            old = [O.decode_block(pages[x, h], page, d, dtype) for x in table[s] if x >= 0]
            new = [O.decode_block(after[x, h], page, d, dtype) for x in table[s] if x >= 0]
            for name in ("k_code", "v_code", "k_scale", "k_low", "v_scale", "v_low"):
                if not old:
                    continue
                a, b = np.concatenate([o[name] for o in old]), np.concatenate([o[name] for o in new])
                assert np.array_equal(b[:len(src)], a[src]), (s, h, name)
    return c


def heavy(c, shape):
    return (torch.randn(shape, generator=c.g, device="cuda") * 2).exp()


@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 0), (31, 4, 8), (32, 0, 32), (33, 2, 0), (100, 4, 50), (1000, 0, 0)])
@pytest.mark.parametrize("d,page", [(128, 32), (64, 16), (128, 64)])
def test_evict(budget, sink, recent, d, page):
    evict_case([0, 1, 31, 32, 33, 64, 101, 300, 2500], budget, sink, recent, heavy, d, page)


@pytest.mark.parametrize("weights", [
    lambda c, s: torch.zeros(s, device="cuda"),
    lambda c, s: torch.randint(0, 3, s, generator=c.g, device="cuda").float(),
    lambda c, s: -torch.randint(0, 2, s, generator=c.g, device="cuda").float(),
    lambda c, s: torch.where(torch.rand(s, generator=c.g, device="cuda") < 0.5, float("nan"), 1.0),
    lambda c, s: torch.where(torch.rand(s, generator=c.g, device="cuda") < 0.1, float("inf"), 0.5),
    lambda c, s: torch.full(s, float("nan"), device="cuda"),
])
@pytest.mark.parametrize("shuffled", [False, True])
def test_evict_ties_and_odd_weights(weights, shuffled):
    pos = (lambda c, s: torch.randperm(int(np.prod(s)), generator=c.g, device="cuda").int().view(s)) if shuffled else None
    evict_case([70, 500, 64], 64, 3, 9, weights, pos=pos)


@pytest.mark.parametrize("most,budget", [(5000, 700), (9000, 8999), (17000, 33), (40000, 4096)])
def test_evict_sequences_shared_by_several_blocks(most, budget):
    """Long sequences are handled by two to eight blocks; ties and moves cross between them."""
    evict_case([most, most // 3, budget, budget + 1], budget, 3, budget // 3,
               lambda c, s: (torch.rand(s, generator=c.g, device="cuda") < 0.3) * torch.randint(0, 50, s, generator=c.g, device="cuda").float(),
               d=64, page=64, hkv=1)


@pytest.mark.parametrize("over", [1, 2, 15, 16, 17, 18])
@pytest.mark.parametrize("kind", ["weights", "ties", "all stay", "equal"])
def test_evict_a_few_over_the_budget(over, kind):
    """Up to 16 slots over go one by one, more by selection: the same slots either way."""
    weights = heavy if kind == "weights" else lambda c, s: torch.randint(0, 2, s, generator=c.g, device="cuda").float()
    pos = {"weights": None,
           "ties": lambda c, s: torch.randperm(int(np.prod(s)), generator=c.g, device="cuda").int().view(s) % 700,
           "all stay": lambda c, s: torch.randint(0, 20, s, generator=c.g, device="cuda").int() + 5000,
           "equal": lambda c, s: torch.full(s, 7, dtype=torch.int32, device="cuda")}[kind]
    for budget in (3, 33, 600):
        evict_case([budget + over, budget + 1, budget + over // 2, over], budget, 1, budget // 4, weights, pos=pos)


def test_evict_equal_positions_too():
    """Positions a caller has repeated: the lowest slots stay."""
    evict_case([200], 50, 0, 0, lambda c, s: torch.ones(s, device="cuda"), pos=lambda c, s: torch.full(s, 7, dtype=torch.int32, device="cuda"))
    evict_case([200], 50, 8, 0, lambda c, s: torch.ones(s, device="cuda"), pos=lambda c, s: torch.full(s, 7, dtype=torch.int32, device="cuda"))


def test_evict_then_attend_reads_the_survivors():
    c = evict_case([900, 40], 128, 4, 64, heavy)
    q = c.rand(2, 1, 8, 128).bfloat16()
    out, lse = c.cache.attend(q)
    check_attend(c, q, None, None, None, None, out, lse, 128 ** -0.5)


# ------------------------------------------------------------------------------ refusals ----

def test_refusals():
    c = Made([40, 3], 2, 128, 16)
    q, kn = c.rand(2, 4, 8, 128).bfloat16(), c.rand(2, 4, 2, 128).bfloat16()
    L, ref = c.cache._L, c.cache._ref

    def refused(fn, text):
        with pytest.raises(B.OilbirdError) as e:
            fn()
        assert e.value.code == B.EINVAL and text in str(e.value)

    odd = torch.zeros(2, 4, 8, 132, dtype=torch.bfloat16, device="cuda")[..., :128]
    refused(lambda: c.cache.attend(odd), "multiples of 8")
    refused(lambda: c.cache.attend(torch.zeros(2 * 4 * 8 * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 4, 8, 128)), "16-byte aligned")
    refused(lambda: c.cache.attend(c.rand(2, 65, 8, 128).bfloat16()), "nodes per sequence")
    refused(lambda: c.cache.attend(c.rand(2, 1, 7, 128).bfloat16()), "n_q_heads")
    refused(lambda: c.cache.attend(c.rand(2, 1, 130, 128).bfloat16()), "n_q_heads")
    refused(lambda: c.cache.attend(q, kn), "both or neither")
    refused(lambda: c.cache.attend(q, scale=float("nan")), "scale")
    refused(lambda: c.cache.evict(10, sink=6, recent=5), "budget")
    refused(lambda: c.cache.evict(0, sink=0, recent=0), "budget")
    with pytest.raises(AssertionError):
        c.cache.attend(q.half())
    with pytest.raises(AssertionError):
        c.cache.attend(q, kn, kn[:, :2])
    with pytest.raises(AssertionError):
        c.cache.append(kn, kn[:, :, :1])
    with pytest.raises(ValueError):
        B.KVCache(1, 1, 96, 100)
    with pytest.raises(ValueError):
        B.KVCache(1, 1, 64, 100, page_size=48)
    with pytest.raises(ValueError):
        B.KVCache.over(c.pages, c.weight, c.pos, c.table.long(), c.seq_len, c.n_pos)
    with pytest.raises(ValueError):
        B.KVCache.over(c.pages[..., :-1].contiguous(), c.weight, c.pos, c.table, c.seq_len, c.n_pos)
    # the C entry points themselves
    assert L.oilbird_kv_attend(None, 8, 1, None, None, None, None, 0, None, 1.0, None, None, None, None) == B.EINVAL
    bad = B.CKVCache.from_buffer_copy(c.cache._c)
    for field, value, text in (("head_dim", 96, "head_dim"), ("page_size", 8, "page_size"), ("n_seq", 0, "n_seq"),
                               ("n_seq", 1025, "n_seq"), ("n_pages", 0, "n_pages"), ("max_pages", 1 << 30, "max_pages"),
                               ("dtype", 2, "dtype"), ("pages", 0, "missing"), ("workspace_bytes", 100, "workspace"),
                               ("pages", c.pages.data_ptr() + 8, "aligned"), ("device", 99, "device")):
        old = getattr(bad, field)
        setattr(bad, field, value)
        rc = L.oilbird_kv_evict(bad, 10, 0, 0, None)
        assert rc == B.EINVAL and text in L.oilbird_kv_last_error().decode(), field
        setattr(bad, field, old)
    # nothing was launched by any of these
    torch.cuda.synchronize()
    assert c.seq_len.tolist() == [40, 3]


def test_empty_calls():
    c = Made([4], 1, 64, 16)
    c.cache.append(torch.zeros(1, 0, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 0, 1, 64, dtype=torch.bfloat16, device="cuda"))
    k, v = c.cache.read(0)
    assert k.shape == (1, 0, 1, 64) and v.shape == (1, 0, 1, 64) and c.seq_len.tolist() == [4]


def test_owned_cache():
    cache = B.KVCache(3, 2, 64, 100, page_size=32, dtype=torch.float16)
    k = torch.randn(3, 100, 2, 64, device="cuda").half()
    cache.append(k, k)
    rk, _ = cache.read(100)
    step = (k.float().amax(-1) - k.float().amin(-1)) / 15
    # half a step, the scale's rounding over fifteen codes, the value's own rounding
    assert torch.all((rk.float() - k.float()).abs().amax(-1) <= step * (0.5 + 15 * 2.0 ** -11) + 2.0 ** -11 * 8)
    assert cache.seq_len.tolist() == [100] * 3 and cache.dropped() == 0
    cache.append(k, k)                                           # 128 slots a sequence: 28 more fit
    assert cache.seq_len.tolist() == [128] * 3 and cache.dropped() == 3 * 72


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,hq", [(3, 4), (40, 4)])
def test_attend_what_a_row_does_not_see_does_not_reach_it(dtype, m, hq):
    """Infinities and NaN in hidden nodes stay there; in a node's values they reach the rows that
    see it, in their channels."""
    c = Made([70, 0], 1, 128, 64, dtype)
    q, kn, vn = (c.rand(2, m, h, 128).to(KIND[dtype]) for h in (hq, 1, 1))
    mask = torch.ones(2, m, dtype=torch.int64, device="cuda") << torch.arange(m, device="cuda")
    mask[:, m - 1] |= 1 << 1                                     # the last row also sees node 1
    want, wl = c.cache.attend(q, kn, vn, mask=mask)
    kn[:, 0], vn[:, 0] = float("nan"), float("inf")              # row 0 alone sees node 0
    vn[:, 1, 0, 5] = float("-inf")
    got, gl = c.cache.attend(q, kn, vn, mask=mask)
    assert torch.isnan(got[:, 0]).all() and torch.isnan(gl[:, 0]).all()
    for row in (1, m - 1):
        assert torch.all(got[:, row, :, 5] == float("-inf"))
        keep = [ch for ch in range(128) if ch != 5]
        # (the values' common scale may have changed with the odd element taken out)
        assert torch.allclose(got[:, row][..., keep].float(), want[:, row][..., keep].float(), rtol=2 * UNIT[dtype], atol=2.0 ** -11)
    if m > 3:
        assert torch.equal(gl[:, 2:m - 1], wl[:, 2:m - 1])
        assert torch.allclose(got[:, 2:m - 1].float(), want[:, 2:m - 1].float(), rtol=2 * UNIT[dtype], atol=2.0 ** -11)


@pytest.mark.parametrize("m,hq,hkv,lens", [(64, 16, 1, [900, 130]), (33, 8, 2, [4000]), (17, 8, 1, [5, 129, 0, 127, 128, 1000]),
                                            (64, 4, 4, [300]), (32, 4, 1, [2000, 90]), (33, 4, 1, [2000, 90])])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "f16")])
def test_attend_many_rows(m, hq, hkv, lens, d, dtype):
    """Row blocks of 256, of 128 and fewer (both groups on the same rows), items whole and cut."""
    attend_case(lens, m, hq, hkv, d, 32, dtype, ragged=len(lens) > 2)
