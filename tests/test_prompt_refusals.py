"""What the prompt calls and token scores refuse before they touch a device, with made-up addresses; the constants
of the binding."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_03839_b200 import binding as B

HEADER = open(os.path.join(os.path.dirname(__file__), "..", "include", "oilbird.h")).read()
AT = 1 << 20          # an address that nobody reads
cpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: for machines without a GPU")


@pytest.mark.parametrize("name", ["LOGITS_BF16", "LOGITS_F16", "LOGITS_F32", "SCORES_MAX_VOCAB", "SCORES_MAX_TOP"])
def test_constants_are_the_headers(name):
    assert getattr(B, name) == int(re.search(r"#define OILBIRD_%s\s+(\d+)" % name, HEADER).group(1))


def prompt(first=0, count=0, rows=100, first_k=0, count_k=0, rows_k=100, n_seq=2, hq=4, hkv=2, d=64, dtype=0, device=0):
    return (ctypes.c_int64 * 9)(first, count, rows, first_k, count_k, rows_k, n_seq | hq << 32, hkv | d << 32, dtype | device << 32)


def rows(at=AT, seq=100 * 256, row=256, head=64):
    return ctypes.byref(B.CKVRows(at, seq, row, head))


def refused(rc, text):
    assert rc == B.EINVAL and text in B.lib().oilbird_prompt_last_error().decode()


def attend(p=None, q=None, k=None, v=None, scale=1.0, out=None, lse=AT):
    return B.lib().oilbird_prompt_attend(p or prompt(), q or rows(), k or rows(), v or rows(), scale, out or rows(), lse, None, None)


def weigh(p=None, q=None, lse=AT, k=None, rw=None, scale=1.0, weight=AT):
    return B.lib().oilbird_prompt_weigh(p or prompt(), q or rows(), lse, None, k or rows(), rw, scale, weight, None)


@cpu
@pytest.mark.parametrize("call", [attend, weigh])
def test_shapes(call):
    assert B.lib().oilbird_prompt_attend(None, rows(), rows(), rows(), 1.0, rows(), AT, None, None) == B.EINVAL
    for more, text in ((dict(d=96), "head_dim"), (dict(dtype=2), "dtype"), (dict(n_seq=0), "n_seq"), (dict(n_seq=1025), "n_seq"),
                       (dict(hkv=0), "n_kv_heads"), (dict(hq=0), "n_q_heads"), (dict(hq=5), "n_q_heads"), (dict(hq=130), "n_q_heads"),
                       (dict(rows=-1), "query rows"), (dict(rows_k=2 ** 31), "key rows"), (dict(first=AT + 2), "query rows"),
                       (dict(count_k=AT + 1), "key rows"), (dict(device=64), "device"), (dict(device=-1), "device")):
        refused(call(prompt(**more)), text)
    for scale in (float("nan"), float("inf")):
        refused(call(scale=scale), "scale")


@cpu
@pytest.mark.parametrize("call", [attend, weigh])
def test_rows(call):
    for bad, text in ((dict(at=AT + 8), "16-byte"), (dict(row=260), "multiples of 8"), (dict(head=12), "multiples of 8"),
                      (dict(seq=4), "multiples of 8"), (dict(row=-256), "not negative"), (dict(row=1 << 39), "below"), (dict(at=None), "missing")):
        refused(call(q=rows(**bad)), text)
        refused(call(k=rows(**bad)), text)


@cpu
def test_arrays():
    refused(attend(v=rows(at=AT + 2)), "v")
    refused(attend(out=rows(at=AT + 2)), "out")
    refused(attend(lse=AT + 2), "lse")
    refused(weigh(lse=None), "lse")
    refused(weigh(weight=None), "weight")
    for name in ("lse", "rw", "weight"):
        refused(weigh(**{name: AT + 1}), "4-byte")


@cpu
def test_nothing_to_do_is_done():
    """No query rows: attention is done before any device is looked for; no keys: weights are."""
    assert attend(prompt(rows=0), q=rows(at=None), out=rows(at=None)) == B.OK
    assert weigh(prompt(rows_k=0), k=rows(at=None)) == B.OK


def scores(logits=AT, stride=1000, n=2, vocab=1000, dtype=2, tokens=AT, n_tokens=1, k=1, out=(AT,) * 5, device=0):
    return B.lib().oilbird_token_scores(logits, stride, n, vocab, dtype, tokens, n_tokens, k,
                                        None if out is None else (ctypes.c_int64 * 5)(*out), device, None)


@cpu
def test_scores():
    for more, text in ((dict(dtype=3), "dtype"), (dict(n=-1), "rows"), (dict(n=2 ** 24 + 1), "rows"), (dict(vocab=0), "vocab"),
                       (dict(vocab=2 ** 24 + 1), "vocab"), (dict(k=65), "k:"), (dict(k=-1), "k:"), (dict(n_tokens=-1), "n_tokens"),
                       (dict(stride=-1), "row_stride"), (dict(out=None), "out"), (dict(logits=None), "logits"), (dict(logits=AT + 2), "logits"),
                       (dict(tokens=None), "tokens"), (dict(out=(0, AT, AT, AT, AT)), "logp"), (dict(out=(AT, AT, AT, 0, AT)), "top_id"),
                       (dict(out=(AT, AT + 2, AT, AT, AT)), "4-byte"), (dict(tokens=AT + 1), "4-byte"), (dict(device=64), "device")):
        assert scores(**more) == B.EINVAL and text in B.lib().oilbird_token_scores_error().decode(), more
    assert scores(n=0, logits=None) == B.OK


@cpu
def test_there_is_no_cpu_fallback():
    q, x = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 10)
    first = torch.tensor([0, 3], dtype=torch.int32)
    for call in (lambda: B.prompt_attend(q, q, q, first=first), lambda: B.prompt_weigh(q, q[..., 0].float(), q, first=first),
                 lambda: B.token_scores(x)):
        with pytest.raises(AssertionError, match="CPU fallback"):
            call()
