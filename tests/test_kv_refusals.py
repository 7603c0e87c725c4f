"""What the 4-bit cache's C entry points refuse before they touch a device, with made-up addresses."""
import ctypes

import pytest
import torch

from paper_2608_03839_b200 import binding as B

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: for machines without a GPU")

AT = 1 << 20          # an address that nobody reads


@pytest.fixture
def cache():
    return B.CKVCache(AT, AT, AT, AT, AT, AT, AT, B.lib().oilbird_kv_workspace_bytes(128), 8, 2, 4, 64, 2, 128,
                      B.KV_BF16, 0)


def rows(at=AT, seq=1024, row=256, head=128):
    return ctypes.byref(B.CKVRows(at, seq, row, head))


def refused(rc, text):
    assert rc == B.EINVAL and text in B.lib().oilbird_kv_last_error().decode()


def test_misaligned_arrays(cache):
    L, ref = B.lib(), ctypes.byref(cache)
    for n_new, select, weight in ((AT + 2, None, None), (None, AT + 1, None), (None, None, AT + 3)):
        refused(L.oilbird_kv_append(ref, rows(), rows(), 4, 4, n_new, select, weight, None), "4-byte aligned")
    refused(L.oilbird_kv_read(ref, 4, AT + 2, AT, AT, None), "4-byte aligned")
    attend = lambda lse, n_new: L.oilbird_kv_attend(ref, 2, 4, rows(), None, None, None, 0, n_new, 1.0, rows(), lse, None, None)
    refused(attend(AT + 2, None), "4-byte aligned")
    refused(attend(None, AT + 1), "4-byte aligned")
    weigh = lambda lse, n_new, rw, nw: L.oilbird_kv_weigh(ref, 2, 4, rows(), lse, None, rows() if nw else None, None, 0,
                                                        n_new, rw, 1.0, nw, None)
    refused(weigh(AT + 2, None, None, None), "4-byte aligned")
    refused(weigh(AT, AT + 2, None, None), "4-byte aligned")
    refused(weigh(AT, None, AT + 2, None), "4-byte aligned")
    refused(weigh(AT, None, None, AT + 2), "4-byte aligned")


def test_rows_and_masks(cache):
    L, ref = B.lib(), ctypes.byref(cache)
    attend = lambda q=None, mask=None, stride=0: L.oilbird_kv_attend(ref, 2, 4, q or rows(), None, None, mask, stride, None, 1.0,
                                                                     rows(), None, None, None)
    refused(attend(rows(AT + 8)), "16-byte aligned")
    for bad in (dict(seq=1020), dict(row=260), dict(head=132)):
        refused(attend(rows(**bad)), "multiples of 8")
    refused(attend(mask=AT + 4, stride=4), "mask")
    refused(attend(mask=AT, stride=3), "mask")
    refused(attend(mask=AT, stride=-4), "mask")


@pytest.mark.parametrize("page", [16, 32, 64])
def test_sequences_end_a_tile_before_two_to_the_31(cache, page):
    """The last tile's slots, rounded up to whole tiles, still count in 32 bits.  (A budget of zero is
    refused next, so that nothing goes further.)"""
    L, ref = B.lib(), ctypes.byref(cache)
    cache.page_size = page
    for slots, text in ((2 ** 31 - page, "max_pages"), (2 ** 31 - 1024 + page, "max_pages"), (2 ** 31 - 1024, "budget")):
        cache.max_pages = slots // page
        refused(L.oilbird_kv_evict(ref, 0, 0, 0, None), text)
