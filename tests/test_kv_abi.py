"""The 4-bit cache's C-ABI as far as it goes without a GPU: sizes, constants, refusals."""
import ctypes
import os
import re

import pytest
import torch

from paper_2608_03839_b200 import binding as B

HEADER = open(os.path.join(os.path.dirname(__file__), "..", "include", "oilbird.h")).read()


@pytest.mark.parametrize("name", ["KV_BF16", "KV_F16", "KV_MAX_SEQ", "KV_MAX_GROUP", "KV_MAX_EVICT_SLOTS"])
def test_constants_are_the_headers(name):
    assert getattr(B, name) == int(re.search(r"#define OILBIRD_%s\s+(\d+)" % name, HEADER).group(1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_block_bytes(d, page):
    # keys and values: 32 bytes of codes, 4 of scale and offset for each slot and 64 channels
    assert B.lib().oilbird_kv_block_bytes(d, page) == 2 * page * (d // 64) * 36
    assert B.lib().oilbird_kv_workspace_bytes(d) > 0


@pytest.mark.parametrize("d,page", [(0, 64), (96, 64), (256, 64), (128, 8), (128, 48), (64, 0), (-64, 16)])
def test_block_bytes_of_what_is_not_supported(d, page):
    assert B.lib().oilbird_kv_block_bytes(d, page) == 0


def test_no_cache_is_refused_with_a_reason():
    L = B.lib()
    assert L.oilbird_kv_evict(None, 10, 0, 0, None) != B.OK
    assert b"cache" in L.oilbird_kv_last_error()
    n = ctypes.c_int64()
    assert L.oilbird_kv_status(None, ctypes.byref(n), None) != B.OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the machine without a GPU")
def test_there_is_no_cpu_fallback():
    with pytest.raises(RuntimeError, match="CUDA device"):
        B.KVCache(1, 2, 64, 128)
