"""Prompt calls whose waits run out: that they say so, on every stream, and only once."""
import threading

import pytest
import torch

from paper_2608_03839_b200 import binding as B

pytestmark = pytest.mark.gpu


def made(lengths, d, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(lengths)
    new = lambda h: torch.randn(n, h, d, generator=g, device="cuda").bfloat16()
    first = torch.tensor([0, *lengths], dtype=torch.int32).cumsum(0, dtype=torch.int32).cuda()
    return new(8), new(2), new(2), first


@pytest.mark.parametrize("d,lengths", [(64, [3000, 300, 1]), (128, [700, 2000])])
def test_waits_that_run_out_are_reported_once(d, lengths):
    """A limit of a nanosecond is over before the first keys have come: at least one of the calls gives up and is
    reported, by the next status and by no other."""
    q, k, v, first = made(lengths, d)
    lse = B.prompt_attend(q, k, v, first=first)[1]
    calls = {"attend": lambda: B.prompt_attend(q, k, v, first=first), "weigh": lambda: B.prompt_weigh(q, lse, k, first=first)}
    calls["weigh"]()
    assert B.prompt_status() == B.OK
    try:
        B.prompt_set_wait_limit(1)
        for name, call in calls.items():
            got = []
            for _ in range(8):
                call()
                got.append(B.prompt_status())
                assert B.prompt_status() == B.OK
            assert B.ESTALL in got, f"{name}: no wait ran out"
    finally:
        B.prompt_set_wait_limit(0)
    for call in calls.values():
        call()
    assert B.prompt_status() == B.OK
