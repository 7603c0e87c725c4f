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


def test_a_status_elsewhere_loses_no_report():
    """Another thread asks for the status all the time, on a stream of its own: a call that gives up is reported to
    one of the two, whenever that happens."""
    q, k, v, first = made([700, 2000], 128)
    want = B.prompt_attend(q, k, v, first=first)[0]
    torch.cuda.synchronize()
    assert B.prompt_status() == B.OK
    elsewhere, done = [0], threading.Event()

    def ask():
        stream = torch.cuda.Stream()
        while not done.is_set():
            elsewhere[0] += B.prompt_status(stream=stream) == B.ESTALL

    thread = threading.Thread(target=ask)
    gave_up = lost = 0
    stream = torch.cuda.Stream()
    try:
        B.prompt_set_wait_limit(1)
        torch.cuda.synchronize()
        thread.start()
        with torch.cuda.stream(stream):
            for _ in range(200):
                before = elsewhere[0]
                out = torch.zeros_like(want)
                B.prompt_attend(q, k, v, first=first, out=out)
                stream.synchronize()
                here = B.prompt_status() == B.ESTALL
                if torch.equal(out, want):
                    continue
                gave_up += 1
                if not here:                               # the other thread has it, or is about to
                    for _ in range(100):
                        if elsewhere[0] > before:
                            break
                        done.wait(0.001)
                    lost += elsewhere[0] == before
    finally:
        done.set()
        thread.join()
        B.prompt_set_wait_limit(0)
        B.prompt_status()
    assert gave_up > 0 and lost == 0, (gave_up, lost)
