"""Memory that the operators hold for their user, where calls run on another
stream than the one it was allocated on: dropped while such a call is under
way, it must not be handed to the next allocation on its own stream.  Nothing
is written to what is allocated here; the addresses are compared."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2410_23244_amd import ops

    return ops


def _ranges(tensors):
    return [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors
            if t.numel()]


def _shared(ranges, done):
    """Which of the ranges new allocations of their sizes and of small ones reach
    while the work before `done` is under way."""
    new = [torch.empty(b - a, dtype=torch.uint8, device="cuda") for a, b in ranges * 2]
    new += [torch.empty(512, dtype=torch.uint8, device="cuda") for _ in range(5000)]
    got = _ranges(new)
    assert not done.query(), "the work ended before the comparison"
    return [r for r in ranges if any(a < r[1] and r[0] < b for a, b in got)]


def _busy(side):
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda._sleep(200_000_000)


def test_the_comparison_sees_memory_that_is_handed_out_again():
    held = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (600, 8_000_000)]
    ranges = _ranges(held)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _busy(side)
    done = side.record_event()
    del held                                             # used by nothing
    assert len(_shared(ranges, done)) == 2


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_dropped_behind_a_step_on_another_stream(ops, bits):
    params = [torch.randn(n, device="cuda").to(torch.bfloat16) for n in (1_000, 77, 2_000_000)]
    grads = [torch.randn_like(p) for p in params]
    opt = ops.AdamW(params, grads, state_bits=bits, masters="new")
    ranges = _ranges([opt.ws, *opt.masters, *(t for s in opt.state for t in s.values())])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _busy(side)
        opt.step()
    done = side.record_event()
    del opt
    shared = _shared(ranges, done)
    torch.cuda.synchronize()
    assert not shared


def test_calibration_dropped_behind_a_fit_on_another_stream():
    from paper_2410_23244_amd.classify import Calibration

    scores = torch.randn(2, 100, 5, device="cuda")
    labels = torch.randint(0, 5, (100,), device="cuda")
    cal = Calibration(5, 2)
    cal.fit(scores, labels, 1)                           # libraries loaded beforehand
    ranges = _ranges(cal.D + cal.b + cal._dD + cal._db + [cal.opt.ws])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        cal.answer(scores)
        torch.cuda.synchronize()
        _busy(side)
        losses = cal.fit(scores, labels, 1)
    done = side.record_event()
    del cal
    shared = _shared(ranges, done)
    torch.cuda.synchronize()
    assert not shared and losses.isfinite().all()
