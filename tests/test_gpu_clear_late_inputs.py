"""Calls on another stream than the default read what was written on that stream just before them."""
import pytest
import torch

from tests.test_gpu_clear_streams import make, refill, step

pytestmark = pytest.mark.gpu


def test_inputs_that_arrive_late_on_the_calls_own_stream():
    """Every input holds other values, in range, until the stream of the calls has waited and copied the right ones: a call that ran
    on the default stream would take the others."""
    from paper_2604_09975_amd import clear as K
    want, stale = step(K, make(1)), step(K, make(7))
    assert not any(torch.equal(a, b) for a, b in zip(want, stale))
    s, right = make(7), make(1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(K, s)                   # the stream has its memory
    torch.cuda.synchronize()
    refill(s, make(7))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        refill(s, right)
        got = step(K, s)
        assert not side.query()      # the copies had not run when the calls were made
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
