"""Scratch of the attention layers as it grows: what a captured step may hold the address of stays alive."""
import weakref

import pytest
import torch

from paper_1904_08368_amd.decoder import Workspace


def test_buffers_that_were_handed_out_stay_alive():
    w = Workspace()
    refs = [weakref.ref(w.of(n, "cpu")) for n in (1000, 1001, 50000)]
    assert all(r() is not None for r in refs) and len({r().data_ptr() for r in refs}) == 3
    assert w.of(10, "cpu") is refs[-1]() and not refs[-1]().any()


@pytest.mark.parametrize("step", [1, 7])
def test_what_is_kept_is_below_twice_the_largest(step):
    w, alive = Workspace(), {}
    for n in range(100, 5000, step):
        t = w.of(n, "cpu")
        assert t.numel() >= n
        alive[t.data_ptr()] = t.numel()
    assert sum(alive.values()) < 2 * max(alive.values()) and max(alive.values()) < 2 * 5000


def test_nothing_is_handed_out_for_nothing():
    assert Workspace().of(0, "cpu") is None


def test_growth_during_a_capture_is_not_kept(monkeypatch):
    """The fill of a buffer made while a graph is captured has not run: no later call may take it for cleared."""
    w = Workspace()
    first = w.of(100, "cpu")
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    inside = w.of(1000, "cpu")
    assert inside.numel() >= 1000 and inside is not first and w.of(100, "cpu") is first
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    outside = w.of(1000, "cpu")
    assert outside is not inside and w.of(1000, "cpu") is outside
