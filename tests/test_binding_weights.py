"""Microscaled weights that are dropped and not destroyed: Python may collect them at any time, a capture on another stream among them, so
nothing waits for the GPU or frees its memory there.  The library is a stand-in that writes down what it is asked for."""
import ctypes as C
import gc
from types import SimpleNamespace

import pytest
import torch

from paper_2510_24051_amd.binding import MxRows, MxWeight, Pie, PieError


def context(monkeypatch, status=0):
    log = []
    made = iter(range(100, 200))

    def create(ctx, parts, rows, n, k, gated, out):
        log.append("create")
        out._obj.value = next(made)
        return 0

    p = Pie.__new__(Pie)
    p.lib = SimpleNamespace(pie_last_error=lambda ctx: b"refused", pie_destroy=lambda ctx: log.append("close"), pie_mx_weight_create=create,
                            pie_synchronize=lambda ctx: (log.append("synchronize"), 0)[1],
                            pie_mx_weight_destroy=lambda ctx, h: (log.append(("destroy", h.value)), status)[1])
    p.ctx, p.device, p._index = C.c_void_p(1), torch.device("cpu"), -1
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: log.append("wait"))
    return p, log


def part():
    return MxRows.empty(4, 64, "mxfp4", "cpu")


def test_dropped_weights_are_freed_by_the_next_call_that_waits(monkeypatch):
    p, log = context(monkeypatch)
    a, b = p.mx_weight([part()]), p.mx_weight([part()])
    del log[:]
    del a
    gc.collect()
    assert log == []
    p.synchronize()
    assert log == ["synchronize", ("destroy", 100)]
    del log[:], b
    gc.collect()
    assert log == []
    c = p.mx_weight([part()])
    assert log == ["wait", ("destroy", 101), "create"]
    c.destroy()  # at once, and once
    assert log[-1] == ("destroy", 102)
    del c, log[:]
    p.synchronize()
    assert log == ["synchronize"]


def test_a_closed_context_frees_its_weights_itself(monkeypatch):
    p, log = context(monkeypatch)
    a, b = p.mx_weight([part()]), p.mx_weight([part()])
    del a, log[:]
    p.close()
    del b
    gc.collect()
    assert log == ["close"]


def test_a_weight_that_cannot_be_destroyed_says_so(monkeypatch):
    p, log = context(monkeypatch, status=-6)
    w = p.mx_weight([part()])
    with pytest.raises(PieError):
        w.destroy()
    assert isinstance(w, MxWeight) and w.handle is not None
