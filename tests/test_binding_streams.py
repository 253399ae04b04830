"""Calls on the caller's tensors where torch's current stream is not the context's: behind what that stream holds, in front of what it
gets.  The streams and the library are stand-ins that write down what they are asked for."""
import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2510_24051_amd.binding import Pie, PieError

MODEL = SimpleNamespace(hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_dim=64, vocab=512, page_size=16, rms_eps=1e-5, rope_theta=1e4)
IMAGE = torch.zeros((2, 1, 2, 16, 2, 64), dtype=torch.bfloat16)
INTS, FLOATS = torch.zeros((1, 4), dtype=torch.int32), torch.zeros((1, 4))
CALLS = {
    "pie_save_kvpage": lambda p: p.save_kvpage([0, 1], IMAGE),
    "pie_restore_kvpage": lambda p: p.restore_kvpage([0, 1], IMAGE),
    "pie_beam_select": lambda p: p.beam_select_async(torch.zeros((1, 512)), [0, 1], 4, INTS, INTS, FLOATS),
    "pie_get_next_beams": lambda p: p.get_next_beams_async([0], [0, 1], 4, INTS, INTS, FLOATS),
}


class Stream:
    def __init__(self, name, log, raw):
        self.name, self.log, self.cuda_stream = name, log, raw

    def wait_event(self, event):
        self.log.append((self.name, "waits for", event.at))


class Event:
    def record(self, stream):
        self.at = (stream.name, len(stream.log))
        stream.log.append((stream.name, "records"))


def context(monkeypatch, current, status=0):
    log = []
    own, other = Stream("own", log, 7), Stream("other", log, 9)

    def call(name):
        return lambda *a: (log.append(("own", name)), status)[1]

    p = Pie.__new__(Pie)
    p.lib = SimpleNamespace(pie_last_error=lambda ctx: b"refused", pie_destroy=lambda ctx: 0, **{n: call(n) for n in CALLS})
    p.ctx, p.device, p.stream, p.model, p.n_layers = C.c_void_p(1), torch.device("cpu"), own, MODEL, 1
    p._index, p._raw_stream, p._before, p._after, p._page_image = 0, 7, Event(), Event(), (1, 2, 16, 2, 64)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: {"own": own, "other": other}[current])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: {"own": 7, "other": 9}[current], raising=False)
    return p, log


@pytest.mark.parametrize("name", list(CALLS))
def test_behind_and_in_front_of_the_current_stream(monkeypatch, name):
    p, log = context(monkeypatch, "other")
    CALLS[name](p)
    assert log == [("other", "records"), ("own", "waits for", ("other", 0)), ("own", name), ("own", "records"), ("other", "waits for", ("own", 3))]


@pytest.mark.parametrize("name", list(CALLS))
def test_nothing_to_wait_for_on_the_context_s_own_stream(monkeypatch, name):
    p, log = context(monkeypatch, "own")
    CALLS[name](p)
    assert log == [("own", name)]


@pytest.mark.parametrize("current", ["own", "other"])
def test_a_refusal_is_still_an_error(monkeypatch, current):
    p, _ = context(monkeypatch, current, status=-2)
    for call in CALLS.values():
        with pytest.raises(PieError) as e:
            call(p)
        assert e.value.status == -2
