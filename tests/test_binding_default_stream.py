"""A context on the device's default stream, while torch's current stream is being captured: the default stream cannot join a capture, so the call is
refused before anything is recorded.  Streams and library are stand-ins (test_binding_streams.py)."""
import pytest
import torch

from paper_2510_24051_amd.binding import MxRows, PieError
from test_binding_streams import CALLS, context


def on_default(monkeypatch, capturing):
    p, log = context(monkeypatch, "other")
    p._raw_stream, p._index = 0, -1  # (tensors of the CPU)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 9, raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    p.lib.pie_mx_quantise = lambda *a: (log.append(("own", "pie_mx_quantise")), 0)[1]
    return p, log


MORE = {**CALLS, "pie_mx_quantise": lambda p: p.mx_quantise(torch.zeros((2, 64)), MxRows.empty(2, 64, "mxfp8", "cpu"))}


@pytest.mark.parametrize("name", list(MORE))
def test_refused_while_another_stream_captures(monkeypatch, name):
    p, log = on_default(monkeypatch, True)
    with pytest.raises(PieError) as e:
        MORE[name](p)
    assert e.value.status == -6 and "default stream" in str(e.value) and log == []


@pytest.mark.parametrize("name", list(MORE))
def test_ordered_as_ever_otherwise(monkeypatch, name):
    p, log = on_default(monkeypatch, False)
    MORE[name](p)
    assert [x[1] for x in log] == ["records", "waits for", name, "records", "waits for"]
