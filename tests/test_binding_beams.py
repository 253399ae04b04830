"""Lists of searches that the binding refuses before the library is asked."""
import pytest
import torch

from test_binding_streams import FLOATS, INTS, context


@pytest.mark.parametrize("n_out", [4, 0, -4])
def test_a_list_of_searches_has_its_first_row(monkeypatch, n_out):
    p, log = context(monkeypatch, "own")
    with pytest.raises(ValueError):
        p.beam_select_async(torch.zeros((1, 512)), [], n_out, INTS[:, :abs(n_out)], INTS[:, :abs(n_out)], FLOATS[:, :abs(n_out)])
    with pytest.raises(ValueError):
        p.get_next_beams_async([0], [], n_out, INTS[:, :abs(n_out)], INTS[:, :abs(n_out)], FLOATS[:, :abs(n_out)])
    with pytest.raises(ValueError):
        p.get_next_beams([0], [], n_out)
    assert log == []
