"""A context that only plans refuses the page and beam calls of the binding, whose own checks of tensors come before the library's."""
from types import SimpleNamespace

import pytest
import torch

from paper_2510_24051_amd.binding import Pie, PieError

MODEL = SimpleNamespace(hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_dim=64, vocab=512, page_size=16, rms_eps=1e-5, rope_theta=1e4)
IMAGE = torch.zeros((2, 1, 2, 16, 2, 64), dtype=torch.bfloat16)
INTS, FLOATS = torch.zeros((1, 4), dtype=torch.int32), torch.zeros((1, 4))


@pytest.mark.parametrize("call", [
    lambda p: p.save_kvpage([0, 1], IMAGE),
    lambda p: p.restore_kvpage([0, 1], IMAGE),
    lambda p: p.fork_kvpage([0], [1]),
    lambda p: p.compact_kvpage([0, 1], [0], [3]),
    lambda p: p.beam_select_async(torch.zeros((1, 512)), [0, 1], 4, INTS, INTS, FLOATS),
    lambda p: p.get_next_beams_async([0], [0, 1], 4, INTS, INTS, FLOATS),
], ids=["save", "restore", "fork", "compact", "select", "next"])
def test_planner_refuses(call):
    with pytest.raises(PieError) as e:
        call(Pie.planner(MODEL, 32, 16, 8, 4))
    assert e.value.status == -1
