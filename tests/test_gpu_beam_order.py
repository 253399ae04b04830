"""Which candidates a selection names and in which order."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from oracle import pie_oracle as O
from test_gpu_beams import LARGEST, logits, select

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from paper_2510_24051_amd import Pie
    m = W.ModelDesc(hidden=128, n_q_heads=2, n_kv_heads=2, head_dim=64, mlp_dim=256, vocab=131072, page_size=16, rms_eps=1e-5, rope_theta=1e4, n_layers=1)
    return Pie(m, 4, 4, max_batch_tokens=4, max_batch_requests=4, max_dist_rows=700)


def oracle(z, indptr, n_out, scores=None, finished=None, eos=-1, t=1.0):
    s = None if scores is None else np.asarray(scores, np.float32)
    return O.beam_select(z.double().cpu().numpy(), indptr, n_out, s, finished, eos, t, largest=LARGEST[z.dtype])


# ---- scores so far from 0 that the logits do not change them ---------------------------------------------------------------
FAR = {"all above": [np.inf] * 4, "one above": [-3.0, np.inf, 2.0, -1.0], "two above": [np.inf, 0.0, -5.0, np.inf], "all far below": [-1e30] * 4,
       "lowest": [-np.finfo(np.float32).max] * 4, "two far": [-2e30, -1e30, -2e30, -1e30], "one alive": [-np.inf, -1e35, np.nan, -np.inf]}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [5, 1003, 5003, 40000])
@pytest.mark.parametrize("name", list(FAR))
def test_scores_that_absorb_the_logits_tie(ctx, name, V, dtype):
    """One step of a 64-bit score of 1e30 is 1e14: all of a row's candidates are equal, so they go by beam and token."""
    scores, z = FAR[name], logits(4, V, dtype, V + 1)
    for n_out in (1, 6, 200):
        for indptr in ([0, 4], [0, 2, 4]):
            b, v, s = select(ctx, z, indptr, n_out, scores)
            wb, wv, ws = oracle(z, indptr, n_out, scores)
            far = ~(np.abs(ws) < 1e6)  # (groups without such a score are the other tests' business)
            assert np.array_equal(b[far], wb[far]) and np.array_equal(v[far], wv[far]), (n_out, indptr)
            assert np.array_equal(s[far], ws[far].astype(np.float32))


def test_finished_beams_among_scores_that_absorb_the_logits(ctx):
    z = logits(5, 3000, torch.float32, 12)
    b, v, s = select(ctx, z, [0, 5], 6, [1e30, 1e30, 1e30, 0.0, np.inf], [0, 1, 0, 0, 1], eos=2999)
    assert list(zip(b[0], v[0])) == [(4, 2999), (0, 0), (0, 1), (0, 2), (0, 3), (0, 4)]
    assert s[0, 0] == np.finfo(np.float32).max and (s[0, 1:] == np.float32(1e30)).all()


# ---- rows of which one token has nearly all of the probability ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1024, 4096, 4099, 32000, 131072])
def test_many_small_terms_beside_a_large_one(ctx, dtype, V):
    """exp(-16.75) is less than half of fp32's step at 1: added to the likeliest token's 1 one by one in 32 bits, the others vanish.
    Each term is off by its argument's roundings (three of 2^-24 at 24.2, in units of log 2) and 2^-23: 5e-6 of itself, the likeliest
    token's not at all; so is the logarithm, beside its rounding to fp32."""
    for at in (0, V - 1, V // 2):
        z = torch.full((2, V), -16.75, dtype=dtype, device="cuda")
        z[0, at] = 0.0
        z[1] = -math.inf
        z[1, 5] = 3.0  # (its score is the beam's)
        want = -math.log1p((V - 1) * math.exp(-16.75))
        _, _, s = select(ctx, z, [0, 1, 2], 1, np.zeros(2))
        assert abs(float(s[0, 0]) - want) <= abs(want) * (5e-6 + 2.0 ** -24) and s[1, 0] == 0.0
        for behind in (False, True):  # a beam next to it, on either side: 2e-5 of that sum away
            other = np.float32(want * (1.00002 if behind else 0.99998))
            b, v, _ = select(ctx, z, [0, 2], 2, np.array([0.0, other]))
            order = [(0, at), (1, 5)] if behind else [(1, 5), (0, at)]
            assert list(zip(b[0], v[0])) == order, (at, behind)
