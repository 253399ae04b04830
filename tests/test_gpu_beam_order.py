"""Which candidates a selection names and in which order: every one of them is looked up in the logits, in 64 bits.

Within one beam the order is that of the logits, equal ones by token, whatever the row's normaliser is rounded to.  Between beams it
is that of the scores, which are as exact as the rows' logarithms (NEAR, derived in test_gpu_beams.py).  Beams that are equal in
everything have equal scores, so theirs is exact again."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from oracle import pie_oracle as O
from test_gpu_beams import LARGEST, LSE, logits, select

pytestmark = pytest.mark.gpu

NEAR = 2 * LSE
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


# ---- every candidate looked up -----------------------------------------------------------------------------------------------
def candidates(row, score, done, eos, t, largest):
    """(tokens, scores) of one beam in their order."""
    score = min(float(score), float(np.finfo(np.float32).max))
    if math.isnan(score) or score == -math.inf:
        return np.zeros(0, np.int64), np.zeros(0)
    if done:
        return np.array([eos]), np.array([score])
    tokens = np.nonzero(~np.isnan(row) & (row > -math.inf))[0]
    if not len(tokens):
        return tokens, np.zeros(0)
    x = np.minimum(row[tokens], largest) / t
    d = x - x.max()
    each = score + (d - math.log(np.exp(d).sum()))
    order = np.lexsort((tokens, -each))
    return tokens[order], each[order]


def named(ctx, z, indptr, n_out, scores=None, finished=None, eos=-1, t=1.0):
    b, v, s = select(ctx, z, indptr, n_out, scores, finished, eos, t)
    rows, t = z.double().cpu().numpy(), float(np.float32(t))
    start = np.zeros(len(rows), np.float32) if scores is None else np.asarray(scores, np.float32)
    done = np.zeros(len(rows), bool) if finished is None else np.asarray(finished).astype(bool)
    for g in range(len(indptr) - 1):
        mine = range(indptr[g], indptr[g + 1])
        lists = [candidates(rows[r], start[r], done[r], eos, t, LARGEST[z.dtype]) for r in mine]
        alike = [(start[r].tobytes(), None if done[r] else rows[r].tobytes()) for r in mine]
        taken = np.zeros(len(lists), int)
        heads = np.array([c[1][0] if len(c[1]) else -math.inf for c in lists])
        n = min(n_out, sum(len(c[0]) for c in lists))
        assert (b[g, n:] == -1).all() and (v[g, n:] == -1).all() and np.isneginf(s[g, n:]).all()
        for i in range(n):
            r = int(b[g, i])
            assert 0 <= r < len(lists) and taken[r] < len(lists[r][0]), (g, i, r)
            tokens, each = lists[r]
            k = taken[r]
            e = each[k]
            if int(v[g, i]) != tokens[k]:  # (only where a rounding of 64 bits tells them apart; scores beyond 1e25 absorb the logits whole)
                at = np.nonzero(tokens == v[g, i])[0]
                x = rows[indptr[g] + r]
                assert len(at) == 1 and x[v[g, i]] != x[tokens[k]] and abs(e) < 1e25, (g, i, r, int(v[g, i]), int(tokens[k]))
                assert abs(each[at[0]] - e) <= 8 * np.spacing(abs(e)), (g, i, r, int(v[g, i]), int(tokens[k]))
            assert abs(float(s[g, i]) - e) <= LSE + abs(e) * 2.0 ** -24 or (np.isneginf(s[g, i]) and e < -np.finfo(np.float32).max), (g, i)
            assert heads.max() <= e + NEAR + 8 * np.spacing(abs(e)), (g, i)  # nothing that is left comes before it
            for other in np.nonzero(heads >= e)[0]:
                if other != r and alike[other] == alike[r]:
                    assert other > r and heads[other] == e, (g, i)
            taken[r] += 1
            heads[r] = each[k + 1] if k + 1 < len(each) else -math.inf
        for r in range(len(lists)):  # no candidate twice
            got = v[g, :n][b[g, :n] == r]
            assert len(set(got.tolist())) == len(got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,stride,offset", [(1, 1, 0), (63, 64, 0), (1000, 1003, 1), (2049, 2056, 8), (8191, 8191, 5), (50257, 50304, 0)])
def test_every_candidate_is_the_next_of_its_beam(ctx, dtype, V, stride, offset):
    z = logits(13, V, dtype, V, stride, offset)
    scores = np.random.default_rng(V).standard_normal(13) - 20
    for n_out, t in ((1, 1.0), (9, 0.75), (70, 1.25)):
        named(ctx, z, [0, 4, 5, 5, 13], n_out, scores, t=t)


@pytest.mark.parametrize("rows,n_out", [(1, 1), (1, 256), (8, 1), (8, 16), (64, 256), (256, 1), (256, 256)])
def test_every_candidate_of_many_beams(ctx, rows, n_out):
    named(ctx, logits(rows, 5003, torch.float32, rows + n_out), [0, rows], n_out, np.random.default_rng(rows).standard_normal(rows))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,n_out", [(100, 30), (4096, 1), (4096, 7), (4097, 256), (60001, 64)])
def test_long_runs_of_equal_logits_across_the_cut(ctx, dtype, V, n_out):
    z = torch.randint(0, 4, (3, V), generator=torch.Generator(device="cuda").manual_seed(V), device="cuda").to(dtype)
    named(ctx, z, [0, 3], n_out, np.zeros(3))
    named(ctx, z[:1].repeat(5, 1), [0, 2, 5], n_out, np.full(5, -3.0))


@pytest.mark.parametrize("dtype", TYPES)
def test_every_candidate_of_masked_rows_is_allowed(ctx, dtype):
    V, inf, low = 3001, math.inf, torch.finfo(dtype).min
    z = logits(10, V, dtype, 3)
    z[0] = -inf                       # a row with nothing left
    z[1, 5:] = -inf                   # fewer left than asked for
    z[2, ::2] = float("nan")          # NaN counts as masked
    z[3, 1:] = low                    # the type's lowest value is a logit like any other
    z[4] = low
    z[5] = float("nan")
    z[6, 7] = inf
    z[7, 7], z[7, 2999] = inf, inf
    z[8, :3000] = -inf                # only the last token
    for indptr in ([0, 10], list(range(11)), [0, 1, 6, 10]):
        for n_out in (1, 8, 70):
            named(ctx, z, indptr, n_out, np.zeros(10))
            named(ctx, z, indptr, n_out, np.arange(10) * 0.5 - 20, np.arange(10) % 4 == 2, eos=3000, t=0.75)


def test_every_candidate_far_apart_close_together_and_crowded(ctx):
    named(ctx, logits(6, 20000, torch.float32, 77, spread=30.0), [0, 3, 6], 25, np.array([0.0, -1e4, -1e-3, -3e4, -1e30, 0.0]))
    named(ctx, logits(4, 20000, torch.float32, 78, spread=1e-3), [0, 4], 50, np.array([-5.0, -5.0 - 1e-6, -5.0 + 1e-6, -5.0]))
    named(ctx, logits(4, 20000, torch.float32, 79), [0, 4], 8, np.zeros(4), t=1e-3)
    for s in (1e10, 2.0 ** 39, 2.0 ** 41, 1e15):
        named(ctx, logits(4, 20000, torch.float32, 81), [0, 4], 30, np.array([s, 0.0, s, -s]))
    z = logits(4, 40000, torch.float32, 6)
    z[2, 12000:12512] = 20.0 + torch.rand(512, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    named(ctx, z, [0, 4], 256, np.zeros(4))
    z[:, 512:20000] = 25.0 + torch.rand((4, 20000 - 512), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") * 1e-3
    named(ctx, z, [0, 4], 256, np.zeros(4))


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
