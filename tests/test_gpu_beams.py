"""The selection over beams and vocabulary on the GPU against the oracle's, in 64 bits.

Scores: a row's normaliser is a sum of up to 131072 exponentials in fp32, each off by the rounding of its argument (up to 25 in
magnitude: 25 x 2^-24 x 1.5 = 2.3e-6) and one unit in the last place, sums of a few dozen terms in fp32 and of the rest in 64 bits:
at most 4e-6 on its logarithm.  A stored score is rounded to fp32 once.  Candidates further apart than twice that have one order."""
import math

import numpy as np
import pytest
import torch

import workloads as W
from oracle import pie_oracle as O

pytestmark = pytest.mark.gpu

LSE = 4e-6
LARGEST = {torch.float32: float(torch.finfo(torch.float32).max), torch.bfloat16: float(torch.finfo(torch.bfloat16).max), torch.float16: 65504.0}


@pytest.fixture(scope="module")
def ctx():
    from paper_2510_24051_amd import Pie
    m = W.ModelDesc(hidden=128, n_q_heads=2, n_kv_heads=2, head_dim=64, mlp_dim=256, vocab=131072, page_size=16, rms_eps=1e-5, rope_theta=1e4, n_layers=1)
    return Pie(m, 4, 4, max_batch_tokens=4, max_batch_requests=4, max_dist_rows=700)


def select(ctx, z, indptr, n_out, scores=None, finished=None, eos=-1, t=1.0):
    G = len(indptr) - 1
    ob, ot = (torch.full((G, n_out), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    os_ = torch.full((G, n_out), -7.0, device="cuda")
    s = None if scores is None else torch.tensor(np.asarray(scores, np.float32), device="cuda")
    f = None if finished is None else torch.tensor(np.asarray(finished, np.uint8), device="cuda")
    torch.cuda.synchronize()
    ctx.beam_select_async(z, indptr, n_out, ob, ot, os_, s, f, eos, t)
    ctx.synchronize()
    return ob.cpu().numpy(), ot.cpu().numpy(), os_.cpu().numpy()


def check(ctx, z, indptr, n_out, scores=None, finished=None, eos=-1, t=1.0, exact_ids=False):
    b, v, s = select(ctx, z, indptr, n_out, scores, finished, eos, t)
    s32 = None if scores is None else np.asarray(scores, np.float32)
    wb, wv, ws = O.beam_select(z.double().cpu().numpy(), indptr, n_out, s32, finished, eos, t, largest=LARGEST[z.dtype])
    none = wb < 0
    assert np.array_equal(b < 0, none) and np.array_equal(v < 0, none) and np.all(np.isneginf(s[none]))
    assert np.all(np.abs(s[~none].astype(np.float64) - ws[~none]) <= LSE + np.abs(ws[~none]) * 2.0 ** -24)
    for g, i in np.argwhere((b != wb) | (v != wv)):
        assert not exact_ids and b[g, i] >= 0
        # the candidate named is the oracle's at a rank whose score is as near
        at = np.argwhere((wb[g] == b[g, i]) & (wv[g] == v[g, i]))
        near = ws[g, at[0, 0]] if len(at) else ws[g, -1]
        assert abs(near - ws[g, i]) <= 2 * LSE, (g, i)
    for g in range(len(indptr) - 1):
        pairs = [(x, y) for x, y in zip(b[g], v[g]) if x >= 0]
        assert len(set(pairs)) == len(pairs)
    return b, v, s


def logits(n, V, dtype, seed, stride=None, offset=0, spread=2.0):
    """[n, V] views of rows `stride` apart, `offset` elements into their buffer; what lies between the rows is never looked at."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    stride = stride or V
    buf = torch.full((offset + n * stride + 8,), 1e4, dtype=dtype, device="cuda")
    z = torch.as_strided(buf, (n, V), (stride, 1), offset)
    z.copy_(torch.randn((n, V), generator=gen, device="cuda") * spread)
    return z


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,stride,offset", [(1, 1, 0), (2, 3, 1), (63, 64, 0), (257, 257, 3), (1000, 1003, 1), (2048, 2048, 0), (2049, 2056, 8),
                                             (8191, 8191, 5), (32000, 32000, 0), (50257, 50304, 0), (131072, 131072, 0)])
def test_sizes_strides_and_types(ctx, dtype, V, stride, offset):
    z = logits(13, V, dtype, V, stride, offset)
    scores = np.random.default_rng(V).standard_normal(13) - 20
    for n_out, t in ((1, 1.0), (9, 0.75), (40, 1.25)):
        check(ctx, z, [0, 4, 5, 5, 13], n_out, scores, t=t)


@pytest.mark.parametrize("rows,n_out", [(1, 1), (1, 256), (2, 17), (8, 16), (31, 100), (64, 256), (256, 3), (256, 256)])
def test_beams_and_candidates(ctx, rows, n_out):
    z = logits(rows, 5003, torch.float32, rows + n_out)
    check(ctx, z, [0, rows], n_out, np.random.default_rng(rows).standard_normal(rows))


def test_many_groups(ctx):
    """More groups than one launch names, some without beams."""
    sizes = np.random.default_rng(0).integers(0, 3, 600)
    sizes[::97] = 4
    indptr = np.concatenate([[0], np.cumsum(sizes)])
    z = logits(int(indptr[-1]), 300, torch.float32, 9)
    check(ctx, z, indptr, 5, np.random.default_rng(1).standard_normal(int(indptr[-1])))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,n_out", [(100, 30), (4096, 7), (4097, 256), (60001, 64)])
def test_equal_scores_go_by_beam_and_token(ctx, dtype, V, n_out):
    for rows in (1, 5):
        same = torch.full((rows, V), 0.75, dtype=dtype, device="cuda")
        b, v, _ = check(ctx, same, [0, rows], n_out, exact_ids=True)
        assert np.array_equal(b[0] * V + v[0], np.where(np.arange(n_out) < rows * V, np.arange(n_out), b[0] * V + v[0]))
    # the beams of a first step are equal in everything: every candidate of the first comes before its equals
    z = logits(1, V, dtype, 4).repeat(6, 1)
    check(ctx, z, [0, 6], n_out, np.full(6, -3.0), exact_ids=True)
    # few distinct values: long runs of ties across the cut
    z = torch.randint(0, 4, (3, V), device="cuda").to(dtype)
    check(ctx, z, [0, 3], n_out, np.zeros(3), exact_ids=True) if V < 200 else check(ctx, z, [0, 3], n_out, np.zeros(3))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_masked_logits(ctx, dtype):
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
    for indptr in ([0, 10], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10], [0, 1, 6, 10]):
        for n_out in (1, 8, 70):
            b, v, s = select(ctx, z, indptr, n_out, np.zeros(10))
            wb, wv, ws = O.beam_select(z.double().cpu().numpy(), indptr, n_out, np.zeros(10), largest=LARGEST[dtype])
            assert not np.isnan(s).any()
            assert np.array_equal(b < 0, wb < 0)
            sure = np.abs(ws) < 1e4  # (differences of logits of 1e38 exceed fp32)
            sure &= wb >= 0
            assert np.all(np.abs(s[sure] - ws[sure]) <= LSE + 1e-6 * 4)
    # a row alone whose other logits are the lowest: the one token, then the lowest in order
    b, v, s = select(ctx, z, [0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0][:1] + [10], 3, np.r_[[-np.inf] * 3, 0.0, [-np.inf] * 6])
    assert b[0].tolist() == [3, 3, 3] and v[0].tolist() == [0, 1, 2] and abs(s[0, 0]) < LSE


def test_dead_and_finished_beams(ctx):
    V = 2500
    z = logits(8, V, torch.float32, 8)
    z[2] = float("nan")  # not looked at where the beam is finished
    scores = np.array([-1.0, -np.inf, -0.25, np.nan, -0.25, -np.inf, 2.0, -4.0])
    fin = np.array([0, 0, 1, 0, 1, 1, 0, 0])
    b, v, s = check(ctx, z, [0, 8], 12, scores, fin, eos=V - 1)
    done = [(x, y) for x, y in zip(b[0], v[0]) if fin[x]]
    assert done == [(2, V - 1), (4, V - 1)] and not {1, 3, 5} & set(b[0].tolist())
    b, v, s = check(ctx, z, [0, 2, 4, 6, 8], 4, scores, fin, eos=0)
    assert b[1].tolist() == [0, -1, -1, -1] and v[1].tolist() == [0, -1, -1, -1] and s[1, 0] == -0.25  # one finished beam, one dead
    # all finished: as many candidates as beams, equal scores by beam
    b, v, _ = check(ctx, z, [0, 8], 3, np.full(8, -2.0), np.ones(8, int), eos=3, exact_ids=True)
    assert b[0].tolist() == [0, 1, 2] and v[0].tolist() == [3, 3, 3]
    b, _, _ = check(ctx, z, [0, 8], 3, np.full(8, -np.inf))
    assert (b == -1).all()
    check(ctx, z[:2], [0, 2, 2, 2], 5)  # (no scores, groups without beams)


def test_scores_far_apart_and_close_together(ctx):
    z = logits(6, 20000, torch.float32, 77, spread=30.0)  # the best token has nearly all of the probability
    check(ctx, z, [0, 3, 6], 25, np.array([0.0, -1e4, -1e-3, -3e4, -1e30, 0.0]))
    z = logits(4, 20000, torch.float32, 78, spread=1e-3)
    check(ctx, z, [0, 4], 50, np.array([-5.0, -5.0 - 1e-6, -5.0 + 1e-6, -5.0]))
    check(ctx, logits(4, 20000, torch.float32, 79), [0, 4], 8, np.zeros(4), t=1e-3)
    check(ctx, logits(4, 20000, torch.float32, 80), [0, 4], 8, np.arange(4.0), t=1e6)


def test_the_smallest_and_largest_temperatures(ctx):
    z = logits(2, 700, torch.float32, 5)
    z[0, 5], z[0, 9] = -math.inf, torch.finfo(torch.float32).min
    for t in (1.1e-30, 1e-20):
        b, v, s = select(ctx, z, [0, 1, 2], 2, t=t)
        assert not np.isnan(s).any() and s[0, 0] == 0.0
        assert v[:, 0].tolist() == z.argmax(1).cpu().tolist()
    for t in (1e20, 9e29):  # all the same but the masked one and, where it still counts, the lowest
        b, v, s = select(ctx, z, [0, 1, 2], 256, t=t)
        assert np.allclose(s, -np.log([[698], [700]]), atol=LSE) and not {5, 9} & set(v[0].tolist())


def test_crowded_candidates(ctx):
    """Every one of the best candidates in one place of one row: the survivors of a coarse cut are many."""
    V = 40000
    z = logits(4, V, torch.float32, 6)
    z[2, 12000:12512] = 20.0 + torch.rand(512, device="cuda")
    check(ctx, z, [0, 4], 256, np.zeros(4))
    z[:, 512:20000] = 25.0 + torch.rand((4, 20000 - 512), device="cuda") * 1e-3
    check(ctx, z, [0, 4], 256, np.zeros(4))
    z[:] = 3.0  # ties everywhere but for a few
    z[1, 7::1000] = 3.5
    check(ctx, z, [0, 4], 256, np.zeros(4), exact_ids=True)


def test_in_a_graph_and_on_another_stream():
    from paper_2510_24051_amd import Pie
    m = W.ModelDesc(hidden=128, n_q_heads=2, n_kv_heads=2, head_dim=64, mlp_dim=256, vocab=32000, page_size=16, rms_eps=1e-5, rope_theta=1e4, n_layers=1)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a = Pie(m, 4, 4, max_batch_tokens=4, max_batch_requests=4, max_dist_rows=16, stream=s1)
    b = Pie(m, 4, 4, max_batch_tokens=4, max_batch_requests=4, max_dist_rows=16, stream=s2)
    z, scores = logits(16, 32000, torch.float32, 1), torch.zeros(16, device="cuda")
    outs = [[torch.zeros((4, 8), dtype=torch.int32, device="cuda") for _ in range(2)] + [torch.zeros((4, 8), device="cuda")] for _ in range(2)]
    torch.cuda.synchronize()
    graphs = []
    for ctx, s, o in ((a, s1, outs[0]), (b, s2, outs[1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.beam_select_async(z, [0, 4, 8, 12, 16], 8, *o, scores=scores)
        graphs.append(g)
    for replay in range(4):
        z.copy_(logits(16, 32000, torch.float32, 50 + replay))
        scores.copy_(torch.randn(16, device="cuda"))
        torch.cuda.synchronize()
        for g, s in zip(graphs, (s1, s2)):  # both at once: workspaces are the contexts' own
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want = select(a, z, [0, 4, 8, 12, 16], 8, scores.cpu().numpy())
        for o in outs:
            for got, w in zip(o, want):
                assert np.array_equal(got.cpu().numpy(), w), replay
                got.zero_()


def test_from_embeds(ctx):
    """get_next_beams is the selection over the logits of get_next_dist."""
    from paper_2510_24051_amd import TAP_LOGITS, Pie
    m = W.ModelDesc(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_dim=512, vocab=4096, page_size=16, rms_eps=1e-5, rope_theta=1e4, n_layers=1)
    c = Pie(m, 4, 64, max_batch_tokens=64, max_batch_requests=4, max_dist_rows=64)
    head = W.make_head_weights(m, 5)
    c.load_head(head)
    rng = np.random.default_rng(5)
    c.embed_write(np.arange(64), O.bf16_encode(O.bf16_round(rng.standard_normal((64, 256)))))
    for n in (1, 6, 24, 64):
        ids, scores = rng.permutation(64)[:n], rng.standard_normal(n).astype(np.float32)
        fin = (rng.random(n) < 0.2).astype(np.uint8)
        indptr = [0, n // 3, n]
        b, v, s = c.get_next_beams(ids, indptr, 10, scores, fin, eos_token=17, temperature=0.75)
        z = c.read_tap(TAP_LOGITS, n)
        wb, wv, ws = select(c, torch.from_numpy(z).cuda(), indptr, 10, scores, fin, 17, 0.75)
        assert np.array_equal(b, wb) and np.array_equal(v, wv) and np.array_equal(s, ws)
        emb = O.EmbedPool(64, 256)
        emb.write(np.arange(64), c.embed_read(np.arange(64)))
        zo = O.logits_from_embeds(m, head, emb, ids, round_intermediates=True)
        _, _, so = O.beam_select(zo, indptr, 10, scores, fin, 17, 0.75)
        np.testing.assert_allclose(s, so, atol=4e-3)  # logits within 1e-3, twice, over 0.75


def test_groups_without_any_beam(ctx):
    b, v, s = select(ctx, torch.empty((0, 1000), device="cuda"), [0, 0, 0], 3)
    assert (b == -1).all() and (v == -1).all() and np.isneginf(s).all()


def test_what_lies_behind_the_outputs_stays(ctx):
    z = logits(8, 3000, torch.float32, 2)
    room = [torch.full((64,), 77, dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.float32)]
    torch.cuda.synchronize()
    ctx.beam_select_async(z, [0, 3, 8], 5, *[r[20:30].view(2, 5) for r in room])
    ctx.synchronize()
    for r in room:
        assert (r[:20] == 77).all() and (r[30:] == 77).all() and (r[20:30] != 77).all()


def test_wrong_tensors_are_refused(ctx):
    o = [torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.zeros((1, 4), device="cuda")]
    z = torch.zeros((2, 64), device="cuda")
    bad = [dict(logits=z.t()), dict(logits=z.double()), dict(logits=z[:1]), dict(logits=z.cpu()), dict(out_scores=o[0]), dict(out_beams=o[0][:, :3]),
           dict(scores=torch.zeros(3, device="cuda")), dict(scores=torch.zeros(2, device="cuda").double()), dict(finished=torch.zeros(2, device="cuda"))]
    for change in bad:
        args = dict(logits=z, group_indptr=[0, 2], n_out=4, out_beams=o[0], out_tokens=o[1], out_scores=o[2])
        args.update(change)
        with pytest.raises(ValueError):
            ctx.beam_select_async(**args)


@pytest.mark.parametrize("V", [300, 40000])
@pytest.mark.parametrize("n", [15, 16, 17, 255, 256, 257])
def test_as_many_groups_as_a_launch_names(ctx, V, n):
    indptr = np.concatenate([[0], np.cumsum(np.arange(n) % 2 if n > 20 else np.full(n, 2))])
    check(ctx, logits(int(indptr[-1]), V, torch.bfloat16, n), indptr, 3, np.random.default_rng(n).standard_normal(int(indptr[-1])))
