"""A decoder layer of microscaled weights through pie_forward: every stage against the public operators (bit for bit, from the same inputs) and
against the oracle in 64 bits from the GPU's own input of that stage."""
import copy

import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx
from oracle import pie_oracle as O
from gpu_helpers import assert_close, dec
from test_gpu_mx import NORM_REL, check_computed, device_rows, rows_of, sum_error

pytestmark = pytest.mark.gpu

NAMES = ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown")


def quantised(weights):
    """(the layer with MxRows, the same layer's weights as values)."""
    mxw, vals = copy.copy(weights), {}
    for n in NAMES:
        r, v = device_rows(dec(getattr(weights, n)), "mxfp4")
        setattr(mxw, n, r)
        vals[n] = v
    return mxw, vals


def make(w, tokens=None, **kw):
    from paper_2510_24051_amd import Pie
    b = w.batch
    ctx = Pie(w.model, w.n_kv_pages, w.n_embeds, max_batch_tokens=tokens or b.n_tokens, max_batch_requests=b.n_requests, max_dist_rows=4, **kw)
    ctx.embed_write(b.in_embed_ids, w.embed_bits)
    for l in range(kw.get("n_layers", 1)):
        if len(w.prior.page_ids):
            ctx.kv_write(l, w.prior.page_ids, w.prior.slots, w.prior.k_bits, w.prior.v_bits)
    return ctx


def workload(name, hidden, hq, hkv, d, mlp, reqs, seed, page=16, mask=None):
    m = W.ModelDesc(hidden=hidden, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, mlp_dim=mlp, vocab=0, page_size=page, rms_eps=1e-5, rope_theta=1e4, n_layers=1)
    pages = sum((a + b + page - 1) // page for a, b in reqs) + 3
    return W.build_workload(name, m, [W.RequestSpec(a, b) for a, b in reqs], n_kv_pages=pages, seed=seed, std=0.05)


CASES = {"one_token": (256, 4, 2, 64, 512, [(1, 5)]), "odd_widths": (288, 8, 2, 64, 352, [(1, 40), (3, 0), (1, 17)]),
         "mixed": (256, 4, 2, 64, 512, [(32, 10), (1, 30), (1, 1), (70, 0)]), "wide": (1024, 8, 2, 128, 2048, [(1, 100)] * 20 + [(130, 20)]),
         "prompts": (512, 8, 8, 64, 1536, [(300, 0), (1, 64), (250, 16)]), "split": (512, 64, 8, 64, 4096, [(1, 20)] * 41)}


@pytest.mark.parametrize("case", list(CASES))
def test_layer_stage_by_stage(case):
    w = workload(case, *CASES[case], seed=len(case))
    m, b, T = w.model, w.batch, w.batch.n_tokens
    ctx = make(w)
    mxw, v = quantised(w.weights)
    ctx.load_layer_mx(0, mxw)
    pb = ctx.batch_create(b)
    ctx.forward(0, pb)
    ctx.synchronize()
    from paper_2510_24051_amd import TAP_ACT, TAP_ATTN, TAP_Q, TAP_RESID
    q_bits, attn_bits, h, act = ctx.read_tap(TAP_Q, T), ctx.read_tap(TAP_ATTN, T), ctx.read_tap(TAP_RESID, T), dec(ctx.read_tap(TAP_ACT, T))
    dev = lambda bits: torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
    gain = lambda bits: dev(np.ascontiguousarray(bits))  # noqa: E731
    x = dev(w.embed_bits)
    Hq, Hkv, D, H, I = m.n_q_heads, m.n_kv_heads, m.head_dim, m.hidden, m.mlp_dim
    # norm, q, k, v with the operators; then the rotary step in 64 bits
    xn = rows_of("mxfp8", T, H)
    ctx.mx_norm(x, gain(w.weights.g1), xn)
    x64 = dec(w.embed_bits)
    check_computed(xn, mx.norm(x64, dec(w.weights.g1), m.rms_eps), NORM_REL, "norm 1")
    qkv = torch.empty((T, (Hq + 2 * Hkv) * D), dtype=torch.bfloat16, device="cuda")
    ctx.mx_product(xn, ctx.mx_weight([mxw.wq, mxw.wk, mxw.wv]), qkv)
    q = qkv[:, :Hq * D].double().cpu().numpy().reshape(T, Hq, D)
    assert_close(dec(q_bits).reshape(T, Hq, D), O.rope(q, b.positions, m.rope_theta), "q after the rotary step", max_abs=2.0 ** -8 * np.abs(q).max() * 2, mean_abs=2e-3)
    pages, slots = [], []
    for r in range(b.n_requests):
        n = b.tok_indptr[r + 1] - b.tok_indptr[r]
        j = np.arange(b.kv_len[r] - n, b.kv_len[r])
        pages += list(b.page_ids[b.page_indptr[r]:b.page_indptr[r + 1]][j // m.page_size])
        slots += list(j % m.page_size)
    k_bits, v_bits = ctx.kv_read(0, pages, slots)
    assert np.array_equal(v_bits.reshape(T, -1), qkv[:, (Hq + Hkv) * D:].contiguous().view(torch.int16).cpu().numpy().view(np.uint16))
    # attention from the pool's own keys and values
    kv = O.KvPool(w.n_kv_pages, m.page_size, Hkv, D)
    if len(w.prior.page_ids):
        kv.write(w.prior.page_ids, w.prior.slots, w.prior.k_bits, w.prior.v_bits)
    kv.write(np.array(pages), np.array(slots), k_bits, v_bits)
    for r in range(b.n_requests):
        t = np.arange(b.tok_indptr[r], b.tok_indptr[r + 1])
        L = int(b.kv_len[r])
        pg, j = b.page_ids[b.page_indptr[r]:b.page_indptr[r + 1]], np.arange(L)
        allowed = j[None] <= (L - len(t) + np.arange(len(t)))[:, None]
        o = O.masked_attention(dec(q_bits).reshape(T, Hq, D)[t], dec(kv.k_bits[pg[j // m.page_size], j % m.page_size]),
                               dec(kv.v_bits[pg[j // m.page_size], j % m.page_size]), allowed)
        assert_close(dec(attn_bits)[t].reshape(o.shape), o, f"attention of request {r}")
    # output projection onto the residual, second norm, gate and up, down: bit for bit
    a = rows_of("mxfp8", T, Hq * D)
    ctx.mx_quantise(dev(attn_bits), a)
    c = torch.empty((T, H), device="cuda")
    ctx.mx_product(a, ctx.mx_weight([mxw.wo]), c)
    aq = mx.requantised(dec(attn_bits))
    err = sum_error(aq, v["wo"], "mxfp8") + 2.0 ** -23 * np.abs(h)
    assert np.all(np.abs(h - (x64 + aq @ v["wo"].T)) <= err)
    assert np.all(np.abs(h - (x.float() + c).cpu().numpy()) <= err)
    h_dev = torch.from_numpy(h).cuda()
    hn, act_rows, act_out = rows_of("mxfp8", T, H), rows_of("mxfp8", T, I), torch.empty((T, I), device="cuda")
    ctx.mx_norm(h_dev, gain(w.weights.g2), hn)
    ctx.mx_swiglu(hn, ctx.mx_weight([mxw.wgate, mxw.wup], gated=True), act_rows)
    ctx.mx_dequantise(act_rows, act_out)
    assert np.array_equal(act_out.cpu().numpy(), act.astype(np.float32))
    stored = np.nonzero(b.out_embed_ids >= 0)[0]
    y = dec(ctx.embed_read(b.out_embed_ids[stored]))
    want = h[stored] + act[stored] @ v["wdown"].T
    assert np.all(np.abs(y - want) <= (sum_error(act[stored], v["wdown"], "mxfp8") + 2.0 ** -23 * np.abs(want)) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want))
    ctx.close()


@pytest.mark.parametrize("shape,reqs", [((256, 4, 2, 512), [(1, 20), (9, 3), (1, 1)]), ((512, 64, 8, 4096), [(1, 20)] * 41)])
def test_layers_of_both_kinds_in_one_model(shape, reqs):
    """forward_all over layers of both kinds in several orders, against the oracle.  The second shape's output and down projections are split over
    workgroups, and their sums left to the norm behind, in either kind of layer."""
    H, hq, hkv, I = shape
    dw = W.build_deep_workload("kinds", W.ModelDesc(hidden=H, n_q_heads=hq, n_kv_heads=hkv, head_dim=64, mlp_dim=I, vocab=1024, page_size=16, rms_eps=1e-5,
                                                    rope_theta=1e4, n_layers=4), [W.RequestSpec(*r) for r in reqs], n_kv_pages=256, seed=9)
    from paper_2510_24051_amd import Pie, mx_product_plan
    if I == 4096:
        assert mx_product_plan(41, H, I)["splits"] > 1 and mx_product_plan(41, H, hq * 64)["splits"] > 1
    w, b = dw.base, dw.base.batch
    m, T = w.model, b.n_tokens
    made = [quantised(lw) for lw in dw.layers]

    def context(kinds, tokens=T):
        ctx = Pie(m, w.n_kv_pages, w.n_embeds, max_batch_tokens=tokens, max_batch_requests=b.n_requests, n_layers=len(kinds))
        ctx.load_embedding(dw.table_bits)
        for l, kind in enumerate(kinds):
            (ctx.load_layer_mx(l, made[l][0]) if kind else ctx.load_layer(l, dw.layers[l]))
            if len(dw.priors[l].page_ids):
                ctx.kv_write(l, dw.priors[l].page_ids, dw.priors[l].slots, dw.priors[l].k_bits, dw.priors[l].v_bits)
        ctx.embed_txt(dw.token_ids, b.positions, b.in_embed_ids)
        return ctx

    stored = np.nonzero(b.out_embed_ids >= 0)[0]

    def oracle(kinds):
        """The model in 64 bits, with the roundings that each kind of layer has; and a bound of the root mean square error e of its rows.
        Rows that differ a little have activations of 8 bits that round either way: two quantisations of (nearly) one value are each off by an error
        that is spread evenly over a step (2^-3 to 2^-4 of the value), at most 2^-4 / sqrt(3) = 0.036 root mean square each, 0.051 together, and of 0.05
        times their rms is what a product makes of that.  (bf16: 2^-8.)  A branch of rms b adds that part of b to e, and what it makes of the
        error that its input had, relative to the input and at most doubled by the nonlinearity: e + (0.051 + 2 e / rms(x)) b."""
        x = dec(dw.table_bits[dw.token_ids])
        rms = lambda a: float(np.sqrt(np.mean(np.square(a))))  # noqa: E731
        e = 0.0
        for l, kind in enumerate(kinds):
            lw, v = dw.layers[l], made[l][1]
            xn = mx.norm(x, dec(lw.g1), m.rms_eps)
            xn = mx.requantised(xn) if kind else O.bf16_round(xn)
            pick = lambda n: v[n] if kind else dec(getattr(lw, n))  # noqa: E731
            q, k, vv = (O.bf16_round(xn @ pick(n).T).reshape(T, -1, m.head_dim) for n in ("wq", "wk", "wv"))
            q, k = (O.bf16_round(O.rope(t, b.positions, m.rope_theta)) for t in (q, k))
            kv = O.KvPool(w.n_kv_pages, m.page_size, m.n_kv_heads, m.head_dim)
            pr = dw.priors[l]
            if len(pr.page_ids):
                kv.write(pr.page_ids, pr.slots, pr.k_bits, pr.v_bits)
            attn = np.zeros((T, m.n_q_heads, m.head_dim))
            for r in range(b.n_requests):
                t = np.arange(b.tok_indptr[r], b.tok_indptr[r + 1])
                L, pg = int(b.kv_len[r]), b.page_ids[b.page_indptr[r]:b.page_indptr[r + 1]]
                j = np.arange(L)
                new = j[L - len(t):]
                kv.write(pg[new // m.page_size], new % m.page_size, O.bf16_encode(k[t]), O.bf16_encode(vv[t]))
                at = (pg[j // m.page_size], j % m.page_size)
                attn[t] = O.masked_attention(q[t], dec(kv.k_bits[at]), dec(kv.v_bits[at]), j[None] <= (L - len(t) + np.arange(len(t)))[:, None])
            attn = O.bf16_round(attn).reshape(T, -1)
            if kind:
                h, _, y = mx.layer_tail(x, attn, dec(lw.g2), v["wo"], v["wgate"], v["wup"], v["wdown"], m.rms_eps)
            else:
                h = x + attn @ dec(lw.wo).T
                hn = O.bf16_round(mx.norm(h, dec(lw.g2), m.rms_eps))
                y = h + O.bf16_round(O.silu(hn @ dec(lw.wgate).T) * (hn @ dec(lw.wup).T)) @ dec(lw.wdown).T
            for before, after in ((x, h), (h, y)):
                e += ((0.051 if kind else 2.0 ** -8) + 2 * e / rms(before)) * rms(after - before)
            x = y
        return x, e + 2.0 ** -8 / np.sqrt(3) * rms(x)

    for kinds in ((0, 1, 1, 0), (1, 0, 0, 1), (1, 1, 1, 1)):
        ctx = context(kinds)
        pb = ctx.batch_create(b)
        ctx.forward_all(pb)
        ctx.synchronize()
        bits = ctx.embed_read(b.out_embed_ids[stored])
        want, limit = oracle(kinds)
        err = dec(bits) - want[stored]
        print(f"    layers {kinds}: rms error {np.sqrt(np.mean(err ** 2)):.2e}, at most {limit:.2e}; rms of the rows {np.sqrt(np.mean(want ** 2)):.2f}")
        assert np.sqrt(np.mean(err ** 2)) <= limit and np.abs(err).max() <= 8 * limit
        ctx.embed_txt(dw.token_ids, b.positions, b.in_embed_ids)
        ctx.forward_all(pb)
        ctx.synchronize()
        assert np.array_equal(ctx.embed_read(b.out_embed_ids[stored]), bits)  # the same again
        ctx.close()


@pytest.mark.parametrize("kinds", [(0, 1), (1, 0), (1, 1)])
def test_sums_left_to_the_next_layer(kinds):
    """A layer whose down projection is split over workgroups leaves its sums to the first norm of the next.  Here that one's own output and down
    projections are 0, so its output is its input: the first layer's output, which pie_forward gives by itself, up to the order of the fp32 sums: within one
    step of bf16, and another one for few."""
    m = W.ModelDesc(hidden=512, n_q_heads=64, n_kv_heads=8, head_dim=64, mlp_dim=4096, vocab=1024, page_size=16, rms_eps=1e-5, rope_theta=1e4, n_layers=2)
    dw = W.build_deep_workload("left", m, [W.RequestSpec(1, 20)] * 41, n_kv_pages=256, seed=3)
    from paper_2510_24051_amd import Pie, mx_product_plan
    assert mx_product_plan(41, 512, 4096)["splits"] > 1
    w, b = dw.base, dw.base.batch
    zero = copy.copy(dw.layers[1])
    zero.wo, zero.wdown = np.zeros_like(zero.wo), np.zeros_like(zero.wdown)
    ctx = Pie(m, w.n_kv_pages, w.n_embeds, max_batch_tokens=b.n_tokens, max_batch_requests=b.n_requests, n_layers=2)
    for l, lw in enumerate((dw.layers[0], zero)):
        (ctx.load_layer_mx(l, quantised(lw)[0]) if kinds[l] else ctx.load_layer(l, lw))
        ctx.kv_write(l, dw.priors[l].page_ids, dw.priors[l].slots, dw.priors[l].k_bits, dw.priors[l].v_bits)
    ctx.load_embedding(dw.table_bits)
    stored = np.nonzero(b.out_embed_ids >= 0)[0]
    pb = ctx.batch_create(b)
    got = []
    for call in (lambda: ctx.forward(0, pb), lambda: ctx.forward_all(pb)):
        ctx.embed_txt(dw.token_ids, b.positions, b.in_embed_ids)
        call()
        ctx.synchronize()
        got.append(dec(ctx.embed_read(b.out_embed_ids[stored])))
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(got[0]), 2.0 ** -100))) - 7)
    d = np.abs(got[1] - got[0])
    print(f"    {kinds}: {np.mean(d > 0) * 100:.3f}% of the values differ")
    assert np.all(d <= 1.01 * step + 2e-5) and np.mean(d > 0) < 0.01


def test_reloading_and_both_kinds_in_turn():
    """A layer loaded as bf16, then microscaled, then bf16 again gives each time what a fresh context gives."""
    w = workload("reload", 256, 4, 2, 64, 512, [(1, 20), (5, 0)], seed=2)
    b, stored = w.batch, np.nonzero(w.batch.out_embed_ids >= 0)[0]
    mxw, _ = quantised(w.weights)

    def run(ctx):
        ctx.embed_write(b.in_embed_ids, w.embed_bits)
        pb = ctx.batch_create(b)
        ctx.forward(0, pb)
        ctx.synchronize()
        pb.destroy()
        return ctx.embed_read(b.out_embed_ids[stored])

    plain, scaled, both = make(w), make(w), make(w)
    plain.load_layer(0, w.weights)
    scaled.load_layer_mx(0, mxw)
    want = run(plain), run(scaled)
    assert not np.array_equal(*want)
    for kind in (0, 1, 0, 1, 1):
        (both.load_layer_mx(0, mxw) if kind else both.load_layer(0, w.weights))
        assert np.array_equal(run(both), want[kind])


def test_captured_layer():
    """forward of a microscaled layer in a graph, replayed with other input Embeds."""
    w = workload("graph", 512, 8, 2, 64, 1024, [(1, 60), (1, 7), (40, 3)], seed=4)
    b, stored = w.batch, np.nonzero(w.batch.out_embed_ids >= 0)[0]
    ctx = make(w)
    ctx.load_layer_mx(0, quantised(w.weights)[0])
    pb = ctx.batch_create(b)
    rng = np.random.default_rng(0)
    inputs = [W.normal_bf16(rng, w.embed_bits.shape) for _ in range(3)]

    def eager(bits):
        ctx.embed_write(b.in_embed_ids, bits)
        ctx.forward(0, pb)
        ctx.synchronize()
        return ctx.embed_read(b.out_embed_ids[stored])

    want = [eager(i) for i in inputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=ctx.stream):
        ctx.forward(0, pb)
    for i in (2, 0, 1, 2):
        ctx.embed_write(b.in_embed_ids, inputs[i])
        ctx.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(ctx.embed_read(b.out_embed_ids[stored]), want[i])
        assert np.array_equal(eager(inputs[1]), want[1])
