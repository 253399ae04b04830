"""forward_dist over microscaled layers, and layers of both kinds: what forward_all and get_next_dist give one after the other, bit for bit, and the
oracle's distribution of the Embeds that it stores."""
import numpy as np
import pytest

import workloads as W
from gpu_helpers import dec
from helpers import check_topk
from oracle import pie_oracle as O
from test_gpu_mx_layer import quantised

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kinds", [(1, 1), (0, 1), (1, 0)])
def test_forward_dist_of_microscaled_layers(kinds):
    from paper_2510_24051_amd import Pie, PieError
    dw = W.deep_tiny(n_layers=2)
    w, b = dw.base, dw.base.batch
    rows = w.dist_rows
    made = [quantised(lw)[0] for lw in dw.layers]

    def context():
        ctx = Pie(w.model, w.n_kv_pages, w.n_embeds, max_batch_tokens=b.n_tokens, max_batch_requests=b.n_requests, max_dist_rows=len(rows), n_layers=2)
        ctx.load_embedding(dw.table_bits)
        ctx.load_head(w.head)
        for l, kind in enumerate(kinds):
            (ctx.load_layer_mx(l, made[l]) if kind else ctx.load_layer(l, dw.layers[l]))
            if len(dw.priors[l].page_ids):
                ctx.kv_write(l, dw.priors[l].page_ids, dw.priors[l].slots, dw.priors[l].k_bits, dw.priors[l].v_bits)
        ctx.embed_txt(dw.token_ids, b.positions, b.in_embed_ids)
        return ctx

    ctx = context()
    pb = ctx.batch_create(b)
    ids1, p1 = ctx.forward_dist(pb, rows, w.top_k, 0.7)
    at = b.out_embed_ids[rows]
    bits = ctx.embed_read(at)
    ctx2 = context()
    ctx2.forward_all(ctx2.batch_create(b))
    ids2, p2 = ctx2.get_next_dist(at, w.top_k, 0.7)
    assert np.array_equal(ids1, ids2) and np.array_equal(p1, p2) and np.array_equal(bits, ctx2.embed_read(at))
    assert np.isfinite(dec(bits)).all() and dec(bits).any()
    probe = O.EmbedPool(w.n_embeds, w.model.hidden)
    probe.write(at, bits)
    oi, op, z = O.get_next_dist(w.model, w.head, probe, at, w.top_k, 0.7, round_intermediates=True)
    check_topk(ids1, p1, z / 0.7, oi, op)
    with pytest.raises(PieError):
        ctx.forward_dist(pb, [b.n_tokens], 4)
    ids3, p3 = ctx2.get_next_dist(at, w.top_k, 0.7)  # (the Embeds are as they were)
    assert np.array_equal(ids3, ids1) and np.array_equal(p3, p1)
