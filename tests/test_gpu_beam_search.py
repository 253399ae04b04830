"""The operators together, as a program that searches with beams uses them: a prompt, its last page forked for every beam, steps of
selection, page reorder and forward through all layers, then eviction of tokens with compaction, and pages swapped out and back."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import pie_oracle as O
from gpu_helpers import assert_close, dec

pytestmark = pytest.mark.gpu


def batch(tok, ins, outs, pos, tables, lens):
    return W.Batch(n_requests=len(lens), n_tokens=len(ins), tok_indptr=np.array(tok, np.int32), in_embed_ids=np.array(ins, np.int32),
                   out_embed_ids=np.array(outs, np.int32), positions=np.array(pos, np.int32),
                   page_indptr=np.concatenate([[0], np.cumsum([len(t) for t in tables])]).astype(np.int32),
                   page_ids=np.concatenate(tables).astype(np.int32), kv_len=np.array(lens, np.int32), mask_indptr=None, mask_words=None)


@pytest.mark.parametrize("P", [16, 32])
def test_a_search(P):
    from paper_2510_24051_amd import Pie
    m = W.ModelDesc(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_dim=512, vocab=1024, page_size=P, rms_eps=1e-5, rope_theta=1e4, n_layers=2)
    B, n_prompt, steps = 4, 2 * P + P // 2 + 3, P // 2 + 4  # the steps run over the end of a page
    rng = np.random.default_rng(P)
    table = O.bf16_encode(O.bf16_round(rng.standard_normal((m.vocab, m.hidden))))
    head = W.make_head_weights(m, 3, std=0.3)

    def context():
        c = Pie(m, 64, 128, max_batch_tokens=128, max_batch_requests=8, max_dist_rows=8, n_layers=2)
        for layer in range(2):
            c.load_layer(layer, W.make_layer_weights(m, 100 + layer, std=0.08))
        c.load_head(head)
        c.load_embedding(table)
        return c

    ctx = context()
    prompt = rng.integers(0, m.vocab, n_prompt)
    n_pages = -(-n_prompt // P)
    free = list(range(63, n_pages - 1, -1))
    ctx.embed_txt(prompt, np.arange(n_prompt), np.arange(n_prompt))
    ctx.forward_all(ctx.batch_create(batch([0, n_prompt], np.arange(n_prompt), [-1] * (n_prompt - 1) + [100], np.arange(n_prompt), [np.arange(n_pages)], [n_prompt])))
    # the first step: one row, B beams
    b, tok, score = ctx.get_next_beams([100], [0, 1], B)
    assert b[0].tolist() == [0] * B
    # full pages are shared, the last one is everybody's own
    tables = [list(range(n_pages)) for _ in range(B)]
    for i in range(1, B):
        tables[i][-1] = free.pop()
    ctx.fork_kvpage([n_pages - 1] * (B - 1), [t[-1] for t in tables[1:]])
    own_from = n_pages - 1
    words, total, length = [[int(t)] for t in tok[0]], score[0].copy(), n_prompt
    for step in range(steps):
        if length % P == 0:
            for t in tables:
                t.append(free.pop())
        length += 1
        ctx.embed_txt([w[-1] for w in words], [length - 1] * B, np.arange(B))
        ctx.forward_all(ctx.batch_create(batch(np.arange(B + 1), np.arange(B), 100 + np.arange(B), [length - 1] * B, tables, [length] * B)))
        b, tok, new = ctx.get_next_beams(100 + np.arange(B), [0, B], B, scores=total)
        # the selection from the same Embeds, by the oracle
        emb = O.EmbedPool(128, m.hidden)
        emb.write(100 + np.arange(B), ctx.embed_read(100 + np.arange(B)))
        z = O.logits_from_embeds(m, head, emb, 100 + np.arange(B), round_intermediates=True)
        _, _, want = O.beam_select(z, [0, B], B, total)
        np.testing.assert_allclose(new[0], want[0], atol=4e-3)
        each = total.astype(np.float64)[:, None] + z - np.log(np.exp(z).sum(1, keepdims=True))
        np.testing.assert_allclose(each[b[0], tok[0]], new[0], atol=4e-3)
        # every beam's own pages become its parent's, in place
        src = [tables[p][j] for p in b[0] for j in range(own_from, len(tables[0]))]
        dst = [tables[i][j] for i in range(B) for j in range(own_from, len(tables[0]))]
        ctx.fork_kvpage(src, dst)
        words, total = [words[p] + [int(t)] for p, t in zip(b[0], tok[0])], new[0].copy()
    # the best beam's words in a fresh context, as one prompt: the same keys and values, the same next candidates
    fresh = context()
    seq = np.concatenate([prompt, words[0][:-1]])
    n = len(seq)
    assert n == length
    pages = np.arange(len(tables[0]))
    fresh.embed_txt(seq, np.arange(n), np.arange(n))
    fresh.forward_all(fresh.batch_create(batch([0, n], np.arange(n), [-1] * (n - 1) + [100], np.arange(n), [pages], [n])))
    j = np.arange(n)
    for layer in range(2):
        k, v = ctx.kv_read(layer, np.array(tables[0])[j // P], j % P)
        k2, v2 = fresh.kv_read(layer, pages[j // P], j % P)
        for x, y in ((k, k2), (v, v2)):
            x, y = dec(x), dec(y)
            assert np.abs(x - y).max() <= 0.06 * max(1.0, np.abs(y).max()) and np.abs(x - y).mean() <= 4e-3
    # its first pages go out of the pool and come back elsewhere; then a third of its tokens is evicted and the rest compacted
    image = torch.empty((len(tables[0]), 2, 2, P, 2, 64), dtype=torch.bfloat16, device=ctx.device)
    ctx.save_kvpage(tables[0], image)
    back = [free.pop() for _ in tables[0]]
    ctx.restore_kvpage(back, image)
    stays = np.array([(i % 3 != 1) or i >= n - 4 for i in range(n)])
    bits = [sum(int(i >= n or stays[i]) << (i - p * P) for i in range(p * P, (p + 1) * P)) for p in range(len(back))]  # (slots to come too)
    ctx.mask_kvpage(back, bits)
    # one more token over the masked pages, and over the compacted ones: the same output
    ctx.embed_txt([5], [n], [0])
    one = lambda t, length: batch([0, 1], [0], [101], [n], [t], [length])  # noqa: E731
    if n % P == 0:
        back.append(free.pop())
    ctx.forward_all(ctx.batch_create(one(back, n + 1)))
    y = dec(ctx.embed_read([101]))
    kept = ctx.compact_kvpage([0, len(back)], back, [n])[0]
    assert kept == stays.sum()
    ctx.forward_all(ctx.batch_create(one(back[:-(-(kept + 1) // P)], kept + 1)))
    y2 = dec(ctx.embed_read([101]))
    assert_close(y, y2, "one token over masked and over compacted pages")
