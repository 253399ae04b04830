"""CPU pins of the oracle's beam selection, page forks and compaction."""
import numpy as np
import pytest
import torch

from oracle import pie_oracle as O


def pool(rng, n_pages, P, H=2, D=64):
    kv = O.KvPool(n_pages, P, H, D)
    kv.k_bits[:] = O.bf16_encode(O.bf16_round(rng.standard_normal(kv.k_bits.shape)))
    kv.v_bits[:] = O.bf16_encode(O.bf16_round(rng.standard_normal(kv.v_bits.shape)))
    return kv


@pytest.mark.parametrize("beams,V,M", [(1, 7, 3), (4, 50, 9), (3, 200, 200)])
def test_beam_select_is_topk_of_the_flattened_group(beams, V, M):
    rng = np.random.default_rng(beams * V)
    z, s = rng.standard_normal((2 * beams, V)) * 3, rng.standard_normal(2 * beams)
    b, t, v = O.beam_select(z, [0, beams, 2 * beams], M, scores=s, temperature=0.7)
    each = torch.from_numpy(s)[:, None] + torch.log_softmax(torch.from_numpy(z) / 0.7, dim=1)
    for g in range(2):
        top = torch.topk(each[g * beams:(g + 1) * beams].reshape(-1), M)
        assert np.array_equal(b[g] * V + t[g], top.indices.numpy())
        np.testing.assert_allclose(v[g], top.values.numpy(), rtol=1e-12)


def test_beam_select_special_rows():
    z = np.array([[0.0, 1.0, np.nan, -np.inf], [5.0, 5.0, 5.0, 5.0], [-np.inf] * 4, [9.0, 0.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0], [np.inf, 0.0, 1.0, np.inf]])
    s = np.array([0.0, 0.0, 0.0, -0.5, -np.inf, 0.0])
    b, t, v = O.beam_select(z, [0, 5, 5, 6], 6, scores=s, finished=[0, 0, 0, 1, 0, 0], eos_token=3, largest=1e30)
    lse = np.log(1 + np.e)
    # row 0: 1 - lse = -0.313, -lse = -1.313; row 1: four times -1.386; row 3 finished: -0.5 at token 3
    assert b[0].tolist() == [0, 3, 0, 1, 1, 1] and t[0].tolist() == [1, 3, 0, 0, 1, 2]
    np.testing.assert_allclose(v[0], [1 - lse, -0.5, -lse] + [-np.log(4)] * 3)
    assert b[1].tolist() == [-1] * 6 and np.all(np.isneginf(v[1]))
    assert t[2][:2].tolist() == [0, 3] and np.allclose(v[2][:2], -np.log(2))


def test_fork_assigns_all_at_once():
    rng = np.random.default_rng(1)
    kv, before = pool(rng, 12, 16), None
    kv.visible[3, 5] = False
    before = kv.k_bits.copy()
    src, dst = [0, 1, 2, 3, 3, 7], [1, 2, 0, 4, 5, 7]
    O.fork_kvpage([kv], src, dst)
    for p in range(12):
        want = src[dst.index(p)] if p in dst else p
        assert np.array_equal(kv.k_bits[p], before[want])
    assert not kv.visible[4, 5] and not kv.visible[5, 5] and kv.visible[2, 5]


@pytest.mark.parametrize("P", [16, 32])
def test_attention_over_compacted_pages_is_attention_over_the_masked_ones(P):
    rng = np.random.default_rng(P)
    kv = pool(rng, 20, P)
    L, table = 5 * P - 3, rng.permutation(20)[:5]
    kv.visible[table] = rng.random((5, P)) < 0.4
    j = np.arange(L)
    allowed = kv.visible[table[j // P], j % P]
    q = rng.standard_normal((1, 2, 64))
    k, v = O.bf16_decode(kv.k_bits[table[j // P], j % P]), O.bf16_decode(kv.v_bits[table[j // P], j % P])
    want = O.masked_attention(q, k, v, allowed[None, :])
    n = O.compact_kvpage([kv], [0, 5], table, [L], 1e4)[0]
    assert n == allowed.sum()
    j = np.arange(n)
    assert kv.visible[table[:-(-n // P)]].all()
    k, v = O.bf16_decode(kv.k_bits[table[j // P], j % P]), O.bf16_decode(kv.v_bits[table[j // P], j % P])
    np.testing.assert_allclose(O.masked_attention(q, k, v, np.ones((1, n), bool)), want, rtol=1e-12, atol=1e-12)


def test_a_shifted_key_is_the_key_at_its_new_position():
    rng = np.random.default_rng(3)
    kv, plain = pool(rng, 4, 16), rng.standard_normal((40, 2, 64))
    pos = np.arange(40)
    kv.k_bits[pos // 16, pos % 16] = O.bf16_encode(O.bf16_round(O.rope(plain, pos, 1e4)))
    kv.visible[0, 3:] = False
    kv.visible[1] = False
    shifts = np.where(pos >= 32, -29, 0)
    n = O.compact_kvpage([kv], [0, 3], [0, 1, 2], [40], 1e4, shifts=shifts)[0]
    assert n == 11
    at = np.arange(n)
    got, want = O.bf16_decode(kv.k_bits[0, at]), O.rope(plain[np.r_[0:3, 32:40]], at, 1e4)
    assert np.abs(got - want).max() < 4 * 2 ** -8 * 2  # two roundings of values up to 4
