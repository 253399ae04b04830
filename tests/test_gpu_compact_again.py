"""A compacted table with the masks as the call left them: nothing of it moves again, and what is masked later is compacted once more."""
import numpy as np
import pytest

from oracle import pie_oracle as O
from test_gpu_pages import SHAPES, THETA, Both, check_compacted, model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hkv,P,layers", SHAPES)
@pytest.mark.parametrize("shift", [False, True])
@pytest.mark.parametrize("apart", [False, True])
def test_compacting_again(D, Hkv, P, layers, shift, apart):
    rng = np.random.default_rng(D + P + shift)
    lens = [200, 3, 5 * P, 77]
    n_pages = [-(-n // P) for n in lens]
    ip = np.concatenate([[0], np.cumsum(n_pages)])
    b = Both(model(D, Hkv, P), 2 * int(ip[-1]), layers, D)
    ids = rng.permutation(b.n_pages)
    table, into = ids[:ip[-1]], ids[ip[-1]:]

    def mask(pages, lengths, indptr):
        keep = [rng.random(n) < 0.6 for n in lengths]
        bits = np.zeros(len(pages), np.uint32)
        for s, k in enumerate(keep):
            for j in np.nonzero(k)[0]:
                bits[indptr[s] + j // P] |= np.uint32(1 << (j % P))
        b.ctx.mask_kvpage(pages, bits)
        O.mask_kvpage(b.kvs, pages, bits)
        return np.array([int(k.sum()) for k in keep])

    def compact(pages, lengths, **to):
        sh = np.arange(int(np.sum(lengths))) % 7 - 3 if shift else None
        n = b.ctx.compact_kvpage(ip, pages, lengths, shifts=sh, **to)
        assert np.array_equal(n, O.compact_kvpage(b.kvs, ip, pages, lengths, THETA, shifts=sh, **to))
        return n

    want = mask(table, lens, ip)
    n = compact(table, lens, **(dict(dst_page_indptr=ip, dst_page_ids=into) if apart else {}))
    assert np.array_equal(n, want)
    differ = check_compacted(b)
    assert differ < 0.01 if shift else differ == 0.0
    table = into if apart else table
    before = b.save(np.arange(b.n_pages))
    assert np.array_equal(b.ctx.compact_kvpage(ip, table, n), n)  # all that is left is visible and in its place
    assert np.array_equal(b.save(np.arange(b.n_pages)), before)
    if not shift:
        want = mask(table, n, ip)
        assert np.array_equal(compact(table, n), want)
        b.same("masked and compacted again")
