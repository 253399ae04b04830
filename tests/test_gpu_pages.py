"""Pages forked, saved, restored and compacted on the GPU, against the oracle's pools: bit for bit, except keys that are rotated,
whose one rounding to bf16 may fall to the other side."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import pie_oracle as O

pytestmark = pytest.mark.gpu

THETA = 1e4


def model(D=64, Hkv=2, P=16):
    return SimpleNamespace(hidden=128, n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=D, mlp_dim=256, vocab=0, page_size=P, rms_eps=1e-5, rope_theta=THETA)


class Both:
    """A context and the oracle's pools with the same contents."""

    def __init__(self, m, n_pages, layers, seed, stream=None):
        from paper_2510_24051_amd import Pie
        self.m, self.n_pages, self.layers = m, n_pages, layers
        self.ctx = Pie(m, n_pages, 1, max_batch_tokens=1, max_batch_requests=1, n_layers=layers, stream=stream)
        rng = np.random.default_rng(seed)
        shape = (n_pages, layers, 2, m.page_size, m.n_kv_heads, m.head_dim)
        bits = O.bf16_encode(O.bf16_round(rng.standard_normal(shape)))
        bits[0, 0, :, 0, 0, :8] = [0x7FC1, 0xFF80, 0x7F80, 0x8000, 0x0001, 0xFFFF, 0x0000, 0x7F7F]  # any bits pass through
        self.kvs = []
        for layer in range(layers):
            kv = O.KvPool(n_pages, m.page_size, m.n_kv_heads, m.head_dim)
            kv.k_bits[:], kv.v_bits[:] = bits[:, layer, 0], bits[:, layer, 1]
            self.kvs.append(kv)
        self.restore(np.arange(n_pages), bits)

    def tensor(self, bits):
        return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(self.ctx.device).view(torch.bfloat16)

    def restore(self, ids, bits):
        t = self.tensor(bits)
        torch.cuda.synchronize()
        self.ctx.restore_kvpage(ids, t)
        self.ctx.synchronize()

    def save(self, ids):
        m = self.m
        t = torch.zeros((len(ids), self.layers, 2, m.page_size, m.n_kv_heads, m.head_dim), dtype=torch.bfloat16, device=self.ctx.device)
        torch.cuda.synchronize()
        self.ctx.save_kvpage(ids, t)
        self.ctx.synchronize()
        return t.view(torch.int16).cpu().numpy().view(np.uint16)

    def same(self, what=""):
        got, want = self.save(np.arange(self.n_pages)), O.save_kvpage(self.kvs, np.arange(self.n_pages))
        assert np.array_equal(got, want), f"{what}: {np.argwhere(got != want)[:4].tolist()} of {np.sum(got != want)}"


SHAPES = [(64, 1, 16, 1), (64, 3, 32, 2), (128, 2, 16, 3), (128, 8, 32, 2)]  # head dim, kv heads, page size, layers


@pytest.mark.parametrize("D,Hkv,P,layers", SHAPES)
def test_saved_and_restored_pages_are_what_kv_read_and_kv_write_see(D, Hkv, P, layers):
    b = Both(model(D, Hkv, P), 11, layers, D + P)
    pages, slots = np.repeat(np.arange(11), P), np.tile(np.arange(P), 11)
    for layer in range(layers):
        k, v = b.ctx.kv_read(layer, pages, slots)
        assert np.array_equal(k.reshape(b.kvs[layer].k_bits.shape), b.kvs[layer].k_bits)
        assert np.array_equal(v.reshape(b.kvs[layer].v_bits.shape), b.kvs[layer].v_bits)
    new = np.random.default_rng(1).integers(0, 1 << 16, (2, P, Hkv, D)).astype(np.uint16)
    b.ctx.kv_write(layers - 1, np.full(P, 4), np.arange(P), new[0], new[1])
    b.kvs[layers - 1].k_bits[4], b.kvs[layers - 1].v_bits[4] = new
    ids = [4, 10, 0, 4]  # (a page may be saved twice)
    assert np.array_equal(b.save(ids), O.save_kvpage(b.kvs, ids))
    image = np.random.default_rng(2).integers(0, 1 << 16, (3, layers, 2, P, Hkv, D)).astype(np.uint16)
    b.restore([9, 2, 5], image)
    for layer, kv in enumerate(b.kvs):
        kv.k_bits[[9, 2, 5]], kv.v_bits[[9, 2, 5]] = image[:, layer, 0], image[:, layer, 1]
    b.same("restored")
    b.ctx.save_kvpage([], torch.empty((0, layers, 2, P, Hkv, D), dtype=torch.bfloat16, device=b.ctx.device))


def test_more_pages_than_a_launch_names():
    b = Both(model(64, 1, 16), 2500, 1, 5)
    b.same("all 2500")
    ids = np.random.default_rng(6).permutation(2500)
    image = b.save(ids)
    b.restore(ids[::-1], image)
    b.kvs[0].k_bits[ids[::-1]], b.kvs[0].v_bits[ids[::-1]] = image[:, 0, 0], image[:, 0, 1]
    b.same("scattered back")


@pytest.mark.parametrize("D,Hkv,P,layers", SHAPES)
@pytest.mark.parametrize("form", ["fan", "pairs", "rotation", "swap", "chain", "random", "long"])
def test_fork(D, Hkv, P, layers, form):
    n_pages = 600 if form == "long" else 40
    b = Both(model(D, Hkv, P), n_pages, layers, 7)
    rng = np.random.default_rng(len(form) + D)
    if form == "fan":
        src, dst = [3] * 35, [i for i in range(40) if i not in (3, 5, 6, 7, 8)]
    elif form == "pairs":
        src, dst = np.arange(20), np.arange(39, 19, -1)
    elif form == "rotation":
        src, dst = np.roll(np.arange(40), 1), np.arange(40)
    elif form == "swap":
        src, dst = [1, 2, 9, 4, 1, 2], [2, 1, 9, 5, 6, 7]  # a swap, a page onto itself, and copies of what is swapped
    elif form == "chain":
        src, dst = np.arange(39), np.arange(1, 40)
    else:
        dst = rng.permutation(n_pages)[:n_pages - 7]
        src = rng.integers(0, n_pages, len(dst))
    b.ctx.mask_kvpage([3], [0x00F0])
    O.mask_kvpage(b.kvs, [3], [0x00F0])
    b.ctx.fork_kvpage(src, dst)
    O.fork_kvpage(b.kvs, src, dst)
    b.same(form)
    b.ctx.fork_kvpage(dst, src) if len(set(np.asarray(src).tolist())) == len(src) else None  # and back, queued behind
    if len(set(np.asarray(src).tolist())) == len(src):
        O.fork_kvpage(b.kvs, dst, src)
    b.same(form + " back")


def bf16_step(x):
    return np.abs(x) * 2.0 ** -8


def compact_case(D, Hkv, P, layers, lens, keep, in_place, shift, seed):
    """keep(s, L, rng) -> bool [L].  Returns the context and pools after both have been compacted, and the new lengths."""
    rng = np.random.default_rng(seed)
    n_pages = [-(-L // P) + s % 2 for s, L in enumerate(lens)]
    spare = sum(n_pages) + 3
    b = Both(model(D, Hkv, P), 2 * spare, layers, seed)
    ids = rng.permutation(2 * spare).astype(np.int32)
    ip = np.concatenate([[0], np.cumsum(n_pages)]).astype(np.int32)
    table, visible = ids[:ip[-1]], [keep(s, L, rng) for s, L in enumerate(lens)]
    bits = np.zeros(len(table), np.uint32)
    for s, L in enumerate(lens):
        for j in range(L):
            bits[ip[s] + j // P] |= np.uint32(int(visible[s][j]) << (j % P))
    if len(table):
        b.ctx.mask_kvpage(table, bits)
        O.mask_kvpage(b.kvs, table, bits)
    kept = np.array([int(v.sum()) for v in visible], np.int32)
    shifts = np.concatenate([np.cumsum(v) - 1 - np.arange(len(v)) for v in visible] + [[]]).astype(np.int32) if shift else None
    dp = di = None
    if not in_place:
        dp = np.concatenate([[0], np.cumsum(-(-kept // P))]).astype(np.int32)
        di = ids[ip[-1]:ip[-1] + dp[-1]]
    args = dict(dst_page_indptr=dp, dst_page_ids=di, shifts=shifts)
    plain = [(kv.k_bits.copy(), kv.v_bits.copy()) for kv in b.kvs]
    n = b.ctx.compact_kvpage(ip, table, np.array(lens, np.int32), **args)
    want = O.compact_kvpage(b.kvs, ip, table, lens, THETA, **args)
    assert np.array_equal(n, kept) and np.array_equal(want, kept)
    return b, plain


def check_compacted(b):
    got, want = b.save(np.arange(b.n_pages)), O.save_kvpage(b.kvs, np.arange(b.n_pages))
    assert np.array_equal(got[:, :, 1], want[:, :, 1]), "V"
    same = got[:, :, 0] == want[:, :, 0]
    g, w = O.bf16_decode(got[:, :, 0][~same]), O.bf16_decode(want[:, :, 0][~same])
    assert np.array_equal(np.isnan(g), np.isnan(w))  # (infinities and NaN among the bits that are rotated)
    g, w = g[~np.isnan(g)], w[~np.isnan(w)]
    # both round a rotated key once; its two products of values up to 5 differ by 4 x 2^-24 x 5 at most, so where the roundings
    # differ they are one step apart, or tiny both
    assert np.all(np.abs(g - w) <= 2 * bf16_step(np.maximum(np.abs(g), np.abs(w))) + 40 * 2.0 ** -24)
    return float(np.mean(~same))


def half(s, L, rng):
    return rng.random(L) < 0.5


def window(s, L, rng):
    j = np.arange(L)
    return (j < 3) | (j >= L - 40)


FORMS = {
    "half": half, "window": window, "all": lambda s, L, rng: np.ones(L, bool), "none": lambda s, L, rng: np.zeros(L, bool),
    "last": lambda s, L, rng: np.arange(L) == L - 1, "most": lambda s, L, rng: rng.random(L) < 0.97,
    "but_first": lambda s, L, rng: np.arange(L) > 0, "pages": lambda s, L, rng: np.arange(L) // 32 % 2 == s % 2,
}


@pytest.mark.parametrize("D,Hkv,P,layers", SHAPES)
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("in_place,shift", [(True, False), (True, True), (False, False), (False, True)])
def test_compact(D, Hkv, P, layers, form, in_place, shift):
    lens = [1, 77, 0, 160, 33, 16, 259]
    b, plain = compact_case(D, Hkv, P, layers, lens, FORMS[form], in_place, shift, D + Hkv + len(form))
    differ = check_compacted(b)
    assert differ == 0.0 if not shift or form in ("all", "none") else differ < 0.01
    if form in ("all", "none") and in_place:
        assert all(np.array_equal(kv.k_bits, k) and np.array_equal(kv.v_bits, v) for kv, (k, v) in zip(b.kvs, plain))


def test_compact_a_long_context_in_place():
    b, _ = compact_case(128, 2, 16, 2, [20011], lambda s, L, rng: rng.random(L) < 0.6, True, True, 3)
    check_compacted(b)


def test_compacting_twice_moves_nothing_more():
    b, _ = compact_case(64, 2, 16, 1, [200], half, True, True, 4)
    n = int(half(0, 200, np.random.default_rng(0)).sum())
    first = b.save(np.arange(b.n_pages))
    table = np.arange(b.n_pages)[:8]
    b.ctx.mask_kvpage(table, np.full(8, 0xFFFF))
    assert b.ctx.compact_kvpage([0, 8], table, [128])[0] == 128 and n > 0
    assert np.array_equal(b.save(np.arange(b.n_pages)), first)


def test_a_far_shift_is_exact():
    """A shift of a million positions: the angle is taken in 64 bits."""
    b = Both(model(128, 2, 16), 4, 1, 12)
    sh = np.full(32, 1000003, np.int32)
    b.ctx.compact_kvpage([0, 2], [0, 1], [32], shifts=sh, dst_page_indptr=[0, 2], dst_page_ids=[2, 3])
    O.compact_kvpage(b.kvs, [0, 2], [0, 1], [32], THETA, shifts=sh, dst_page_indptr=[0, 2], dst_page_ids=[2, 3])
    got, want = b.save([2, 3])[:, 0, 0], O.save_kvpage(b.kvs, [2, 3])[:, 0, 0]
    ok = np.isfinite(O.bf16_decode(want)) & np.isfinite(O.bf16_decode(got))
    g, w = O.bf16_decode(got[ok]), O.bf16_decode(want[ok])
    moderate = np.abs(w) < 100
    assert ok.mean() > 0.99 and np.all(np.abs(g - w)[moderate] <= 2 * bf16_step(w)[moderate] + 40 * 2.0 ** -24 * 100)


def test_pages_behind_four_gigabytes():
    """Offsets of pages within a layer, of layers and of images pass 32 bits."""
    from paper_2510_24051_amd import Pie
    m = model(128, 8, 16)
    ctx = Pie(m, 70000, 1, max_batch_tokens=1, max_batch_requests=1, n_layers=2)  # 4.6 GB a layer
    rng = np.random.default_rng(9)
    bits = (rng.integers(0, 1 << 16, (6, 2, 2, 16, 8, 128)) & 0xBFFF).astype(np.uint16)  # (no infinities or NaN)

    def tensor(b):
        return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).to(ctx.device).view(torch.bfloat16)

    def read(ids):
        t = torch.empty((len(ids), 2, 2, 16, 8, 128), dtype=torch.bfloat16, device=ctx.device)
        torch.cuda.synchronize()
        ctx.save_kvpage(ids, t)
        ctx.synchronize()
        return t.view(torch.int16).cpu().numpy().view(np.uint16)

    far = [69999, 69990, 65537, 65536, 3, 66000]
    given = tensor(bits)
    torch.cuda.synchronize()
    ctx.restore_kvpage(far, given)
    assert np.array_equal(read(far), bits)
    k, v = ctx.kv_read(1, [69999, 3], [5, 6])
    assert np.array_equal(k, bits[[0, 4], 1, 0, [5, 6]]) and np.array_equal(v, bits[[0, 4], 1, 1, [5, 6]])
    ctx.fork_kvpage([69999, 3, 65536], [65536, 69999, 68000])  # (65536 first goes to 68000)
    assert np.array_equal(read([65536, 69999, 68000, 3]), bits[[0, 4, 3, 4]])
    ctx.mask_kvpage([69990, 66000], [0xF00F, 0x00FF])
    assert ctx.compact_kvpage([0, 2], [69990, 66000], [32])[0] == 16
    keep = np.concatenate([bits[1][:, :, [0, 1, 2, 3, 12, 13, 14, 15]], bits[5][:, :, :8]], axis=2)
    assert np.array_equal(read([69990])[0], keep)
    ctx.close()


def test_shared_pages():
    """Sequences on one prefix: compacted into pages of their own, and in place where the prefix stays as it is."""
    for P in (16, 32):
        b = Both(model(64, 2, P), 40, 2, P)
        prefix, own = [3, 4, 5], [[10, 11], [12, 13], [14, 15]]
        lens = [4 * P, 5 * P - 3, 5 * P]
        b.ctx.mask_kvpage([4, 11, 12, 13, 14], [0x0F0F0F0F, 0xFF00FF00, 0x1, 0xAAAAAAAA, 0x0])
        O.mask_kvpage(b.kvs, [4, 11, 12, 13, 14], [0x0F0F0F0F, 0xFF00FF00, 0x1, 0xAAAAAAAA, 0x0])
        ip, ids = [0, 5, 10, 15], np.concatenate([prefix + o for o in own])
        dp, di = [0, 5, 10, 15], np.arange(20, 35)
        for args in (dict(dst_page_indptr=dp, dst_page_ids=di), dict(dst_page_indptr=dp, dst_page_ids=di, shifts=np.arange(sum(lens)) % 5 - 2)):
            n = b.ctx.compact_kvpage(ip, ids, lens, **args)
            assert np.array_equal(n, O.compact_kvpage(b.kvs, ip, ids, lens, THETA, **args))
            check_compacted(b)
            b.restore(di, O.save_kvpage(b.kvs, di))
        b.ctx.mask_kvpage([4], [0xFFFFFFFF])
        O.mask_kvpage(b.kvs, [4], [0xFFFFFFFF])
        n = b.ctx.compact_kvpage(ip, ids, lens)
        assert np.array_equal(n, O.compact_kvpage(b.kvs, ip, ids, lens, THETA))
        b.same("in place behind a shared prefix")


def test_a_compaction_is_refused_in_a_capture_and_does_not_end_it():
    from paper_2510_24051_amd import PieError
    s = torch.cuda.Stream()
    b = Both(model(64, 2, 16), 16, 1, 2, stream=s)
    b.ctx.mask_kvpage([0], [0xFFF0])
    O.mask_kvpage(b.kvs, [0], [0xFFF0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        b.ctx.fork_kvpage([1], [2])
        with pytest.raises(PieError) as e:
            b.ctx.compact_kvpage([0, 2], [0, 1], [32])
        assert e.value.status == -6
    with torch.cuda.stream(s):
        g.replay()
    s.synchronize()
    O.fork_kvpage(b.kvs, [1], [2])
    b.same("the capture's fork")
    assert b.ctx.compact_kvpage([0, 2], [0, 1], [32])[0] == 28
    O.compact_kvpage(b.kvs, [0, 2], [0, 1], [32], THETA)
    b.same("and the compaction behind it")


def test_wrong_images_are_refused():
    b = Both(model(64, 2, 16), 8, 2, 3)
    good = torch.zeros((2, 2, 2, 16, 2, 64), dtype=torch.bfloat16, device=b.ctx.device)
    for image in (good[:1], good[:, :1], good.float(), good.cpu(), good.transpose(4, 5), good[..., :32], good[..., 0]):
        for call in (b.ctx.save_kvpage, b.ctx.restore_kvpage):
            with pytest.raises(ValueError):
                call([0, 1], image)
    with pytest.raises(ValueError):
        b.ctx.fork_kvpage([0, 1], [2])
    for bad in (dict(page_indptr=[0, 1, 2]), dict(kv_len=[3, 4]), dict(shifts=[1]), dict(dst_page_indptr=[0, 1]), dict(page_ids=[0, 1])):
        with pytest.raises(ValueError):
            b.ctx.compact_kvpage(**{**dict(page_indptr=[0, 1], page_ids=[0], kv_len=[5]), **bad})


def test_fork_save_and_restore_in_a_graph():
    """Captured once and replayed with eager calls in between; every replay does what the eager calls do."""
    s = torch.cuda.Stream()
    b = Both(model(128, 2, 16), 16, 2, 21, stream=s)
    m = b.m
    image = torch.zeros((4, 2, 2, 16, m.n_kv_heads, m.head_dim), dtype=torch.bfloat16, device="cuda")
    given = b.tensor(np.random.default_rng(3).integers(0, 0x7F00, tuple(image.shape[:1]) + tuple(image.shape[1:])).astype(np.uint16))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        b.ctx.fork_kvpage([0, 1, 2, 2], [1, 2, 0, 9])
        b.ctx.restore_kvpage([10, 11, 12, 13], given)
        b.ctx.save_kvpage([1, 0, 9, 12], image)
    bits = given.view(torch.int16).cpu().numpy().view(np.uint16)
    for replay in range(4):
        with torch.cuda.stream(s):
            g.replay()
        s.synchronize()
        O.fork_kvpage(b.kvs, [0, 1, 2, 2], [1, 2, 0, 9])
        for layer, kv in enumerate(b.kvs):
            kv.k_bits[10:14], kv.v_bits[10:14] = bits[:, layer, 0], bits[:, layer, 1]
        assert np.array_equal(image.view(torch.int16).cpu().numpy().view(np.uint16), O.save_kvpage(b.kvs, [1, 0, 9, 12])), replay
        b.ctx.fork_kvpage([5, 6], [6, 5])  # eager work between the replays
        O.fork_kvpage(b.kvs, [5, 6], [6, 5])
        image.zero_()
        torch.cuda.synchronize()
        b.same(f"replay {replay}")


@pytest.mark.parametrize("D,Hkv,P,layers", [(64, 1, 16, 1), (128, 2, 32, 1)])
@pytest.mark.parametrize("form,shift", [("half", False), ("half", True), ("most", False), ("window", True), ("pages", True)])
def test_compact_few_waves_in_place(D, Hkv, P, layers, form, shift):
    """Long contexts with few heads and layers: through scratch blocks, or side by side where a gap is long enough; short ones beside
    them go in order, and the last block is as full as it is."""
    b, _ = compact_case(D, Hkv, P, layers, [5003, 40, 1601, 3200], FORMS[form], True, shift, 31 + D)
    check_compacted(b)
    b2, _ = compact_case(D, Hkv, P, layers, [5003, 40, 1601, 3200], FORMS[form], False, shift, 32 + D)
    check_compacted(b2)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 160])
def test_lists_about_as_long_as_an_argument_block(n):
    b = Both(model(64, 1, 16), 2 * n + 1, 2, n)
    src, dst = np.arange(n), np.arange(2 * n, n, -1)
    b.ctx.fork_kvpage(src, dst)
    O.fork_kvpage(b.kvs, src, dst)
    b.same("one to one")
    b.ctx.fork_kvpage(np.roll(dst, 1), dst)
    O.fork_kvpage(b.kvs, np.roll(dst, 1), dst)
    b.same("turned")
    image = b.save(dst)
    assert np.array_equal(image, O.save_kvpage(b.kvs, dst))
    b.restore(src, image)
    for layer, kv in enumerate(b.kvs):
        kv.k_bits[src], kv.v_bits[src] = image[:, layer, 0], image[:, layer, 1]
    b.same("restored")
    lens = np.full(n, 13)
    assert (b.ctx.compact_kvpage(np.arange(n + 1), src, lens, dst_page_indptr=np.arange(n + 1), dst_page_ids=dst) == 13).all()
    O.compact_kvpage(b.kvs, np.arange(n + 1), src, lens, THETA, dst_page_indptr=np.arange(n + 1), dst_page_ids=dst)
    b.same("compacted")
