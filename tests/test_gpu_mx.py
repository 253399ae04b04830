"""Microscaled rows on the GPU against the oracle in 64 bits.

Tolerances.  Quantisation of given values: none, every bit is the oracle's.  What is quantised from computed values y (the norm, the
SwiGLU) may differ from the oracle's quantisation of y by the computation's error: an element lies within half a step of y / scale, and
REL |y| more; a block's scale may be one step off where the largest of it is that near to a power of two.
  NORM_REL: h^2 rounded, 8 added in a thread, 6 levels in a wave, up to 16 waves, then division, root, reciprocal and two products: under
  32 roundings of 2^-24 on the sum (half of them on its root) and 6 behind it: 2^-19.
  Products: in fp32, of K / 8 sums of eight, an error of at most a unit 2^-23 of the running magnitude each; with 8-bit rows each of the
  eight products but the largest drops less than 2^-13 of the largest's power of two (the instruction's alignment)."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx
from oracle import pie_oracle as O
from test_host_mx import FORM_SIZES

pytestmark = pytest.mark.gpu

NORM_REL = 2.0 ** -19
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    from paper_2510_24051_amd import Pie
    return Pie(W.model_tiny(), 8, 8, max_batch_tokens=8, max_batch_requests=8)


def rows_of(form, rows, k, fill=0xAA, gap=0):
    """MxRows of `rows` rows, their elements and scales `gap` apart from the next row's, all bytes `fill`."""
    from paper_2510_24051_amd import MxRows
    w, s = k // (2 if form == "mxfp4" else 1), (k // 32 + 3) // 4 * 4
    e = torch.full((rows, w + 16 * gap), fill, dtype=torch.uint8, device="cuda")
    b = torch.full((rows, s + 4 * gap), fill, dtype=torch.uint8, device="cuda")
    r = MxRows(form, e[:, :w], b[:, :s])
    r.whole = e, b
    return r


def host(r):
    """Elements as values, scale bytes, and the bytes behind the scales."""
    b = r.scales.cpu().numpy()
    return mx.decode(r.elements.cpu().numpy(), r.format), b[:, :r.k // 32], b[:, r.k // 32:]


def check_gaps(r, fill=0xAA):
    for t, used in zip(r.whole, (r.elements.shape[1], r.scales.shape[1])):
        assert (t[:, used:] == fill).all(), "bytes between the rows were written"


def device_rows(values, form, gap=0, pad=0):
    """Given values, quantised by the oracle, on the device; `pad` is what stands behind the last scale."""
    e, b = mx.quantise(values, form)
    r = rows_of(form, values.shape[0], values.shape[1], fill=pad, gap=gap)
    r.elements.copy_(torch.from_numpy(mx.encode(e, form)))
    r.scales[:, :b.shape[1]] = torch.from_numpy(b).cuda()
    r.scales[:, b.shape[1]:] = pad
    return r, mx.values(e, b)


def awkward(rng, rows, k):
    """Values over many magnitudes: ties, zeros, denormals, the largest, whole blocks of zero."""
    x = rng.normal(size=(rows, k)) * np.exp2(rng.integers(-30, 30, size=(rows, k // 32)).repeat(32, 1))
    x[rng.random((rows, k)) < 0.1] = 0.0
    x[rng.random((rows, k // 32)).repeat(32, 1) < 0.05] = 0.0
    i = rng.integers(0, rows * k // 32, size=max(1, rows * k // 320))
    b = x.reshape(-1, 32)
    b[i] = np.round(b[i] / np.abs(b[i]).max(1, keepdims=True).clip(1e-30) * 32) / 4  # multiples of a quarter: many ties
    return x


def special(x, rng):
    """In place: infinities, NaN, denormals and the largest values, here and there."""
    for v in (np.inf, -np.inf, np.nan, 1e-45, -1e-40, 3.0e38, -0.0):
        for _ in range(2):
            x[rng.integers(x.shape[0]), rng.integers(x.shape[1])] = v
    return x


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,k,stride,offset", [(1, 32, 0, 0), (1, 64, 0, 0), (7, 96, 3, 1), (5, 4096, 8, 0), (3, 14336, 0, 0), (130, 160, 32, 4), (2, 28672, 1, 3),
                                                  (1000, 2048, 0, 0)])
def test_quantise(ctx, form, dtype, rows, k, stride, offset):
    rng = np.random.default_rng(rows * k + len(dtype))
    x = awkward(rng, rows, k)
    if dtype == "f16":
        x = np.clip(x, -6e4, 6e4)
    x = special(x, rng)
    wide = torch.full((rows * (k + stride) + offset,), float("nan"), dtype=TYPES[dtype], device="cuda")  # what lies between the rows is not looked at
    t = wide[offset:].view(rows, k + stride)[:, :k]
    t.copy_(torch.from_numpy(x).float())
    r = rows_of(form, rows, k, gap=offset)
    ctx.mx_quantise(t, r)
    e, b, pad = host(r)
    we, wb = mx.quantise(t.double().cpu().numpy(), form)
    assert np.array_equal(b, wb) and np.array_equal(e, we) and not pad.any()
    check_gaps(r)
    # and back: exact in fp32, rounded once in 16 bits
    for to in TYPES.values():
        out = torch.full((rows, k + stride), 7.0, dtype=to, device="cuda")
        ctx.mx_dequantise(r, out[:, :k])
        want = torch.from_numpy(mx.values(we, wb)).float().to(to)
        assert torch.equal(torch.nan_to_num(out[:, :k].cpu(), nan=-5.0), torch.nan_to_num(want, nan=-5.0)) and (out[:, k:] == 7.0).all()


def test_dequantise_every_code(ctx):
    for form in ("mxfp8", "mxfp4"):
        codes = np.arange(256, dtype=np.uint8).reshape(1, 256)
        n = 256 * (2 if form == "mxfp4" else 1)
        r = rows_of(form, 256, n)
        r.elements.copy_(torch.from_numpy(np.repeat(codes, 256, 0)))
        r.scales.copy_(torch.arange(256, dtype=torch.uint8)[:, None].expand(256, r.scales.shape[1]))
        out = torch.empty((256, n), device="cuda")
        ctx.mx_dequantise(r, out)
        with np.errstate(over="ignore", invalid="ignore"):
            want = mx.values(mx.decode(np.repeat(codes, 256, 0), form), np.repeat(np.arange(256, dtype=np.uint8)[:, None], n // 32, 1)).astype(np.float32)
        assert np.array_equal(out.cpu().numpy(), want, equal_nan=True)


def check_computed(r, y, rel, what, err=0.0):
    """r is y (64 bits) quantised, y computed with an error of rel |y| + err."""
    e, b, pad = host(r)
    wb = mx.scale_bytes(y, r.format)
    assert not pad.any()
    off = b.astype(int) - wb.astype(int)
    err = np.broadcast_to(err, y.shape)
    if off.any():  # next to a power of two
        rows, blocks = np.nonzero(off)
        yb = np.abs(y).reshape(y.shape[0], -1, 32)[rows, blocks]
        eb = (np.abs(yb) * rel + err.reshape(y.shape[0], -1, 32)[rows, blocks]).max(1)
        assert np.all(np.abs(off) <= 1) and np.all(wb[rows, blocks] < 255)
        lo, hi = mx.scale_bytes(np.maximum(yb.max(1) - eb, 0)[:, None].repeat(32, 1), r.format), mx.scale_bytes((yb.max(1) + eb)[:, None].repeat(32, 1), r.format)
        got = b[rows, blocks]
        assert np.all((lo[:, 0] <= got) & (got <= hi[:, 0])), f"{what}: scales off"
    s = np.repeat(mx.scales_of(b), 32, 1)
    v, top = y / s, mx.LARGEST[r.format]
    slack = np.abs(v) * rel + err / s
    near = np.maximum(mx.element_step(np.minimum(np.abs(v) + slack, top), r.format), 0)
    bad = np.abs(e - np.clip(v, -top, top)) > near / 2 + slack
    assert not bad.any(), f"{what}: {bad.sum()} elements off, e.g. {e[bad][:3]} for {v[bad][:3]}"
    return float((e != mx.quantise(y, r.format)[0]).mean())


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("rows,k,dtype,delta,stride", [(1, 32, "f32", "", 0), (3, 64, "bf16", "f16", 0), (2, 544, "f16", "bf16", 1), (157, 2048, "bf16", "", 0),
                                                       (64, 4096, "f32", "bf16", 4), (9, 8192, "f32", "f32", 0), (5, 5024, "bf16", "bf16", 8), (33, 4128, "f32", "f16", 3)])
def test_norm(ctx, form, rows, k, dtype, delta, stride):
    gen = torch.Generator(device="cuda").manual_seed(rows + k)
    view = lambda t: torch.randn((rows, k + stride), generator=gen, device="cuda").mul_(torch.logspace(-2, 2, rows, device="cuda")[:, None]).to(TYPES[t])[:, :k]  # noqa: E731
    x, d = view(dtype), view(delta) if delta else None
    gain = torch.randn(k + 1, generator=gen, device="cuda").bfloat16()[stride % 2:][:k]
    was = x.clone()
    h = torch.full((rows, k + stride), 3.0, dtype=TYPES[dtype], device="cuda")
    r = rows_of(form, rows, k, gap=1)
    ctx.mx_norm(x, gain, r, delta=d, h=h[:, :k])
    want_h = was if d is None else (was.float() + d.float()).to(was.dtype)
    assert torch.equal(h[:, :k], want_h) and (h[:, k:] == 3.0).all() and torch.equal(x, was)
    y = mx.norm(want_h.double().cpu().numpy(), gain.double().cpu().numpy(), ctx.model.rms_eps)
    check_computed(r, y, NORM_REL, f"norm {rows} x {k}")
    check_gaps(r)
    again = rows_of(form, rows, k)
    ctx.mx_norm(x, gain, again, delta=d, h=x)  # in place
    assert torch.equal(x, want_h) and torch.equal(again.elements, r.elements) and torch.equal(again.scales, r.scales)
    if d is not None and d.dtype == x.dtype:
        x.copy_(was)
        ctx.mx_norm(x, gain, again, delta=d, h=d)
        assert torch.equal(d, want_h) and torch.equal(x, was) and torch.equal(again.elements, r.elements)


def test_norm_of_zeros_and_nans(ctx):
    x = torch.zeros((4, 96), device="cuda")
    x[1, 5], x[2, 40] = float("nan"), float("inf")
    x[3] = 1.0
    r = rows_of("mxfp8", 4, 96)
    ctx.mx_norm(x, torch.ones(96, dtype=torch.bfloat16, device="cuda"), r)
    e, b, _ = host(r)
    assert not e[0].any() and not b[0].any()  # 0 / sqrt(eps)
    assert (b[1] == 255).all() and not e[1].any()  # the mean is NaN
    assert b[2].tolist() == [0, 255, 0] and not e[2].any()  # 1 / sqrt(inf) = 0: zeros, and NaN where the infinity is
    assert (b[3] == 119 - 1).all() or (b[3] == 119).all()


def test_norm_of_squares_that_32_bits_do_not_hold():
    """From 2^-70 (with an epsilon below their squares) to 2^120, alone and beside ordinary rows: the root is of the 64-bit mean, and may be a denormal
    of 32 bits, off by 2^-22 of it."""
    from paper_2510_24051_amd import Pie
    from types import SimpleNamespace
    m = W.model_tiny()
    own = Pie(SimpleNamespace(**{**{f: getattr(m, f) for f in ("hidden", "n_q_heads", "n_kv_heads", "head_dim", "mlp_dim", "vocab", "page_size", "rope_theta")},
                                 "rms_eps": 1e-44}), 8, 8, max_batch_tokens=8, max_batch_requests=8)
    for k in (64, 544, 4096):
        gen = torch.Generator(device="cuda").manual_seed(k)
        powers = torch.tensor([-70, -66, -60, -40, 0, 40, 62, 64, 70, 100, 120], device="cuda")
        x = torch.randn((len(powers), k), generator=gen, device="cuda").clamp(-4, 4) * torch.exp2(powers.float())[:, None]
        gain = torch.randn(k, generator=gen, device="cuda").bfloat16()
        r = rows_of("mxfp8", len(powers), k)
        own.mx_norm(x, gain, r)
        eps = float(np.float32(1e-44))
        check_computed(r, mx.norm(x.double().cpu().numpy(), gain.double().cpu().numpy(), eps), NORM_REL, f"norm of {k}")


# ---- past 32 bits ----------------------------------------------------------------------------------
@pytest.fixture
def large():
    yield
    torch.cuda.empty_cache()


def test_quantise_past_32_bits(ctx, large):
    """2^34 values: more than 2^31 pieces of eight, and bytes past 2^32 on both sides."""
    from paper_2510_24051_amd import MxRows
    k, n, times = 1 << 20, 1025, 16
    gen = torch.Generator(device="cuda").manual_seed(5)
    part = torch.randn((n, k), generator=gen, dtype=torch.bfloat16, device="cuda")
    want = MxRows.empty(n, k, "mxfp8")
    ctx.mx_quantise(part, want)
    x = torch.empty((n * times, k), dtype=torch.bfloat16, device="cuda")
    for i in range(times):
        x[i * n:(i + 1) * n] = part
    r = MxRows.empty(n * times, k, "mxfp8")
    assert n * times * k // 8 >= 1 << 31
    ctx.mx_quantise(x, r)
    back = torch.empty_like(part)
    ctx.mx_dequantise(want, back)
    x.zero_()
    ctx.mx_dequantise(r, x)
    for i in range(times):
        rows = slice(i * n, (i + 1) * n)
        assert torch.equal(r.elements[rows], want.elements) and torch.equal(r.scales[rows], want.scales) and torch.equal(x[rows], back)


def test_norm_of_the_most_rows(ctx, large):
    """2^24 rows of 256 threads each: 2^32."""
    from paper_2510_24051_amd import MxRows
    rows, k = 1 << 24, 544
    gen = torch.Generator(device="cuda").manual_seed(6)
    part = torch.randn((1 << 14, k), generator=gen, device="cuda").bfloat16()
    gain = torch.randn(k, generator=gen, device="cuda").bfloat16()
    want = MxRows.empty(1 << 14, k, "mxfp8")
    ctx.mx_norm(part, gain, want)
    x = part.repeat(1 << 10, 1)
    r = MxRows.empty(rows, k, "mxfp8")
    h = torch.zeros_like(x)
    ctx.mx_norm(x, gain, r, h=h)
    assert torch.equal(h, x)
    assert (r.elements.view(1 << 10, 1 << 14, k) == want.elements).all() and (r.scales.view(1 << 10, 1 << 14, -1) == want.scales).all()


@pytest.mark.parametrize("gated", [False, True])
def test_product_past_32_bits(ctx, large, gated):
    """More rows than one launch takes, and results past 2^32 bytes; every row is computed as it is among few others (whole numbers: exactly)."""
    from paper_2510_24051_amd import MxRows
    n, k, period = 4096, 32, 1536
    m = (1 << 20) + 300
    rng = np.random.default_rng(7)
    w, _ = weight_of(ctx, [rng.choice(WEIGHTS, size=(n, k)) for _ in range(1 + gated)], gated=gated)
    a, _ = device_rows(rng.choice([0.0, 1, -1, 2], size=(period, k)), "mxfp4")
    times = (m + period - 1) // period
    many = MxRows("mxfp4", a.elements.repeat(times, 1)[:m].contiguous(), a.scales.repeat(times, 1)[:m].contiguous())
    if gated:
        want, out = MxRows.empty(period, n, "mxfp8"), MxRows.empty(m, n, "mxfp8")
        ctx.mx_swiglu(a, w, want)
        ctx.mx_swiglu(many, w, out)
        pairs = [(out.elements, want.elements), (out.scales, want.scales)]
    else:
        want, out = (torch.empty((r, n), dtype=torch.bfloat16, device="cuda") for r in (period, m))
        ctx.mx_product(a, w, want)
        ctx.mx_product(many, w, out)
        pairs = [(out, want)]
    for got, one in pairs:
        whole = m // period * period
        assert (got[:whole].view(-1, *one.shape) == one).all() and torch.equal(got[whole:], one[:m - whole])


# ---- products ------------------------------------------------------------------------------------
def weight_of(ctx, parts, gated=False, gap=0, pad=0):
    """(handle, values [n, k]) of matrices given as values."""
    made = [device_rows(p, "mxfp4", gap=gap, pad=pad) for p in parts]
    return ctx.mx_weight([m[0] for m in made], gated=gated), [m[1] for m in made]


def sum_error(a, w, form):
    """Bound of a product's error [m, n]: see the head of this file."""
    k = a.shape[1]
    out = (k / 8 + 16) * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T)
    if form == "mxfp8":
        power = lambda v: np.where(v != 0, np.exp2(np.frexp(v)[1] - 1.0), 0.0)  # noqa: E731
        pa, pw = power(a), power(w)
        drop = np.zeros(out.shape)
        for g in range(0, k, 8):  # of eight products, seven drop less than 2^-13 of the largest's power of two
            drop += (pa[:, None, g:g + 8] * pw[None, :, g:g + 8]).max(-1)
        out += 7 * 2.0 ** -13 * drop
    return out


WHOLE = [(1, 32, 1), (1, 64, 32), (3, 96, 5), (17, 128, 33), (32, 160, 64), (33, 544, 257), (64, 4096, 96), (65, 256, 130), (129, 1056, 300), (200, 512, 288),
         (257, 2080, 520), (300, 320, 1000), (520, 96, 40), (700, 640, 260), (1030, 288, 515)]


def whole_rows(rng, rows, k, vals, form, gap, low=126):
    """Rows of elements out of vals and scales of 2^(low - 127) to four times that, with what could be read by mistake behind and between them."""
    e = rng.choice(np.array(vals, dtype=np.float64), size=(rows, k))
    b = rng.integers(low, low + 3, size=(rows, k // 32)).astype(np.uint8)
    r = rows_of(form, rows, k, fill=0x7F, gap=gap)  # (0x7F: NaN in E4M3, a huge scale behind the last one)
    r.elements.copy_(torch.from_numpy(mx.encode(e, form)))
    r.scales[:, :k // 32] = torch.from_numpy(b).cuda()
    r.scales[:, k // 32:] = 0xFF
    return r, mx.values(e, b)


ACTS, WEIGHTS = [0, 1, -1, 2, -2, 3, 4, -4], [0, 0, 1, -1, 2, -3, 4]


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("m,k,n", WHOLE)
def test_product_of_whole_numbers(ctx, form, m, k, n):
    """Small whole numbers and scales of 1/2 to 2: every sum is exact, so every bit of an fp32 result is the oracle's, whatever the order."""
    rng = np.random.default_rng(m * k + n)
    from paper_2510_24051_amd import MxRows
    a, av = whole_rows(rng, m, k, ACTS, form, 1)
    w, wv = whole_rows(rng, n, k, WEIGHTS, "mxfp4", 2)
    want = mx.product(av, wv)
    assert np.abs(av).max() * np.abs(wv).max() * k < 2 ** 22
    parts = [w] if n <= 40 else [MxRows("mxfp4", w.elements[i:j], w.scales[i:j]) for i, j in ((0, 7), (7, n - 33), (n - 33, n))]
    weight = ctx.mx_weight(parts)
    for dtype, stride, offset in ((torch.float32, 0, 0), (torch.float32, 1, 3), (torch.bfloat16, 0, 0), (torch.bfloat16, 5, 1), (torch.bfloat16, 8, 8)):
        flat = torch.full((m * (n + stride) + offset,), -9.0, dtype=dtype, device="cuda")
        c = flat[offset:].view(m, n + stride)
        ctx.mx_product(a, weight, c[:, :n])
        got = c[:, :n].double().cpu().numpy()
        wanted = want if dtype == torch.float32 else O.bf16_round(want)
        bad = got != wanted
        assert not bad.any(), f"{bad.sum()} of {bad.size} differ, first at {np.argwhere(bad)[0]}: {got[bad][0]} not {wanted[bad][0]}"
        assert (c[:, n:] == -9.0).all() and (flat[:offset] == -9.0).all(), "bytes outside the result were written"


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("m,k,n", [(2, 1 << 20, 33), (33, (1 << 18) + 32, 40), (300, 1 << 17, 64)])
def test_product_of_long_rows(ctx, form, m, k, n):
    """As above; most weights are 0, so that sums stay exact."""
    rng = np.random.default_rng(m + k)
    a, av = whole_rows(rng, m, k, ACTS, form, 1)
    w, wv = whole_rows(rng, n, k, WEIGHTS + [0] * 150, "mxfp4", 0)
    assert (np.abs(av) @ np.abs(wv).T).max() < 2 ** 22
    out = torch.empty((m, n), device="cuda")
    ctx.mx_product(a, ctx.mx_weight([w]), out)
    assert np.array_equal(out.double().cpu().numpy(), mx.product(av, wv))


@pytest.mark.parametrize("gated,form,m,k,n", FORM_SIZES)
def test_every_form(ctx, gated, form, m, k, n):
    """Every form that a product is taken in (test_host_mx.py has the list and sees that it is whole): exact sums as above."""
    rng = np.random.default_rng(m + k + n)
    a, av = whole_rows(rng, m, k, ACTS, form, 1)
    parts = [whole_rows(rng, n, k, WEIGHTS, "mxfp4", 1, 126 if not gated else 120) for _ in range(2 if gated else 1)]
    weight = ctx.mx_weight([p[0] for p in parts], gated=gated)
    sums = [mx.product(av, p[1]) for p in parts]
    if gated:
        r = rows_of("mxfp8", m, n, gap=1)
        ctx.mx_swiglu(a, weight, r)
        check_computed(r, O.silu(sums[0]) * sums[1], 2.0 ** -21 * (1 + np.abs(sums[0])), f"gated {m} x {k} x {n}")
        check_gaps(r)
    else:
        c = torch.full((m, n + 4), -9.0, device="cuda")
        ctx.mx_product(a, weight, c[:, :n])
        assert np.array_equal(c[:, :n].cpu().numpy(), sums[0].astype(np.float32)) and (c[:, n:] == -9.0).all()
        h = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        ctx.mx_product(a, weight, h)
        assert np.array_equal(h.double().cpu().numpy(), O.bf16_round(sums[0]))


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("m,k,n", [(1, 14336, 64), (5, 4096, 96), (40, 2048, 200), (130, 1024, 64), (600, 512, 96)])
def test_product(ctx, form, m, k, n):
    rng = np.random.default_rng(m + k + n)
    x = rng.normal(size=(m, k)) * np.exp(rng.normal(size=k))
    a, av = device_rows(x, form)
    weight, (wv,) = weight_of(ctx, [rng.normal(size=(n, k)) * k ** -0.5])
    want, err = mx.product(av, wv), sum_error(av, wv, form)
    c = torch.empty((m, n), device="cuda")
    ctx.mx_product(a, weight, c)
    d = np.abs(c.double().cpu().numpy() - want)
    print(f"    {form} {m} x {k} x {n}: error {np.linalg.norm(d) / np.linalg.norm(want):.2e} of the result, at most {np.max(d / err):.3f} of the bound")
    assert np.all(d <= err)
    h = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    ctx.mx_product(a, weight, h)
    assert np.all(np.abs(h.double().cpu().numpy() - want) <= err + 2.0 ** -8 * (np.abs(want) + err))


def test_product_of_nan_blocks(ctx):
    """A NaN block makes its row (or the column of its weight row) NaN and nothing else."""
    rng = np.random.default_rng(5)
    for form in ("mxfp8", "mxfp4"):
        for m in (6, 300):
            a, av = device_rows(rng.normal(size=(m, 256)), form)
            b, bv = device_rows(rng.normal(size=(70, 256)), "mxfp4")
            a.scales[2, 5], b.scales[33, 0] = 255, 255
            c = torch.empty((m, 70), device="cuda")
            ctx.mx_product(a, ctx.mx_weight([b]), c)
            got = c.cpu().numpy()
            want = np.zeros((m, 70), bool)
            want[2], want[:, 33] = True, True
            assert np.array_equal(np.isnan(got), want)
            assert np.all((np.abs(got - av @ bv.T) <= sum_error(av, bv, form))[~want])


GATED = [(1, 32, 32), (2, 96, 64), (20, 256, 96), (33, 160, 512), (64, 1024, 288), (100, 512, 160), (300, 416, 320), (600, 64, 256)]


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("out", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("m,k,n", GATED)
def test_swiglu(ctx, form, out, m, k, n):
    rng = np.random.default_rng(m + k + n)
    a, av = device_rows(rng.normal(size=(m, k)), form, gap=1, pad=0xFF)
    weight, (g, u) = weight_of(ctx, [rng.normal(size=(n, k)) * 1.5 * k ** -0.5 for _ in range(2)], gated=True, gap=1, pad=0xFF)
    r = rows_of(out, m, n, gap=1)
    ctx.mx_swiglu(a, weight, r)
    zg, zu = mx.product(av, g), mx.product(av, u)
    eg, eu = sum_error(av, g, form), sum_error(av, u, form)
    # silu's slope is at most 1.1; exp, the sum, the quotient and the product: six roundings, and two units of exp
    err = 1.1 * eg * (np.abs(zu) + eu) + np.abs(O.silu(zg)) * eu
    flips = check_computed(r, mx.swiglu(av, g, u), 2.0 ** -21 * (1 + np.abs(zg)), f"swiglu {m} x {k} x {n}", err)
    print(f"    {form} -> {out} {m} x {k} x {n}: {flips:.2e} of the elements differ")
    check_gaps(r)


def test_swiglu_far_out(ctx):
    """Gates far below zero give zeros, far above the up value: no overflow, no NaN."""
    x = np.zeros((2, 32))
    x[:, 0] = [1.0, -1.0]
    a, av = device_rows(x, "mxfp8")
    g, u = np.zeros((32, 32)), np.zeros((32, 32))
    g[:, 0], u[:, 0] = 1.5e4, 2.0
    weight, (gv, uv) = weight_of(ctx, [g, u], gated=True)
    r = rows_of("mxfp8", 2, 32)
    ctx.mx_swiglu(a, weight, r)
    e, b, _ = host(r)
    assert np.array_equal(mx.values(e, b)[0], mx.requantised(av @ gv.T * (av @ uv.T))[0]) and not mx.values(e, b)[1].any()


# ---- as a program uses them ------------------------------------------------------------------------
def test_strided_views_streams_and_capture(ctx):
    """norm, product, norm with its output as residual, gated product and product: on another stream than the tensors', and captured and replayed with
    other inputs, with eager calls between the replays."""
    H, I, m = 256, 320, 40
    rng = np.random.default_rng(11)
    gen = torch.Generator(device="cuda").manual_seed(3)
    wo, _ = weight_of(ctx, [rng.normal(size=(H, H)) * H ** -0.5])
    gu, _ = weight_of(ctx, [rng.normal(size=(I, H)) * H ** -0.5 for _ in range(2)], gated=True)
    down, _ = weight_of(ctx, [rng.normal(size=(H, I)) * I ** -0.5])
    gain = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    x, h = torch.empty((m, H), device="cuda"), torch.empty((m, H), device="cuda")
    a, act, d, y = rows_of("mxfp8", m, H), rows_of("mxfp8", m, I), torch.empty((m, H), dtype=torch.bfloat16, device="cuda"), torch.empty((m, H), device="cuda")

    def chain(c):
        c.mx_norm(x, gain, a)
        c.mx_product(a, wo, d)
        c.mx_norm(x, gain, a, delta=d, h=h)
        c.mx_swiglu(a, gu, act)
        c.mx_product(act, down, y)

    def fresh(seed):
        x.copy_(torch.randn((m, H), generator=gen.manual_seed(seed), device="cuda"))
        for t in (h, d, y):
            t.fill_(float("nan"))

    want = []
    for s in range(3):
        fresh(s)
        chain(ctx)  # (torch's current stream is another than the context's)
        want.append((h.clone(), y.clone(), act.elements.clone(), act.scales.clone()))
    assert torch.isfinite(want[0][1]).all() and not torch.equal(want[0][1], want[1][1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=ctx.stream):
        chain(ctx)
    elsewhere, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(elsewhere, stream=side):  # (the context's stream joins the capture)
        chain(ctx)
    for s, g in ((1, graph), (0, elsewhere), (2, graph), (2, elsewhere), (1, elsewhere), (1, graph)):
        fresh(s)
        g.replay()
        torch.cuda.synchronize()
        for got, w in zip((h, y, act.elements, act.scales), want[s]):
            assert torch.equal(got, w)
        fresh(0)
        chain(ctx)
        torch.cuda.synchronize()
        assert torch.equal(y, want[0][1])


def test_no_rows_and_what_the_binding_refuses(ctx):
    from paper_2510_24051_amd import MxRows, PieError
    w, _ = weight_of(ctx, [np.ones((40, 64))])
    g, _ = weight_of(ctx, [np.ones((32, 64))] * 2, gated=True)
    none, gain = MxRows.empty(0, 64, "mxfp8"), torch.ones(64, dtype=torch.bfloat16, device="cuda")
    ctx.mx_quantise(torch.empty((0, 64), device="cuda"), none)
    ctx.mx_dequantise(none, torch.empty((0, 64), device="cuda"))
    ctx.mx_norm(torch.empty((0, 64), device="cuda"), gain, none)
    ctx.mx_product(none, w, torch.empty((0, 40), device="cuda"))
    ctx.mx_swiglu(none, g, MxRows.empty(0, 32, "mxfp8"))
    a, x = rows_of("mxfp8", 2, 64), torch.ones((2, 64), device="cuda")
    out = torch.empty((2, 40), device="cuda")
    for call in (lambda: ctx.mx_quantise(x[:, :32], a), lambda: ctx.mx_quantise(x.double(), a), lambda: ctx.mx_quantise(x.cpu(), a), lambda: ctx.mx_quantise(x.T, a),
                 lambda: ctx.mx_norm(x, gain.float(), a), lambda: ctx.mx_norm(x, gain[:32], a), lambda: ctx.mx_norm(x, gain, a, h=x.bfloat16()),
                 lambda: ctx.mx_norm(x, gain, a, delta=x[:1]), lambda: ctx.mx_product(a, w, out[:, :39]), lambda: ctx.mx_product(a, w, out.half()),
                 lambda: ctx.mx_product(rows_of("mxfp8", 2, 32), w, out), lambda: ctx.mx_swiglu(a, g, rows_of("mxfp8", 2, 64)), lambda: ctx.mx_weight([]),
                 lambda: ctx.mx_weight([rows_of("mxfp4", 4, 64), rows_of("mxfp4", 4, 32)]), lambda: ctx.mx_product(MxRows.empty(2, 64, "mxfp8", "cpu"), w, out)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ctx.mx_product(a, g, torch.empty((2, 32), device="cuda")), lambda: ctx.mx_weight([rows_of("mxfp8", 4, 64)]),
                 lambda: ctx.mx_weight([rows_of("mxfp4", 33, 64)] * 2, gated=True)):
        with pytest.raises(PieError) as e:
            call()
        assert e.value.status == -1
    other = type(ctx)(W.model_tiny(), 8, 8, max_batch_tokens=8, max_batch_requests=8)
    foreign, _ = weight_of(other, [np.ones((40, 64))])
    with pytest.raises(PieError) as e:
        ctx.mx_product(a, foreign, out)
    assert e.value.status == -1
    other.close()
    w.destroy()
    for gone in (foreign, w):
        with pytest.raises(ValueError):
            ctx.mx_product(a, gone, out)
