"""Sums of 8-bit microscaled rows with 4-bit weights, over the whole range of both kinds of element.

A product of two elements is a multiple of 2^-10 (2^-9 of E4M3, 2^-1 of E2M1) and at most 2688 (448 * 6).  Rows of which at most five elements are not 0 then
have sums of magnitude below 2^14 at every point on the way: 24 bits, which fp32 holds.  Whatever order they are added in, 32-bit sums of them are
the oracle's bit for bit, and sums that are kept to fewer bits anywhere are not.

Rows of any elements: a sum of K products is K / 8 sums of eight, whole, in each of two parts, and each is added to a running sum with an error of at most one unit in
its last place, 2^-23 of what the magnitudes add up to; up to 16 more additions join slices and splits."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx
from oracle import pie_oracle as O
from test_gpu_mx import check_computed, check_gaps, rows_of
from test_host_mx import FORM_SIZES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2510_24051_amd import Pie
    return Pie(W.model_tiny(), 8, 8, max_batch_tokens=8, max_batch_requests=8)


def codes(rng, shape, form):
    """Any element: the rows of E4M3 without its NaN."""
    if form == "mxfp4":
        return rng.integers(0, 16, size=shape)
    c = rng.integers(0, 127, size=shape)
    return c | (rng.integers(0, 2, size=shape) << 7)


def few_codes(rng, m, k):
    """Rows of five elements that are not 0: the largest binade beside any others among eight neighbours, and two somewhere."""
    c = np.zeros((m, k), np.int64)
    first = rng.integers(0, k // 8, size=m) * 8
    for r in range(m):
        near = first[r] + rng.choice(8, size=3, replace=False)
        far = rng.choice(k, size=2, replace=False)
        c[r, far] = codes(rng, 2, "mxfp8")
        c[r, near] = codes(rng, 3, "mxfp8")
        c[r, near[0]] = 0x70 + rng.integers(0, 15)  # 256 .. 448
    return c


def device(c, form, scales, gap=1):
    """(rows on the device, their values) of element codes and scale bytes [rows, k / 32]."""
    m, k = c.shape
    r = rows_of(form, m, k, fill=0x7F, gap=gap)
    stored = c.astype(np.uint8) if form == "mxfp8" else (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)
    r.elements.copy_(torch.from_numpy(stored))
    r.scales[:, :k // 32] = torch.from_numpy(scales.astype(np.uint8)).cuda()
    r.scales[:, k // 32:] = 0xFF
    return r, mx.values(mx.codes_values(form)[c], scales)


def ones(m, k, byte=127):
    return np.full((m, k // 32), byte, np.int64)


# (rows, k, n): one row to more than a tile, with ends inside tiles, stages and groups of stages; up to 16 rows in every form that they are taken in, split
# over workgroups and whole (test_host_mx_plans.py sees to it)
SIZES = [(1, 12288, 32), (9, 8192, 2816), (1, 1536, 16896), (1, 12288, 3296), (1, 32, 1), (1, 64, 40), (1, 512, 256), (5, 96, 33), (15, 1056, 64), (16, 2080, 96), (16, 4096, 700), (17, 1056, 64), (3, 8192, 32), (9, 4096, 8192), (31, 256, 130),
         (33, 544, 257), (64, 4096, 96), (129, 1056, 300), (300, 320, 520), (700, 640, 260), (1030, 288, 515)]
LISTED = [(m, k, n) for gated, form, m, k, n in FORM_SIZES if not gated and form == "mxfp8"]


@pytest.mark.parametrize("m,k,n", SIZES + LISTED)
def test_sums_of_few_elements_are_whole(ctx, m, k, n):
    rng = np.random.default_rng(m * 7 + k + n)
    a, av = device(few_codes(rng, m, k), "mxfp8", ones(m, k))
    w, wv = device(codes(rng, (n, k), "mxfp4"), "mxfp4", ones(n, k))
    want = mx.product(av, wv)
    assert (np.abs(av) @ np.abs(wv).T).max() < 2 ** 14
    weight, out = ctx.mx_weight([w]), torch.full((m, n + 3), -9.0, device="cuda")
    ctx.mx_product(a, weight, out[:, :n])
    got = out[:, :n].cpu().numpy()
    bad = got != want.astype(np.float32)
    assert not bad.any(), f"{bad.sum()} of {bad.size} sums differ, first at {np.argwhere(bad)[0]}: {got[bad][0]!r} not {want[bad][0]!r}"
    assert (out[:, n:] == -9.0).all()
    half = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    ctx.mx_product(a, weight, half)
    assert np.array_equal(half.double().cpu().numpy(), O.bf16_round(want))


# 4-bit rows: tiles with a rest behind them, and products split over workgroups
SIZES4 = [(2050, 512, 8192), (1, 8192, 32), (40, 14336, 512), (333, 14336, 96), (16, 4096, 700)]


@pytest.mark.parametrize("m,k,n", SIZES4)
def test_sums_of_4_bit_rows_are_whole(ctx, m, k, n):
    """Any elements: products are multiples of 1/4 and at most 36, sums of 14336 of them below 2^19."""
    rng = np.random.default_rng(m + k + n)
    a, av = device(codes(rng, (m, k), "mxfp4"), "mxfp4", ones(m, k))
    w, wv = device(codes(rng, (n, k), "mxfp4"), "mxfp4", ones(n, k))
    out = torch.full((m, n + 3), -9.0, device="cuda")
    ctx.mx_product(a, ctx.mx_weight([w]), out[:, :n])
    assert np.array_equal(out[:, :n].cpu().numpy(), mx.product(av, wv).astype(np.float32)) and (out[:, n:] == -9.0).all()


GATED_SIZES = [(1, 32, 32), (4, 512, 64), (16, 4096, 96), (16, 256, 4096), (17, 544, 64), (64, 1024, 288), (300, 416, 320), (600, 64, 256)]


@pytest.mark.parametrize("out", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("m,k,n", GATED_SIZES + [(m, k, n) for gated, form, m, k, n in FORM_SIZES if gated and form == "mxfp8"])
def test_gated_sums_of_few_elements_are_whole(ctx, out, m, k, n):
    """The same sums, of gates and ups; behind them only the activation's roundings (test_gpu_mx.py)."""
    rng = np.random.default_rng(m * 7 + k + n)
    a, av = device(few_codes(rng, m, k), "mxfp8", ones(m, k, 119))  # (gates of 0 to 52)
    parts = [device(codes(rng, (n, k), "mxfp4"), "mxfp4", ones(n, k)) for _ in range(2)]
    r = rows_of(out, m, n, gap=1)
    ctx.mx_swiglu(a, ctx.mx_weight([p[0] for p in parts], gated=True), r)
    gate, up = (mx.product(av, p[1]) for p in parts)
    check_computed(r, O.silu(gate) * up, 2.0 ** -21 * (1 + np.abs(gate)), f"gated {m} x {k} x {n}")
    check_gaps(r)


@pytest.mark.parametrize("m", [1, 16, 30, 300])
@pytest.mark.parametrize("k,n", [(32, 64), (64, 40), (256, 96), (544, 64)])
def test_sums_of_any_elements(ctx, m, k, n):
    """Within the bound of 32-bit sums (at the head of this file), scales a factor of up to 2^6 apart."""
    rng = np.random.default_rng(m + k + n)
    a, av = device(codes(rng, (m, k), "mxfp8"), "mxfp8", rng.integers(124, 131, size=(m, k // 32)))
    w, wv = device(codes(rng, (n, k), "mxfp4"), "mxfp4", rng.integers(124, 131, size=(n, k // 32)))
    out = torch.empty((m, n), device="cuda")
    ctx.mx_product(a, ctx.mx_weight([w]), out)
    d, bound = np.abs(out.double().cpu().numpy() - mx.product(av, wv)), (k / 4 + 16) * 2.0 ** -23 * (np.abs(av) @ np.abs(wv).T)
    print(f"    {m} x {k} x {n}: at most {np.max(d / bound):.3f} of the bound")
    assert np.all(d <= bound)


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("m", [2, 16, 40, 300])
def test_scales_at_the_ends_of_their_range(ctx, form, m):
    """Rows' scales of 2^-127 and 2^127 with weights' of the opposite kind: products as with scales of 1."""
    rng = np.random.default_rng(m)
    k, n = 256, 70
    c = few_codes(rng, m, k) if form == "mxfp8" else np.where(rng.random((m, k)) < 0.1, codes(rng, (m, k), form), 0)
    wc = codes(rng, (n, k), "mxfp4")
    for byte in (0, 1, 127, 253, 254):
        a, av = device(c, form, ones(m, k, byte))
        w, wv = device(wc, "mxfp4", ones(n, k, 254 - byte))
        out = torch.empty((m, n), device="cuda")
        ctx.mx_product(a, ctx.mx_weight([w]), out)
        assert np.array_equal(out.double().cpu().numpy(), mx.product(av, wv)), byte


@pytest.mark.parametrize("m", [1, 4, 16, 17, 300])
def test_nan_elements(ctx, m):
    """A NaN among E4M3 elements, of either sign, makes its row NaN and no other, whichever part of the row it is in; -0 and 0 are 0."""
    rng = np.random.default_rng(m)
    k, n = 544, 70
    c = few_codes(rng, m, k)
    c[(c == 0) & (rng.random((m, k)) < 0.3)] = 0x80
    r = m // 2
    c[r, [3, k - 1]] = [0x7F, 0xFF] if m % 2 else [0xFF, 0x7F]
    wc = codes(rng, (n, k), "mxfp4")
    wc[:, 3], wc[: n // 2, k - 1] = 0, 8  # NaN times 0
    a, av = device(c, "mxfp8", ones(m, k))
    w, wv = device(wc, "mxfp4", ones(n, k))
    out = torch.empty((m, n), device="cuda")
    ctx.mx_product(a, ctx.mx_weight([w]), out)
    got = out.double().cpu().numpy()
    others = np.arange(m) != r
    assert np.isnan(got[r]).all() and np.array_equal(got[others], mx.product(av[others], wv))
