"""Pins of the microscaled oracle: the formats' tables, ties, saturation and scales as the published standard gives them."""
import numpy as np
import pytest
import torch

from oracle import mx


def test_tables():
    v = mx.codes_values("mxfp8")
    assert v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1.0 and v[0x7E] == 448.0 and v[0xFE] == -448.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and np.isnan(v).sum() == 2
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, v, equal_nan=True)
    assert mx.codes_values("mxfp4").tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6]


def test_rounding():
    # halves go to the even code, what is above the largest saturates
    assert mx.round_element([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 7.9, -0.25, -5.0], "mxfp4").tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -4]
    assert mx.round_element([17.0, 19.0, 464.0, 511.0, 2.0 ** -10, 3 * 2.0 ** -10], "mxfp8").tolist() == [16, 20, 448, 448, 0, 2.0 ** -8]
    x = np.random.default_rng(1).normal(size=20000) * 100
    t = torch.tensor(x, dtype=torch.float32)
    assert np.array_equal(mx.round_element(t.double().numpy(), "mxfp8"), t.to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("form,top,byte", [("mxfp8", 256.0, 127), ("mxfp8", 255.9, 126), ("mxfp8", 1.0, 119), ("mxfp8", 0.0, 0), ("mxfp4", 4.0, 127),
                                           ("mxfp4", 3.99, 126), ("mxfp4", 2.0 ** -125, 0), ("mxfp4", 2.0 ** -149, 0), ("mxfp8", 2.0 ** 127, 246),
                                           ("mxfp8", np.inf, 255), ("mxfp4", np.nan, 255)])
def test_scales(form, top, byte):
    x = np.zeros((1, 32))
    x[0, 7] = -top
    assert mx.scale_bytes(x, form).tolist() == [[byte]]
    e, b = mx.quantise(x, form)
    assert not e.any() if byte == 255 else np.array_equal(np.flatnonzero(e), [] if mx.round_element(np.ldexp(top, 127 - byte), form) == 0 else [7])


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
def test_round_trip(form):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 160)) * np.exp(rng.normal(size=(5, 1)) * 6)
    e, b = mx.quantise(x, form)
    assert np.array_equal(mx.decode(mx.encode(e, form), form), e)
    v = mx.values(e, b)
    # the largest of a block is at most 2^(EMAX + 1) scales: it loses a quarter (E2M1) or an eighth (E4M3) where it saturates
    step = mx.element_step(np.ldexp(x, 127 - np.repeat(b.astype(int), 32, 1)), form) * np.repeat(mx.scales_of(b), 32, 1)
    sat = np.repeat(mx.scales_of(b), 32, 1) * mx.LARGEST[form]
    assert np.all(np.abs(v - np.clip(x, -sat, sat)) <= step / 2)
    assert np.array_equal(mx.requantised(v, form), v)  # what is in the format stays
