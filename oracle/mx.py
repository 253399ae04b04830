"""CPU oracle of the microscaled formats (OCP Microscaling Formats v1.0: blocks of 32 values, a scale 2^(b - 127), elements E4M3 or E2M1) and
of the operators on them, NumPy in 64 bits."""
from __future__ import annotations

import numpy as np

from .pie_oracle import bf16_decode, bf16_round, rmsnorm, silu

BLOCK = 32
EMAX = {"mxfp8": 8, "mxfp4": 2}
LARGEST = {"mxfp8": 448.0, "mxfp4": 6.0}
FRACTION_BITS = {"mxfp8": 3, "mxfp4": 1}
LEAST_EXPONENT = {"mxfp8": -6, "mxfp4": 0}


def codes_values(form: str) -> np.ndarray:
    """What every element code stands for."""
    if form == "mxfp4":
        pos = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
        return np.concatenate([pos, -pos])
    c = np.arange(128)
    e, f = c >> 3, (c & 7) / 8.0
    pos = np.where(e > 0, (1.0 + f) * 2.0 ** (e - 7.0), f * 2.0 ** -6)
    pos[127] = np.nan
    return np.concatenate([pos, -pos])


def round_element(v: np.ndarray, form: str) -> np.ndarray:
    """To the nearest element, ties to even, saturating."""
    v = np.asarray(v, dtype=np.float64)
    e = np.maximum(np.frexp(v)[1] - 1, LEAST_EXPONENT[form]) - FRACTION_BITS[form]
    return np.clip(np.ldexp(np.rint(np.ldexp(v, -e)), e), -LARGEST[form], LARGEST[form])


def element_step(v: np.ndarray, form: str) -> np.ndarray:
    """Spacing of the elements at v."""
    e = np.maximum(np.frexp(np.asarray(v, dtype=np.float64))[1] - 1, LEAST_EXPONENT[form]) - FRACTION_BITS[form]
    return np.ldexp(1.0, e)


def scale_bytes(x: np.ndarray, form: str) -> np.ndarray:
    """[rows, k / 32] of values [rows, k]."""
    with np.errstate(invalid="ignore"):
        top = np.abs(np.asarray(x, dtype=np.float64).reshape(x.shape[0], -1, BLOCK)).max(-1)
    e = np.frexp(np.where(np.isfinite(top), top, 1.0))[1] - 1 - EMAX[form] + 127
    e = np.where(top == 0, 0, np.clip(e, 0, 254))
    return np.where(np.isfinite(top), e, 255).astype(np.uint8)


def quantise(x: np.ndarray, form: str):
    """(elements as values [rows, k], scale bytes) of values [rows, k]; a block with a NaN or an infinity: scale 255, elements 0."""
    x = np.asarray(x, dtype=np.float64)
    b = scale_bytes(x, form)
    nan = np.repeat(b == 255, BLOCK, axis=1)
    s = np.repeat(b.astype(np.int64) - 127, BLOCK, axis=1)
    return np.where(nan, 0.0, round_element(np.ldexp(np.where(nan, 0.0, x), -s), form)), b


def scales_of(b: np.ndarray) -> np.ndarray:
    return np.where(b == 255, np.nan, np.ldexp(1.0, b.astype(np.int64) - 127))


def values(elements: np.ndarray, b: np.ndarray) -> np.ndarray:
    return elements * np.repeat(scales_of(b), BLOCK, axis=1)


def decode(codes: np.ndarray, form: str) -> np.ndarray:
    """Elements as values of stored bytes [rows, k] or [rows, k / 2]."""
    if form == "mxfp4":
        codes = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[0], -1)
    return codes_values(form)[codes]


def encode(elements: np.ndarray, form: str) -> np.ndarray:
    """Stored bytes of elements given as (exactly representable) values."""
    table = codes_values(form)
    n = len(table) // 2
    order = np.nan_to_num(table[:n], nan=1e9)
    c = np.searchsorted(order, np.abs(elements))
    assert np.array_equal(order[c], np.abs(elements))
    c = (c + n * np.signbit(elements)).astype(np.uint8)
    return c if form == "mxfp8" else (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)


def product(a: np.ndarray, w: np.ndarray) -> np.ndarray:
    """a [rows, k] times w [n, k] transposed, as values."""
    return a @ w.T


def swiglu(a: np.ndarray, gate: np.ndarray, up: np.ndarray) -> np.ndarray:
    """Before quantisation."""
    return silu(a @ gate.T) * (a @ up.T)


def norm(x: np.ndarray, gain: np.ndarray, eps: float) -> np.ndarray:
    """Before quantisation."""
    return rmsnorm(x, gain, eps)


def requantised(x: np.ndarray, form: str = "mxfp8") -> np.ndarray:
    """The values that x has after quantisation."""
    return values(*quantise(x, form))


def layer_tail(x: np.ndarray, attn: np.ndarray, g2: np.ndarray, wo, wgate, wup, wdown, eps: float):
    """What a layer does behind attention, from its input x, attention output, gain and weights as values: (residual, activations, output)."""
    h = x + requantised(attn) @ wo.T
    act = requantised(swiglu(requantised(norm(h, g2, eps)), wgate, wup))
    return h, act, h + act @ wdown.T


__all__ = ["bf16_decode", "bf16_round", "codes_values", "decode", "element_step", "encode", "layer_tail", "norm", "product", "quantise", "requantised",
           "round_element", "scale_bytes", "scales_of", "swiglu", "values"]
