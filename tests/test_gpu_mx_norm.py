"""The norm's values, off by no more than their last rounding to 32 bits.

A value is fma(h, G, h g) with G + g the gain over the root: of the sum, in 64 bits throughout; of the root, one step of Newton's method in 64 bits from
a reciprocal root good to 2^-22, which leaves 1.5 2^-44; of G + g, a pair of fp32 that holds the quotient to 2^-47.  That is rounded once: REL = 2^-24 and 2^-20 of it.
(Where the root is no ordinary number of 32 bits the product is taken in 64 and rounded once.)  So an element of a value further than REL from the border
between two elements is the nearer one.

The rows are made so that values lie within a few units of 32 bits of such borders; sums kept to 32 bits anywhere, for eight columns or a whole
row, or a root or a gain rounded to 32 bits, put some on the wrong side."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx
from test_gpu_mx import check_computed, rows_of

pytestmark = pytest.mark.gpu

REL = 2.0 ** -24 * (1 + 2.0 ** -20)
EPS = 1e-5


@pytest.fixture(scope="module")
def ctx():
    from paper_2510_24051_amd import Pie
    c = Pie(W.model_tiny(), 8, 8, max_batch_tokens=8, max_batch_requests=8)
    assert c.model.rms_eps == EPS
    return c


def near_borders(rng, rows, k, form, gain):
    """fp32 rows: the first thread's eight columns are 2^10 times the others', the first of every block is the block's largest, and all
    others lie 1.2 to 4 units of 2^-24 from the middle between two elements."""
    codes = mx.codes_values(form)
    codes = codes[:len(codes) // 2]
    codes = codes[np.isfinite(codes)]
    low = codes[(codes >= mx.LARGEST[form] / 64) & (codes < mx.LARGEST[form] / 2)]
    high = np.array([codes[codes > c].min() for c in low])
    pick = rng.integers(0, len(low), size=(rows, k))
    z = (low[pick] + high[pick]) / 2 * (1 + rng.choice([-1, 1], size=(rows, k)) * rng.uniform(1.2, 4.0, size=(rows, k)) * 2.0 ** -24)
    z[:, ::32] = mx.LARGEST[form] * rng.uniform(0.7, 0.95, size=(rows, k // 32))
    z[:, :8] = mx.LARGEST[form] * rng.uniform(0.6, 0.95, size=(rows, 8))
    z[:, 32:] *= 2.0 ** -10
    z *= rng.choice([-1.0, 1.0], size=(rows, k))
    n = z / gain  # normalised values before the gain, up to a power of two
    mean = (n * n).mean(1, keepdims=True)
    s = np.exp2(np.floor(-np.log2(mean) / 2 - 0.05))  # the largest that leaves a mean square below 1
    n, mean = n * s, mean * s * s
    assert np.all(mean < 1) and np.all(mean > 0.1)
    return (n * np.sqrt(EPS / (1 - mean))).astype(np.float32)  # with rows of mean square eps mean / (1 - mean), eps has its share


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("rows,k", [(4000, 32), (2000, 64), (1000, 544), (400, 2048), (200, 4096), (60, 8192)])
def test_values_next_to_the_borders(ctx, form, rows, k):
    rng = np.random.default_rng(rows + k)
    gain = np.exp2(rng.integers(-2, 3, size=k)) * rng.choice([-1.0, 1.0], size=k) if k > 64 else np.ones(k)
    x = near_borders(rng, rows, k, form, gain)
    r = rows_of(form, rows, k)
    ctx.mx_norm(torch.from_numpy(x).cuda(), torch.from_numpy(gain).to(torch.bfloat16).cuda(), r)
    check_computed(r, mx.norm(x.astype(np.float64), gain, float(np.float32(EPS))), REL, f"norm {rows} x {k}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(3000, 32), (1000, 544), (1000, 4096), (60, 8192)])
def test_values_of_any_rows(ctx, dtype, rows, k):
    gen = torch.Generator(device="cuda").manual_seed(rows + k)
    x = torch.randn((rows, k), generator=gen, device="cuda")
    x[:, 8 * (k // 64):8 * (k // 64) + 8] *= 100.0  # one thread's columns
    x = x.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    gain = torch.randn(k, generator=gen, device="cuda").bfloat16()
    r = rows_of("mxfp8", rows, k)
    ctx.mx_norm(x, gain, r)
    check_computed(r, mx.norm(x.double().cpu().numpy(), gain.double().cpu().numpy(), float(np.float32(EPS))), REL, f"norm {rows} x {k}")


def test_values_whose_root_32_bits_do_not_hold():
    """Rows of 2^-70 (with an epsilon below their squares) to 2^124: no less exact."""
    from paper_2510_24051_amd import Pie
    m = W.model_tiny()
    own = Pie(SimpleNamespace(**{**{f: getattr(m, f) for f in ("hidden", "n_q_heads", "n_kv_heads", "head_dim", "mlp_dim", "vocab", "page_size", "rope_theta")},
                                 "rms_eps": 1e-44}), 8, 8, max_batch_tokens=8, max_batch_requests=8)
    eps = float(np.float32(1e-44))
    for k in (64, 544, 4096):
        gen = torch.Generator(device="cuda").manual_seed(k)
        powers = torch.tensor([-70, -60, -51, -49, -40, 0, 40, 48, 49, 50, 51, 62, 70, 100, 120, 124], device="cuda").repeat(1 + 100000 // k // 16)
        x = torch.randn((len(powers), k), generator=gen, device="cuda").clamp(-4, 4) * torch.exp2(powers.float())[:, None]
        gain = torch.randn(k, generator=gen, device="cuda").bfloat16()
        r = rows_of("mxfp8", len(powers), k)
        own.mx_norm(x, gain, r)
        check_computed(r, mx.norm(x.double().cpu().numpy(), gain.double().cpu().numpy(), eps), REL, f"norm of {k}")
