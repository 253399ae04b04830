"""How products of microscaled rows are taken, on the CPU: what a weight keeps of its earlier products changes nothing (through the C ABI on the stand-in
for the HIP runtime), and which forms and splits the sizes of the GPU tests go through."""
import os
import subprocess
import sys

import numpy as np
import pytest

from test_host_mx import FORM_SIZES, FORMS, FP4, FP8, Calls
from test_host_runtime_paths import Child, fake  # noqa: F401  (the fixture builds the stand-in)

K, N = 2048, 4096


def kept_plans(c):
    """A weight's products of any numbers of rows in any order launch what a new weight's do, also when there are more of them than it keeps, cut into tiles
    and a rest or not."""
    m = Calls(c, c.context())
    c.fake.fake_watch(b"mx_", 1)  # (the second argument of the products' kernels is their number of rows)

    def weight():
        st, h = m.weight(N, k=K, row_bytes=K // 2)
        assert st == 0
        c.launches()
        return h

    def launched(h, rows, form):
        row = m.mx(FP8, row_bytes=K, scale_bytes=64) if form == FP8 else m.mx(FP4, row_bytes=K // 2, scale_bytes=64)
        assert m.call("pie_mx_product", row, rows, h, m.rows(stride=N)) == 0
        return c.launches()

    calls = [(rows, form) for rows in (1, 64, 8320, 333, 900, 17, 40, 129, 2000, 3, 8192, 130) for form in (FP8, FP4)]
    want = {}
    for call in calls:
        h = weight()
        want[call] = launched(h, *call)
        assert m.call("pie_mx_weight_destroy", h) == 0
    assert len({tuple(v) for v in want.values()}) > 12 and any(len(v) > 1 for v in want.values())
    one, rng = weight(), np.random.default_rng(0)
    for i in rng.integers(0, len(calls), size=400):
        assert launched(one, *calls[i]) == want[calls[i]], calls[i]
    for _ in range(3):  # as many as it keeps, in turn
        for call in calls[:6]:
            assert launched(one, *call) == want[call]


CASES = {f.__name__: f for f in (kept_plans,)}

if __name__ == "__main__":
    CASES[sys.argv[2]](Child(sys.argv[1]))
    print("case passed")
    sys.exit(0)


@pytest.mark.parametrize("case", list(CASES))
def test_host_path(fake, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, case], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "case passed" in r.stdout, f"exit {r.returncode}\n{r.stdout}\n{r.stderr}"


def plans(sizes, gated, form):
    from paper_2510_24051_amd import mx_product_plan
    return [(m, mx_product_plan(m, n, k, gated, form)) for m, k, n in sizes]


def listed(gated, form):
    """Every product whose sums the GPU tests compare bit for bit (or, gated, to the activation's roundings)."""
    import test_gpu_mx_sums as G
    own = G.GATED_SIZES if gated else G.SIZES if form == "mxfp8" else G.SIZES4
    return [(m, k, n) for g, f, m, k, n in FORM_SIZES if (g, f) == (gated, form)] + (own if form == "mxfp8" or not gated else [])


@pytest.mark.parametrize("form", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("gated", [False, True])
def test_splits_and_cuts_are_listed(gated, form):
    """Of either kind, for either format: products split over workgroups, whose sums are joined, and products cut behind whole tiles."""
    p = plans(listed(gated, form), gated, form)
    assert any(x["splits"] > 1 for _, x in p) and any(x["rows"] < m for m, x in p)
    assert {(x["tile_rows"], x["tile_columns"], x["k_slices"]) for _, x in p} == FORMS[gated]


def test_forms_of_up_to_16_rows_are_listed():
    """8-bit rows whose two parts stand side by side: every form of one block of rows, split and whole."""
    for gated in (False, True):
        seen = {(x["tile_columns"], x["k_slices"], x["splits"] > 1) for m, x in plans([s for s in listed(gated, "mxfp8") if s[0] <= 16], gated, "mxfp8") if x["tile_rows"] == 32}
        assert seen == {(c, s, split) for r, c, s in FORMS[gated] if r == 32 for split in (False, True)}


def test_sums_of_split_products_fit_the_workspace():
    """2^24 floats: as many copies of the sums as there are splits, their rows filled up to blocks of 32 columns."""
    from paper_2510_24051_amd import mx_product_plan
    rng = np.random.default_rng(1)
    most = 0
    for _ in range(4000):
        m, n, k = (int(2 ** rng.uniform(0, b)) for b in (14, 15, 10))
        gated = bool(rng.integers(2))
        n = (n + 31) // 32 * 32 if gated else n
        p = mx_product_plan(m, n, 32 * k, gated, ["mxfp8", "mxfp4"][rng.integers(2)])
        if p["splits"] > 1:
            floats = p["splits"] * p["rows"] * ((n + 31) // 32 * 32) * (2 if gated else 1)
            assert floats <= 1 << 24
            most = max(most, floats)
    assert most > 1 << 21  # (some come near)
