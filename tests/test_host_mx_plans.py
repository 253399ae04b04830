"""How products of microscaled rows are taken, on the CPU: what a weight keeps of its earlier products changes nothing (through the C ABI on the stand-in
for the HIP runtime), and which forms and splits the sizes of the GPU tests go through."""
import os
import subprocess
import sys

import numpy as np
import pytest

from test_host_mx import FORM_SIZES, FP4, FP8, Calls
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
