"""Device memory that compactions take, without a GPU (against the stand-in for the HIP runtime, in a process of its own)."""
import os
import subprocess
import sys

import numpy as np

from test_host_runtime_paths import Child, fake  # noqa: F401  (the fixture builds the stand-in)


def scratch_is_as_large_as_it_has_to_be(c):
    """Half of one long sequence, in place: its chains go through scratch blocks.  The block that the context keeps for them holds those
    blocks, an eighth of them for a longer sequence to come, and the plan; it is taken once."""
    ctx = c.context(n_pages=600)
    keep = np.random.default_rng(0).random(8000) < 0.5
    bits = (keep.reshape(500, 16).astype(np.uint32) << np.arange(16, dtype=np.uint32)).sum(1)
    ctx.mask_kvpage(np.arange(500), bits)
    c.fake.fake_largest_malloc()
    kept = ctx.compact_kvpage([0, 500], np.arange(500), [8000])[0]
    assert kept == keep.sum()
    scratch = -(-int(kept) // 16) * 2 * 2 * 16 * 64 * 2  # blocks of 2 heads, K and V, 16 tokens, 64 dims, 2 bytes
    first = c.fake.fake_largest_malloc()
    assert scratch <= first <= scratch * 9 // 8 + (1 << 19), (scratch, first)
    for _ in range(3):
        ctx.mask_kvpage(np.arange(500), bits)
        ctx.compact_kvpage([0, 500], np.arange(500), [8000])
    assert c.fake.fake_largest_malloc() == 0
    ctx.close()


CASES = {f.__name__: f for f in (scratch_is_as_large_as_it_has_to_be,)}

if __name__ == "__main__":
    CASES[sys.argv[2]](Child(sys.argv[1]))
    print("case passed")
    sys.exit(0)


def test_scratch_is_as_large_as_it_has_to_be(fake):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, "scratch_is_as_large_as_it_has_to_be"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "case passed" in r.stdout, f"exit {r.returncode}\n{r.stdout}\n{r.stderr}"
