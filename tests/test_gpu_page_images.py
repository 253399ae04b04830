"""Images of pages on both sides of the size from which they are read past the caches."""
import numpy as np
import pytest
import torch

from test_gpu_pages import model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hkv,P,layers,n", [(128, 8, 16, 32, 31), (128, 8, 16, 32, 32), (64, 8, 32, 32, 31), (64, 8, 32, 32, 33), (64, 1, 16, 1, 16385)])
def test_images_of_about_64_mib(D, Hkv, P, layers, n):
    from paper_2510_24051_amd import Pie
    ctx = Pie(model(D, Hkv, P), 2 * n + 1, 1, max_batch_tokens=1, max_batch_requests=1, n_layers=layers)
    gen = torch.Generator(device="cuda").manual_seed(n)
    bits = torch.randint(-32768, 32768, (n, layers, 2, P, Hkv, D), generator=gen, device="cuda", dtype=torch.int16)
    assert abs(bits.nbytes / (64 << 20) - 1) < 0.05  # (give or take a page)
    ids = np.random.default_rng(n).permutation(2 * n + 1).astype(np.int32)
    back = torch.zeros_like(bits)
    torch.cuda.synchronize()
    ctx.restore_kvpage(ids[:n], bits.view(torch.bfloat16))
    ctx.fork_kvpage(ids[:n], ids[n:2 * n])
    ctx.save_kvpage(ids[n:2 * n], back.view(torch.bfloat16))
    ctx.synchronize()
    assert torch.equal(back, bits)
    for layer, page, slot in ((0, 0, 0), (layers - 1, n - 1, P - 1), (layers // 2, n // 2, 3)):  # token by token, as another call sees it
        k, v = ctx.kv_read(layer, [ids[page]], [slot])
        want = bits[page, layer, :, slot].cpu().numpy().view(np.uint16)
        assert np.array_equal(k[0], want[0]) and np.array_equal(v[0], want[1])
    ctx.close()
