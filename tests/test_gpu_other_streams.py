"""Images and logits on torch's current stream while the context has a stream of its own: no wait by the program in between."""
import numpy as np
import pytest
import torch

import workloads as W
from test_gpu_beams import logits, select
from test_gpu_pages import model

pytestmark = pytest.mark.gpu


def busy():
    """Some milliseconds of the current stream."""
    torch.cuda._sleep(10_000_000)


@pytest.mark.parametrize("current", ["default", "another", "the context's"])
def test_images(current):
    from paper_2510_24051_amd import Pie
    ctx = Pie(model(128, 2, 16), 12, 1, max_batch_tokens=1, max_batch_requests=1, n_layers=3)
    stream = {"default": torch.cuda.default_stream(), "another": torch.cuda.Stream(), "the context's": ctx.stream}[current]
    shape = (5, 3, 2, 16, 2, 128)
    gen = torch.Generator(device="cuda").manual_seed(1)
    given = [torch.randint(-32768, 32768, shape, generator=gen, device="cuda", dtype=torch.int16) for _ in range(4)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        image, seen = torch.zeros(shape, dtype=torch.int16, device="cuda"), []
        for k, bits in enumerate(given):
            busy()
            image.copy_(bits)  # late
            ctx.restore_kvpage(np.arange(5) + k, image.view(torch.bfloat16))
            image.zero_()  # at once
            out = torch.full(shape, 3, dtype=torch.int16, device="cuda")
            ctx.save_kvpage(np.arange(5) + k, out.view(torch.bfloat16))
            seen.append(out.cpu())
            del out
    for k, bits in enumerate(given):
        assert torch.equal(seen[k], bits.cpu()), k
    ctx.close()


@pytest.mark.parametrize("current", ["default", "another"])
def test_logits_and_scores(current):
    from paper_2510_24051_amd import Pie
    m = W.ModelDesc(hidden=128, n_q_heads=2, n_kv_heads=2, head_dim=64, mlp_dim=256, vocab=32000, page_size=16, rms_eps=1e-5, rope_theta=1e4, n_layers=1)
    ctx = Pie(m, 4, 4, max_batch_tokens=4, max_batch_requests=4, max_dist_rows=16)
    stream = {"default": torch.cuda.default_stream(), "another": torch.cuda.Stream()}[current]
    rows = [logits(8, 32000, torch.float32, 60 + k) for k in range(3)]
    starts = [np.random.default_rng(k).standard_normal(8).astype(np.float32) for k in range(3)]
    want = [select(ctx, z, [0, 3, 8], 7, s) for z, s in zip(rows, starts)]
    starts_dev = [torch.from_numpy(s).cuda() for s in starts]
    torch.cuda.synchronize()
    got = []
    with torch.cuda.stream(stream):
        for z, s in zip(rows, starts_dev):
            busy()
            late, late_s = z.clone(), s.clone()
            outs = [torch.empty((2, 7), dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.float32)]
            ctx.beam_select_async(late, [0, 3, 8], 7, *outs, scores=late_s)
            late.fill_(9.0)
            late_s.fill_(-5.0)
            got.append([o.cpu().numpy() for o in outs])
    for g, w in zip(got, want):
        assert all(np.array_equal(x, y) for x, y in zip(g, w))
    ctx.close()


def test_a_capture_on_another_stream_takes_the_calls_in():
    from paper_2510_24051_amd import Pie
    ctx = Pie(model(64, 2, 16), 12, 1, max_batch_tokens=1, max_batch_requests=1, n_layers=2)
    shape = (3, 2, 2, 16, 2, 64)
    given, image, out = (torch.zeros(shape, dtype=torch.int16, device="cuda") for _ in range(3))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        image.copy_(given)
        ctx.restore_kvpage([4, 2, 7], image.view(torch.bfloat16))
        image.zero_()
        ctx.save_kvpage([7, 4, 2], out.view(torch.bfloat16))
    for replay in range(4):
        given.copy_(torch.full(shape, replay + 1, dtype=torch.int16, device="cuda") + torch.arange(3, device="cuda", dtype=torch.int16).view(3, 1, 1, 1, 1, 1) * 100)
        g.replay()
        want = given[[2, 0, 1]].cpu()
        assert torch.equal(out.cpu(), want), replay
        eager = torch.empty_like(out)
        ctx.save_kvpage([7, 4, 2], eager.view(torch.bfloat16))  # eager work between the replays
        assert torch.equal(eager.cpu(), want), replay
        out.zero_()
    ctx.close()
