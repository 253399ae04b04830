"""A microscaled weight that Python collects while another stream, which the context has nothing to do with, is being captured."""
import gc

import numpy as np
import pytest
import torch

import workloads as W
from oracle import mx
from test_gpu_mx import device_rows

pytestmark = pytest.mark.gpu


def test_a_weight_dropped_during_a_capture():
    from paper_2510_24051_amd import Pie
    ctx = Pie(W.model_tiny(), 8, 8, max_batch_tokens=8, max_batch_requests=8)
    rng = np.random.default_rng(3)
    a, av = device_rows(rng.choice([0.0, 1, -1, 2], size=(5, 64)), "mxfp8")
    w, wv = device_rows(rng.choice([0.0, 1, -2, 3], size=(40, 64)), "mxfp4")
    kept, doomed, out = ctx.mx_weight([w]), [ctx.mx_weight([w]) for _ in range(3)], torch.empty((5, 40), device="cuda")
    x = torch.arange(64.0, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        x.add_(1.0)
        doomed.clear()
        gc.collect()
        x.mul_(2.0)
    want = torch.arange(64.0)
    for _ in range(3):
        graph.replay()
        want = (want + 1.0) * 2.0
        ctx.mx_product(a, kept, out)
        torch.cuda.synchronize()
        assert torch.equal(x.cpu(), want) and np.array_equal(out.double().cpu().numpy(), mx.product(av, wv))
    ctx.synchronize()  # (they are freed here)
    assert not ctx._dropped
    ctx.mx_product(a, ctx.mx_weight([w]), out)
    assert np.array_equal(out.double().cpu().numpy(), mx.product(av, wv))
