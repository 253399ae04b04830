"""The calls on microscaled rows without a GPU, through the C ABI on a stand-in for the HIP runtime (fake_hip.cpp): every refusal, that a
refused call launches nothing and leaves nothing allocated, and what a layer of microscaled weights launches."""
import ctypes as C
import os
import subprocess
import sys

import numpy as np
import pytest

from test_host_runtime_paths import MODEL, Child, batch_of, fake  # noqa: F401  (the fixture builds the stand-in)

INVALID, RANGE, UNSUPPORTED, MEMORY, HIP = -1, -2, -7, -5, -6
FP8, FP4 = 0, 1
F32, BF16, F16 = 0, 1, 2
ROOM = np.zeros(1 << 20, np.uint8)
A = (ROOM.ctypes.data + 255) // 256 * 256  # (copies and fills of the stand-in may touch it; kernels do nothing)

# (gated, format, rows, k, n): products that between them go through every form (test_gpu_mx.py computes them)
FORM_SIZES = [
    (False, "mxfp4", 1, 2048, 20000), (False, "mxfp4", 1, 1056, 32), (False, "mxfp4", 2050, 8192, 32), (False, "mxfp4", 1, 544, 32), (False, "mxfp4", 1030, 8192, 32),
    (False, "mxfp4", 1, 32, 32), (False, "mxfp4", 17, 8192, 32), (False, "mxfp4", 33, 1056, 8192), (False, "mxfp4", 2050, 544, 200),
    (False, "mxfp4", 33, 8192, 4096), (False, "mxfp4", 200, 544, 8192), (False, "mxfp4", 1030, 544, 1000), (False, "mxfp4", 257, 8192, 1000),
    (False, "mxfp4", 1030, 512, 1000), (False, "mxfp4", 515, 8192, 1000), (False, "mxfp4", 400, 512, 8192), (False, "mxfp4", 400, 544, 8192),
    (False, "mxfp4", 900, 512, 8192), (False, "mxfp4", 1030, 32, 1000), (False, "mxfp8", 1, 544, 32), (False, "mxfp8", 1030, 8192, 32),
    (False, "mxfp8", 1, 512, 32), (False, "mxfp8", 1, 8192, 32), (False, "mxfp8", 1, 32, 32), (False, "mxfp8", 31, 4096, 32),
    (False, "mxfp8", 130, 8192, 1000), (False, "mxfp8", 33, 544, 8192), (False, "mxfp8", 515, 4096, 1000), (False, "mxfp8", 65, 8192, 1000),
    (False, "mxfp8", 200, 512, 8192), (False, "mxfp8", 257, 8192, 1000), (False, "mxfp8", 1030, 512, 1000), (False, "mxfp8", 700, 8192, 200),
    (False, "mxfp8", 1030, 256, 1000), (False, "mxfp8", 130, 8192, 2048), (False, "mxfp8", 400, 256, 8192), (False, "mxfp8", 400, 512, 8192),
    (False, "mxfp8", 900, 512, 8192), (False, "mxfp8", 1030, 32, 1000), (False, "mxfp8", 2050, 256, 8192), (True, "mxfp4", 1, 544, 32),
    (True, "mxfp4", 1, 4096, 2048), (True, "mxfp4", 1, 32, 32), (True, "mxfp4", 1, 4096, 32), (True, "mxfp4", 2050, 544, 224),
    (True, "mxfp4", 2050, 8192, 32), (True, "mxfp4", 2050, 512, 512), (True, "mxfp4", 2050, 544, 512), (True, "mxfp4", 1030, 8192, 224),
    (True, "mxfp4", 257, 544, 8192), (True, "mxfp4", 200, 544, 8192), (True, "mxfp4", 97, 8192, 4096), (True, "mxfp4", 400, 512, 8192),
    (True, "mxfp4", 130, 32, 32), (True, "mxfp4", 2050, 512, 4096), (True, "mxfp8", 1, 512, 32), (True, "mxfp8", 1, 8192, 32),
    (True, "mxfp8", 1, 32, 32), (True, "mxfp8", 1, 4096, 32), (True, "mxfp8", 2050, 512, 224), (True, "mxfp8", 2050, 4096, 32),
    (True, "mxfp8", 2050, 256, 512), (True, "mxfp8", 200, 8192, 2048), (True, "mxfp8", 2050, 512, 512), (True, "mxfp8", 2050, 8192, 32),
    (True, "mxfp8", 2050, 256, 1024), (True, "mxfp8", 2050, 8192, 224), (True, "mxfp8", 97, 8192, 4096), (True, "mxfp8", 400, 512, 8192),
    (True, "mxfp8", 130, 32, 32), (True, "mxfp8", 2050, 256, 4096)]
FORMS = {False: {(32, 128, 2), (32, 64, 4), (32, 32, 8), (64, 64, 4), (64, 32, 8), (96, 128, 2), (96, 64, 4), (32, 128, 4), (64, 128, 4), (96, 256, 2), (128, 256, 2),
                 (128, 128, 4), (256, 256, 1)},
         True: {(32, 256, 2), (32, 128, 4), (64, 256, 2), (64, 128, 4), (96, 256, 2), (96, 128, 4), (128, 256, 2), (128, 128, 4), (256, 256, 1)}}


class Calls:
    def __init__(self, c, ctx):
        self.c, self.ctx, self.b = c, ctx, c.binding
        self.a = A

    def mx(self, format=FP8, elements=A, row_bytes=64, scales=A, scale_bytes=4):
        return C.byref(self.b.MxRowsC(format, elements, row_bytes, scales, scale_bytes))

    def rows(self, data=A, dtype=F32, stride=64):
        return self.b._ROWS.pack(data or 0, dtype, stride)

    def call(self, name, *args):
        return getattr(self.c.lib, name)(self.ctx.ctx, *args)

    def weight(self, *rows, k=64, gated=0, format=FP4, ctx=None, row_bytes=64):
        h, n = C.c_void_p(), np.array(rows, np.int32)
        parts = (self.b.MxRowsC * len(rows))(*[self.b.MxRowsC(format, A, row_bytes, A, 64) for _ in rows])
        return self.call("pie_mx_weight_create", parts, n.ctypes.data_as(C.c_void_p), len(rows), k, gated, C.byref(h)), h


def rows_refused(c):
    m = Calls(c, c.context())
    q = lambda x=0, rows=3, k=64, out=0: m.call("pie_mx_quantise", m.rows() if x == 0 else x, rows, k, m.mx() if out == 0 else out)  # noqa: E731
    d = lambda a=0, rows=3, k=64, out=0: m.call("pie_mx_dequantise", m.mx() if a == 0 else a, rows, k, m.rows() if out == 0 else out)  # noqa: E731
    c.launches()
    for f in (q, d):
        assert f(rows=-1) == INVALID and f(k=0) == INVALID and f(k=-32) == INVALID and f(k=33) == INVALID and f(k=16) == INVALID
        assert f(k=(1 << 20) + 32) == UNSUPPORTED and f(rows=(1 << 24) + 1) == UNSUPPORTED
        assert f(None, rows=0) == 0 and f(out=None, rows=0) == 0  # nothing is done, nothing looked at
        assert f(None) == INVALID and f(out=None) == INVALID
        mx, plain = (lambda v: f(out=v)) if f is q else f, f if f is q else (lambda v: f(out=v))  # noqa: E731
        for v in (m.mx(format=2), m.mx(format=-1), m.mx(elements=None), m.mx(scales=None), m.mx(elements=A + 8), m.mx(scales=A + 2), m.mx(row_bytes=48),
                  m.mx(row_bytes=72), m.mx(scale_bytes=2), m.mx(row_bytes=-(1 << 23)), m.mx(scale_bytes=-4), m.mx(scale_bytes=6), m.mx(scale_bytes=0), m.mx(FP4, row_bytes=16), m.mx(row_bytes=-64)):
            assert mx(v) == INVALID
        for v in (m.rows(data=None), m.rows(dtype=3), m.rows(dtype=-1), m.rows(stride=63), m.rows(stride=-64), m.rows(data=A + 2), m.rows(data=A + 1, dtype=BF16)):
            assert plain(v) == INVALID
        assert mx(m.mx(row_bytes=(1 << 22) + 16)) == UNSUPPORTED and mx(m.mx(scale_bytes=(1 << 22) + 4)) == UNSUPPORTED
        assert c.launches() == []
        for v in (m.mx(), m.mx(FP4, row_bytes=32), m.mx(row_bytes=80, scale_bytes=8)):
            assert mx(v) == 0
        for v in (m.rows(data=A + 4), m.rows(stride=65), m.rows(data=A + 2, dtype=BF16), m.rows(data=A + 6, dtype=F16, stride=67)):
            assert plain(v) == 0
        assert len(c.launches()) == 7
        assert f(k=96) == INVALID  # rows too short for it
    p = c.Pie.planner(MODEL, 32, 16, 8, 4)
    assert Calls(c, p).call("pie_mx_quantise", m.rows(), 1, 64, m.mx()) == INVALID
    assert c.lib.pie_mx_quantise(None, m.rows(), 1, 64, m.mx()) == INVALID and c.lib.pie_mx_dequantise(None, m.mx(), 1, 64, m.rows()) == INVALID


def norm_refused(c):
    m = Calls(c, c.context())
    n = lambda x=0, delta=None, gain=A, rows=3, k=64, h=None, out=0: m.call("pie_mx_norm", m.rows() if x == 0 else x, delta, gain, rows, k, h,  # noqa: E731
                                                                           m.mx() if out == 0 else out)
    c.launches()
    assert n(rows=-1) == INVALID and n(k=40) == INVALID and n(k=8224) == UNSUPPORTED and n(None) == INVALID and n(out=None) == INVALID and n(gain=None) == INVALID
    assert n(gain=A + 1) == INVALID and n(x=m.rows(stride=32)) == INVALID and n(delta=m.rows(data=None)) == INVALID and n(delta=m.rows(dtype=7)) == INVALID
    assert n(h=m.rows(dtype=BF16)) == INVALID and n(h=m.rows(stride=1)) == INVALID and n(x=m.rows(dtype=BF16), h=m.rows()) == INVALID
    assert n(out=m.mx(elements=A + 4)) == INVALID
    assert n(None, rows=0) == 0 and c.launches() == []
    assert n() == 0 and n(gain=A + 2) == 0 and n(delta=m.rows(dtype=F16)) == 0 and n(h=m.rows()) == 0 and n(x=m.rows(dtype=BF16), h=m.rows(dtype=BF16)) == 0
    wide = m.mx(row_bytes=8192, scale_bytes=256)
    assert n(x=m.rows(stride=8192), k=8192, out=wide) == 0 and len(c.launches()) == 6
    assert Calls(c, c.Pie.planner(MODEL, 32, 16, 8, 4)).call("pie_mx_norm", m.rows(), None, A, 1, 64, None, m.mx()) == INVALID


def weights_refused(c):
    m, other = Calls(c, c.context()), Calls(c, c.context())
    before = c.fake.fake_allocations()
    c.launches()
    assert m.weight()[0] == INVALID and m.weight(0)[0] == INVALID and m.weight(4, -1)[0] == INVALID and m.weight(4, k=48)[0] == INVALID
    assert m.weight(4, format=FP8)[0] == INVALID and m.weight(4, k=160)[0] == INVALID and m.weight((1 << 24), 1)[0] == UNSUPPORTED
    assert m.weight(32, gated=1)[0] == INVALID and m.weight(32, 64, gated=1)[0] == INVALID and m.weight(33, 33, gated=1)[0] == INVALID
    assert m.weight(32, 32, 32, gated=1)[0] == INVALID
    n, one, h = np.array([4], np.int32), (m.b.MxRowsC * 1)(m.b.MxRowsC(FP4, A, 64, A, 64)), C.c_void_p()
    at = n.ctypes.data_as(C.c_void_p)
    assert m.call("pie_mx_weight_create", None, at, 1, 64, 0, C.byref(h)) == INVALID and m.call("pie_mx_weight_create", one, None, 1, 64, 0, C.byref(h)) == INVALID
    assert m.call("pie_mx_weight_create", one, at, 1, 64, 0, None) == INVALID
    c.fake.fake_capturing(1)
    assert m.weight(4)[0] == HIP
    c.fake.fake_capturing(0)
    assert c.fake.fake_allocations() == before and c.launches() == []
    for limit in (1 << 25, 1 << 10):  # no room for the workspace, then (once it is there) for the weight
        c.fake.fake_malloc_limit(limit)
        st, h = m.weight(4096, k=64)
        assert st == MEMORY and not h.value
        c.fake.fake_malloc_limit(1 << 40)
        st, h = m.weight(4)
        assert st == 0 and h.value and m.call("pie_mx_weight_destroy", h) == 0
    st, plain = m.weight(5, 60, 3)
    st2, gated = m.weight(64, 64, gated=1)
    assert st == st2 == 0
    prod = lambda a=0, rows=3, w=plain, out=0, me=m: me.call("pie_mx_product", m.mx() if a == 0 else a, rows, w, m.rows(stride=68) if out == 0 else out)  # noqa: E731
    gate = lambda a=0, rows=3, w=gated, out=0, me=m: me.call("pie_mx_swiglu", m.mx() if a == 0 else a, rows, w, m.mx() if out == 0 else out)  # noqa: E731
    c.launches()
    for f, wrong in ((prod, gated), (gate, plain)):
        assert f(None) == INVALID and f(out=None) == INVALID and f(rows=-1) == INVALID and f(w=None) == INVALID and f(w=wrong) == INVALID
        assert f(rows=(1 << 24) + 1) == UNSUPPORTED and f(me=other) == INVALID and f(a=m.mx(format=3)) == INVALID and f(a=m.mx(row_bytes=32)) == INVALID
        assert f(None, rows=0) == 0
    assert prod(out=m.rows(stride=67)) == INVALID and prod(out=m.rows(stride=68, dtype=F16)) == INVALID and prod(out=m.rows(data=A + 2, stride=68)) == INVALID
    assert gate(out=m.mx(row_bytes=48)) == INVALID and gate(out=m.mx(scale_bytes=0)) == INVALID
    assert c.launches() == []
    assert prod() == 0 and prod(out=m.rows(dtype=BF16, stride=69)) == 0 and gate() == 0 and gate(a=m.mx(FP4, row_bytes=32), out=m.mx(FP4, row_bytes=32)) == 0
    assert len(c.launches()) >= 4
    assert other.call("pie_mx_weight_destroy", plain) == INVALID and m.call("pie_mx_weight_destroy", plain) == 0 and m.call("pie_mx_weight_destroy", None) == 0
    assert m.call("pie_mx_weight_destroy", plain) == INVALID  # no longer a weight of this context
    m.ctx.close()  # (gated goes with it)
    p = Calls(c, c.Pie.planner(MODEL, 32, 16, 8, 4))
    assert p.weight(4)[0] == INVALID


def no_memory(c):
    """C++ allocations that fail: an error, and the context goes on."""
    m = Calls(c, c.context())
    for k in range(1, 4):
        c.fake.fake_fail_new_at(k)
        st, h = m.weight(4)
        c.fake.fake_fail_new_at(0)
        assert st in (0, MEMORY) and (st == 0) == bool(h.value)
    assert m.weight(4)[0] == 0
    m.ctx.close()


def load(c, ctx, layer, **kw):
    m = c.binding
    H, Q, KD, I = MODEL.hidden, MODEL.n_q_heads * MODEL.head_dim, MODEL.n_kv_heads * MODEL.head_dim, MODEL.mlp_dim
    ks = [H, H, H, Q, H, H, I]
    w = [m.MxRowsC(FP4, A, k // 2, A, k // 32) for k in ks]
    for i, v in kw.get("change", {}).items():
        w[i] = v
    return c.lib.pie_load_layer_mx(ctx.ctx, layer, kw.get("g1", A), kw.get("g2", A), (m.MxRowsC * 7)(*w))


def layers(c):
    M = c.binding.MxRowsC
    ctx = c.context(layers=2)
    assert load(c, ctx, 0, g1=None) == INVALID and load(c, ctx, 0, g2=None) == INVALID and load(c, ctx, -1) == RANGE and load(c, ctx, 2) == RANGE
    assert c.lib.pie_load_layer_mx(ctx.ctx, 0, A, A, None) == INVALID
    for i, v in ((0, M(FP8, A, 512, A, 16)), (3, M(FP4, A, 64, A, 4)), (6, M(FP4, A + 8, 128, A, 8)), (5, M(FP4, A, 64, A, 2))):
        assert load(c, ctx, 0, change={i: v}) == INVALID
    c.fake.fake_capturing(1)
    assert load(c, ctx, 0) == HIP
    c.fake.fake_capturing(0)
    b = batch_of([(20, 5), (1, 40)])
    pb = ctx.batch_create(b)
    assert c.status(lambda: ctx.forward(0, pb))[0] == INVALID  # no weights
    assert load(c, ctx, 0) == 0 and load(c, ctx, 1) == 0 and load(c, ctx, 0) == 0
    c.launches()
    ctx.forward(0, pb)
    names = c.launches()
    assert sum("mx_norm" in n for n in names) == 2 and sum("mx_quantise" in n for n in names) == 1 and not any("gemm" in n or "few" in n for n in names), names
    ctx.forward_all(pb)
    room = C.c_void_p(ROOM.ctypes.data)
    assert c.lib.pie_load_layer(ctx.ctx, 0, *[room] * 9) == 0  # back to bf16; the other stays
    c.launches()
    ctx.forward_all(pb)
    names = c.launches()
    assert any("gemm" in n or "few" in n for n in names) and sum("mx_norm" in n for n in names) == 2
    pb.destroy()
    ctx.close()
    assert load(c, c.Pie.planner(MODEL, 32, 16, 8, 4), 0) == INVALID
    for limit in (1 << 12, 1 << 24):  # no room for the activations, or the workspace
        ctx = c.context()
        c.fake.fake_malloc_limit(limit)
        assert load(c, ctx, 0) == MEMORY
        c.fake.fake_malloc_limit(1 << 40)
        assert load(c, ctx, 0) == 0
        ctx.close()


def adapters(c):
    """A batch whose adapter has a pair in a microscaled layer is refused before anything is launched; adapters elsewhere are not."""
    ctx = c.loaded(pairs=[(0, 0, 4)], layers=2, adapters=2, rank=4)
    assert load(c, ctx, 1) == 0
    b = batch_of([(1, 5), (1, 7)])
    b.adapter_ids = np.array([0, -1])
    pb = ctx.batch_create(b)
    c.launches()
    st, msg = c.status(lambda: ctx.forward_all(pb))
    assert st == UNSUPPORTED and "adapter 0" in msg and c.launches() == []
    assert c.status(lambda: ctx.forward(1, pb))[0] == UNSUPPORTED
    ctx.forward(0, pb)
    b.adapter_ids = np.array([1, -1])  # has no pair anywhere
    other = ctx.batch_create(b)
    ctx.forward_all(other)
    pb.destroy(), other.destroy()


def another_device(c):
    """Calls made while the caller's current device is another: everything happens on the context's, and the caller's is current again."""
    ctx = c.context(m=MODEL)
    m = Calls(c, ctx)
    now = C.c_int(-1)
    c.fake.fake_set_device(1)
    st, w = m.weight(64)
    st2, g = m.weight(32, 32, gated=1)
    assert (st, st2) == (0, 0)
    assert m.call("pie_mx_quantise", m.rows(), 3, 64, m.mx()) == 0 and m.call("pie_mx_dequantise", m.mx(), 3, 64, m.rows()) == 0
    assert m.call("pie_mx_norm", m.rows(), None, A, 3, 64, None, m.mx()) == 0
    assert m.call("pie_mx_product", m.mx(), 3, w, m.rows()) == 0 and m.call("pie_mx_swiglu", m.mx(), 3, g, m.mx()) == 0
    parts = (m.b.MxRowsC * 7)(*[m.b.MxRowsC(FP4, A, 2048, A, 128)] * 7)
    assert m.call("pie_load_layer_mx", 0, A, A, parts) == 0
    assert m.call("pie_mx_weight_destroy", w) == 0
    assert c.fake.fake_elsewhere() == 0 and len(c.launches()) > 7
    assert c.fake.hipGetDevice(C.byref(now)) == 0 and now.value == 1
    c.fake.fake_set_device(0)


CASES = {f.__name__: f for f in (another_device, rows_refused, norm_refused, weights_refused, no_memory, layers, adapters)}

if __name__ == "__main__":
    CASES[sys.argv[2]](Child(sys.argv[1]))
    print("case passed")
    sys.exit(0)


@pytest.mark.parametrize("case", list(CASES))
def test_host_path(fake, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, case], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "case passed" in r.stdout, f"exit {r.returncode}\n{r.stdout}\n{r.stderr}"


def test_rows_in_the_binding():
    import torch
    from paper_2510_24051_amd import MxRows
    r = MxRows.empty(3, 96, "mxfp4", "cpu")
    assert (r.rows, r.k) == (3, 96) and r.elements.shape == (3, 48) and r.scales.shape == (3, 4)
    assert MxRows.empty(0, 32, "mxfp8", "cpu").rows == 0
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    MxRows("mxfp8", u8(4, 64).view(torch.float8_e4m3fn), u8(4, 4).view(torch.float8_e8m0fnu))
    MxRows("mxfp8", u8(4, 128)[:, :64], u8(4, 12)[:, 4:8])
    for bad in (("mxfp6", u8(4, 64), u8(4, 4)), ("mxfp8", u8(4, 48), u8(4, 4)), ("mxfp8", u8(4, 64), u8(4, 2)), ("mxfp8", u8(4, 64), u8(3, 4)),
                ("mxfp4", u8(4, 64).view(torch.float8_e4m3fn), u8(4, 4)), ("mxfp8", u8(4, 64).float(), u8(4, 4)), ("mxfp8", u8(64, 4).T, u8(4, 4)),
                ("mxfp8", u8(4, 0), u8(4, 0)), ("mxfp8", u8(4), u8(4, 4))):
        with pytest.raises(ValueError):
            MxRows(*bad)
    with pytest.raises(ValueError):
        MxRows.empty(3, 40, "mxfp8", "cpu")


def test_contexts_that_only_plan_refuse_in_the_binding():
    import torch
    from types import SimpleNamespace
    from paper_2510_24051_amd import MxRows, MxWeight, Pie, PieError
    p = Pie.planner(MODEL, 32, 16, 8, 4)
    r, x = MxRows.empty(2, 64, "mxfp8", "cpu"), torch.zeros((2, 64))
    w = MxWeight(SimpleNamespace(ctx=None), 1, 64, 64, False)
    for call in (lambda: p.mx_quantise(x, r), lambda: p.mx_dequantise(r, x), lambda: p.mx_norm(x, x[0].bfloat16(), r), lambda: p.mx_product(r, w, x),
                 lambda: p.mx_swiglu(r, w, r), lambda: p.mx_weight([r]), lambda: p.load_layer_mx(0, None)):
        with pytest.raises(PieError) as e:
            call()
        assert e.value.status == INVALID and "only plans" in str(e.value)


def test_every_form_is_listed():
    """Which forms the listed products go through, by the library's own rule; some split over workgroups, some cut behind whole rounds of tiles."""
    from paper_2510_24051_amd import mx_product_plan
    for gated in (False, True):
        for form in ("mxfp8", "mxfp4"):
            plans = [mx_product_plan(m, n, k, g, f) for g, f, m, k, n in FORM_SIZES if (g, f) == (gated, form)]
            assert {(p["tile_rows"], p["tile_columns"], p["k_slices"]) for p in plans} == FORMS[gated]
            assert any(p["splits"] > 1 for p in plans) and any(p["rows"] < r[2] for p, r in zip(plans, [s for s in FORM_SIZES if s[:2] == (gated, form)])) or not gated
    assert any(mx_product_plan(m, n, k, g, f)["rows"] < m for g, f, m, k, n in FORM_SIZES if not g)


def test_plans():
    """What a plan may be: parts no more than stages, sums that fit the workspace, whole rounds of whole tiles; and what is refused."""
    from paper_2510_24051_amd import PieError, mx_product_plan
    rng = np.random.default_rng(0)
    for _ in range(3000):
        m, n, k = (int(2 ** rng.uniform(0, b)) for b in (14, 15, 10))
        k, gated, form = 32 * k, bool(rng.integers(2)), ["mxfp8", "mxfp4"][rng.integers(2)]
        n = (n + 31) // 32 * 32 if gated else n
        p = mx_product_plan(m, n, k, gated, form, int(rng.choice([256, 64, 304])))
        assert (p["tile_rows"], p["tile_columns"], p["k_slices"]) in FORMS[gated] and 1 <= p["rows"] <= m and 1 <= p["splits"] <= 8
        assert p["tile_rows"] < 256 or (m > 128 and p["splits"] == 1)
        assert p["rows"] == m or (p["tile_rows"] == 256 and p["rows"] % 256 == 0)
        if p["splits"] > 1:
            assert p["splits"] * m * (n + 31) // 32 * 32 * (2 if gated else 1) <= 1 << 24
            assert p["splits"] * p["k_slices"] * 2 <= -(-k // (128 if form == "mxfp8" else 256))
    for bad in ((0, 32, 32), (1, 0, 32), (1, 32, 0), (1, 32, 48), (1, 33, 32, True), (1, 32, 32, False, "mxfp6"), (1, 32, 32, False, "mxfp8", 0)):
        with pytest.raises(PieError) as e:
            mx_product_plan(*bad)
        assert e.value.status == INVALID
    for bad in ((1 << 25, 32, 32), (1, 1 << 25, 32), (1, 1 << 24, 32, True), (1, 32, 1 << 21)):
        with pytest.raises(PieError) as e:
            mx_product_plan(*bad)
        assert e.value.status == UNSUPPORTED
