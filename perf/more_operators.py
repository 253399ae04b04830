"""A decoder layer in microscaled formats, as measurable cases: quantisation to 8 and 4 bits, the norm that adds the residual and
writes 8 bits with scales, products with weights of 4 bits, and the gated product that leaves its activations in 8 bits.

A row is cut into blocks of 32 values.  A block has one scale, a power of two held as a byte (2^(b - 127)), and elements of E4M3
("mxfp8", a byte each) or E2M1 ("mxfp4", two to a byte, the first in the low half).  The scale of a block is 2^(floor(log2 of its
largest magnitude) - e), e = 8 for E4M3 and 2 for E2M1; elements are rounded to nearest, ties to even, and saturate.  The scales of a row
are followed by as many bytes as make their number a multiple of 4.

Where `own` is false every operator is computed in elementary torch operations.  Where it is true the same passes are made through
the library's entry points.  Elements of 8 bits and scales come back as float8 tensors, elements of 4 bits as the values they stand for.

Sizes are those of the benchmark configurations (tiny layer, 2048-wide model, 8B-shaped model), of their prompts and decode batches."""
import math
from types import SimpleNamespace

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EMAX = {"mxfp8": 8, "mxfp4": 2}
EPS = 1e-5


def listed():
    return [
        # loading a model: the gate and up projections of an 8B-shaped layer, given in bf16, are brought to 4 bits and looked at
        {"name": "quantise_weight", "kind": "quantise", "rows": 28672, "k": 4096, "dtype": "bf16", "gap": 0, "format": "mxfp4"},
        # a decode batch's attention output on its way into the output projection
        {"name": "quantise_64", "kind": "quantise", "rows": 64, "k": 4096, "dtype": "bf16", "gap": 0, "format": "mxfp8"},
        # one token between two blocks: latency counts
        {"name": "norm_1", "kind": "norm", "rows": 1, "k": 4096, "dtype": "f32", "delta": "bf16", "format": "mxfp8"},
        # a ragged decode batch of the 2048-wide model, first norm of the model: no residual to add
        {"name": "norm_157", "kind": "norm", "rows": 157, "k": 2048, "dtype": "bf16", "delta": "", "format": "mxfp8"},
        # eight prompts of 1024 tokens and 128 decode rows: residual stream in fp32, output of the attention block added
        {"name": "norm_8320", "kind": "norm", "rows": 8320, "k": 4096, "dtype": "f32", "delta": "f32", "format": "mxfp8"},
        # the tiny layer's down projection: the smallest product, launches count
        {"name": "product_4", "kind": "product", "rows": 4, "k": 512, "n": 256, "format": "mxfp8"},
        # down projection of 64 decode requests: the longest contraction, a stream of weights
        {"name": "product_64", "kind": "product", "rows": 64, "k": 14336, "n": 4096, "format": "mxfp8"},
        # q, k, v of an odd prompt, activations in 4 bits too
        {"name": "product_333", "kind": "product", "rows": 333, "k": 4096, "n": 6144, "format": "mxfp4"},
        # down projection of the mixed batch
        {"name": "product_8320", "kind": "product", "rows": 8320, "k": 14336, "n": 4096, "format": "mxfp8"},
        # gate and up of one user's token
        {"name": "gated_1", "kind": "gated", "rows": 1, "k": 4096, "n": 14336, "format": "mxfp8", "out": "mxfp8"},
        # of a decode batch
        {"name": "gated_64", "kind": "gated", "rows": 64, "k": 4096, "n": 14336, "format": "mxfp8", "out": "mxfp8"},
        # of the mixed batch: the largest product of a layer
        {"name": "gated_8320", "kind": "gated", "rows": 8320, "k": 4096, "n": 14336, "format": "mxfp8", "out": "mxfp8"},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["quantise", "norm", "product", "product", "gated", "gated"])
    if kind == "quantise":
        k = 32 * log(1, 896)
        return {"kind": kind, "rows": log(1, min(30000, 28672 * 4096 // k)), "k": k, "dtype": rng.choice(["f32", "bf16", "bf16", "f16"]),
                "gap": rng.choice([0, 0, 8, 32]), "format": rng.choice(["mxfp8", "mxfp4"])}
    if kind == "norm":
        return {"kind": kind, "rows": log(1, 8320), "k": 32 * log(8, 128), "dtype": rng.choice(["f32", "bf16"]),
                "delta": rng.choice(["", "f32", "bf16"]), "format": "mxfp8"}
    k, rows = 32 * log(8, 448), log(1, 8320)
    most = 8320 * 4096 * 14336  # products of a listed case
    fmt = rng.choice(["mxfp8", "mxfp8", "mxfp4"])
    if kind == "product":
        return {"kind": kind, "rows": rows, "k": k, "n": log(33, min(28672, most // (rows * k))), "format": fmt}
    return {"kind": kind, "rows": rows, "k": k, "n": 32 * log(4, min(448, most // (rows * k) // 32)), "format": fmt, "out": "mxfp8"}


def work(case):
    rows, k = case["rows"], case["k"]

    def mx(r, c, form):
        return r * (c if form == "mxfp8" else c // 2) + r * (c // 32)

    if case["kind"] == "quantise":
        values = 2 * rows * k if case["format"] == "mxfp4" else 0  # 4 bits come back as values of 16
        return {"bytes": rows * k * DTYPES[case["dtype"]].itemsize + mx(rows, k, case["format"]) + values, "flops": 3 * rows * k}
    if case["kind"] == "norm":
        size = DTYPES[case["dtype"]].itemsize
        moved = rows * k * (size if not case["delta"] else 2 * size + DTYPES[case["delta"]].itemsize)
        return {"bytes": moved + 2 * k + mx(rows, k, case["format"]), "flops": 6 * rows * k}
    if case["kind"] == "product":
        return {"bytes": mx(rows, k, case["format"]) + mx(case["n"], k, "mxfp4") + 2 * rows * case["n"], "flops": 2 * rows * case["n"] * k}
    return {"bytes": mx(rows, k, case["format"]) + mx(2 * case["n"], k, "mxfp4") + mx(rows, case["n"], case["out"]), "flops": 4 * rows * case["n"] * k}


# ------------------------------------------------------------------------------------------------
# the formats, in elementary operations
# ------------------------------------------------------------------------------------------------
def to_mx(y, form):
    """Elements (uint8 codes; two to a byte for mxfp4) and scale bytes [rows, multiple of 4] of fp32 values [rows, k]."""
    rows, k = y.shape
    b = y.reshape(rows, k // 32, 32)
    most = b.abs().amax(-1)
    e = torch.where(most > 0, torch.frexp(most)[1] - 1 - EMAX[form], -127).clamp(-127, 127)
    v = torch.ldexp(b, -e[..., None])
    if form == "mxfp8":
        codes = v.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).reshape(rows, k)
    else:
        a = v.abs()
        c = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
        c = (c + 8 * torch.signbit(v)).to(torch.uint8).reshape(rows, k // 2, 2)
        codes = c[..., 0] + 16 * c[..., 1]
    scales = torch.zeros((rows, (k // 32 + 3) // 4 * 4), dtype=torch.uint8, device=y.device)
    scales[:, :k // 32] = (e + 127).to(torch.uint8)
    return codes, scales


def from_mx(codes, scales, form):
    """fp32 values [rows, k]."""
    rows = codes.shape[0]
    if form == "mxfp8":
        v = codes.view(torch.float8_e4m3fn).to(torch.float32)
    else:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
        v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).reshape(rows, -1)
    k = v.shape[1]
    s = scales[:, :k // 32].contiguous().view(torch.float8_e8m0fnu).to(torch.float32)
    return (v.reshape(rows, k // 32, 32) * s[..., None]).reshape(rows, k)


def shown(codes, scales, k):
    """Elements of 8 bits and their scales, as the numbers that they are."""
    return {"elements": codes.view(torch.float8_e4m3fn), "scales": scales[:, :k // 32].view(torch.float8_e8m0fnu)}


# ------------------------------------------------------------------------------------------------
# what a program has in hand
# ------------------------------------------------------------------------------------------------
def activations(gen, rows, k):
    """Rows as a layer's norm sees them: channels of unlike size, a few of them many times larger."""
    size = torch.exp(0.5 * torch.randn(k, generator=gen, device="cuda"))
    size[torch.randint(0, k, (max(1, k // 256),), generator=gen, device="cuda")] *= 12.0
    return torch.randn((rows, k), generator=gen, device="cuda") * size


def weights(gen, n, k):
    return torch.randn((n, k), generator=gen, device="cuda") * k ** -0.5


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rows, k, form = case["rows"], case["k"], case.get("format")
    s = SimpleNamespace(case=case, ctx=None)
    if case["kind"] == "quantise":
        wide = torch.empty((rows, k + case["gap"]), dtype=DTYPES[case["dtype"]], device="cuda")
        wide[:, :k] = weights(gen, rows, k) if rows > 8320 else activations(gen, rows, k)
        s.x = wide[:, :k]
    elif case["kind"] == "norm":
        s.x = activations(gen, rows, k).to(DTYPES[case["dtype"]])
        s.delta = (0.3 * activations(gen, rows, k)).to(DTYPES[case["delta"]]) if case["delta"] else None
        s.gain = (1.0 + 0.2 * torch.randn(k, generator=gen, device="cuda")).bfloat16()
        s.h = torch.empty_like(s.x) if case["delta"] else None
    else:
        n = case["n"]
        s.a = to_mx(activations(gen, rows, k), form)
        s.w = [to_mx(weights(gen, n, k), "mxfp4") for _ in range(2 if case["kind"] == "gated" else 1)]
        if case["kind"] == "product":
            s.c = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    if own:
        from paper_2510_24051_amd import MxRows, Pie
        model = SimpleNamespace(hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_dim=512, vocab=0, page_size=16, rms_eps=EPS, rope_theta=1e4)
        s.ctx = Pie(model, 1, 1, max_batch_tokens=1, max_batch_requests=1, stream=torch.cuda.current_stream())
        if case["kind"] in ("quantise", "norm"):
            s.to = MxRows.empty(rows, k, form, "cuda")
            s.values = torch.empty((rows, k), dtype=torch.bfloat16, device="cuda") if case["kind"] == "quantise" and form == "mxfp4" else None
        else:
            s.from_ = MxRows(form, *s.a)
            s.weight = s.ctx.mx_weight([MxRows("mxfp4", *w) for w in s.w], gated=case["kind"] == "gated")
            s.to = MxRows.empty(rows, case["n"], case["out"], "cuda") if case["kind"] == "gated" else None
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(s):
    case, k = s.case, s.case["k"]
    if case["kind"] == "quantise":
        if own:
            s.ctx.mx_quantise(s.x, s.to)
            if s.values is None:
                return shown(s.to.elements, s.to.scales, k)
            s.ctx.mx_dequantise(s.to, s.values)
            return {"values": s.values, "scales": shown(s.to.elements, s.to.scales, k)["scales"]}
        codes, scales = to_mx(s.x.float(), case["format"])
        if case["format"] == "mxfp8":
            return shown(codes, scales, k)
        return {"values": from_mx(codes, scales, "mxfp4").bfloat16(), "scales": shown(codes, scales, k)["scales"]}
    if case["kind"] == "norm":
        if own:
            s.ctx.mx_norm(s.x, s.gain, s.to, delta=s.delta, h=s.h)
            got = shown(s.to.elements, s.to.scales, k)
            return got if s.h is None else {**got, "h": s.h}
        h = s.x if s.delta is None else (s.x.float() + s.delta.float()).to(s.x.dtype)
        f = h.float()
        y = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * s.gain.float()
        got = shown(*to_mx(y, case["format"]), k)
        return got if s.delta is None else {**got, "h": h}
    if case["kind"] == "product":
        if own:
            s.ctx.mx_product(s.from_, s.weight, s.c)
            return s.c
        return (from_mx(*s.a, case["format"]) @ from_mx(*s.w[0], "mxfp4").T).bfloat16()
    if own:
        s.ctx.mx_swiglu(s.from_, s.weight, s.to)
        return shown(s.to.elements, s.to.scales, case["n"])
    a = from_mx(*s.a, case["format"])
    g, u = (a @ from_mx(*w, "mxfp4").T for w in s.w)
    return shown(*to_mx(g / (1.0 + torch.exp(-g)) * u, case["out"]), case["n"])


# ------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------
def values64(codes, scales, form):
    """What codes stand for: sign, exponent and fraction taken apart."""
    if form == "mxfp4":
        codes = torch.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    bits, bias = (3, 7) if form == "mxfp8" else (1, 1)
    c = codes.to(torch.int32)
    sign = 1.0 - 2.0 * (c >> (7 if form == "mxfp8" else 3)).double()
    e, f = (c >> bits) & (15 if form == "mxfp8" else 3), (c & ((1 << bits) - 1)).double() / (1 << bits)
    v = sign * torch.where(e > 0, 1.0 + f, f) * torch.exp2((e.clamp(min=1) - bias).double())
    k = v.shape[1]
    s = torch.exp2(scales[:, :k // 32].double() - 127.0)
    return v * s.repeat_interleave(32, 1)


def blocks64(y, form):
    """(elements as values, scales as values) of values [rows, k]."""
    rows, k = y.shape
    most, least, bits = (448.0, -6, 3) if form == "mxfp8" else (6.0, 0, 1)
    b = y.double().reshape(rows, k // 32, 32)
    top = b.abs().amax(-1)
    power = torch.frexp(top)[1].double() - 1.0
    scale = torch.exp2(torch.where(top > 0, power - EMAX[form], torch.full_like(power, -127.0)).clamp(-127.0, 127.0))
    v = b / scale[..., None]
    at = (torch.frexp(v)[1].double() - 1.0).clamp(min=least) - bits  # the last place's power
    v = (torch.round(v * torch.exp2(-at)) * torch.exp2(at)).clamp(-most, most)  # (torch rounds halves to even)
    return v.reshape(rows, k), scale


def exact(case, seed):
    s = prepare_inputs(case, seed)
    if case["kind"] == "quantise":
        v, scale = blocks64(s.x, case["format"])
        return {"elements": v, "scales": scale} if case["format"] == "mxfp8" else {"values": v * scale.repeat_interleave(32, 1), "scales": scale}
    if case["kind"] == "norm":
        h = s.x if s.delta is None else (s.x.double() + s.delta.double()).to(s.x.dtype)
        d = h.double()
        y = d / torch.sqrt((d * d).sum(1, keepdim=True) / d.shape[1] + EPS) * s.gain.double()
        v, scale = blocks64(y, case["format"])
        return {"elements": v, "scales": scale} if s.delta is None else {"elements": v, "scales": scale, "h": h.double()}
    a = values64(*s.a, case["format"])
    if case["kind"] == "product":
        return torch.mm(a, values64(*s.w[0], "mxfp4").T.contiguous())
    g, u = (torch.mm(a, values64(*w, "mxfp4").T.contiguous()) for w in s.w)
    v, scale = blocks64(g * torch.sigmoid(g) * u, case["out"])
    return {"elements": v, "scales": scale}


def prepare_inputs(case, seed):
    """The inputs alone, without the library."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
