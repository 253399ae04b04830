"""ctypes binding of libpie_mi355.so.  Every method marshals arguments for the C call of the same
name (pie_<method>) and does nothing else: all computation runs in the HIP kernels.  PyTorch is
used for device memory and the stream only.  There is no CPU fallback: a missing library raises."""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libpie_mi355.so"

PIE_N_STAGES = 13
STAGE_NAMES = ["norm1", "qkv", "rope_append", "attn_decode", "attn_prefill", "attn_merge", "oproj", "norm2",
               "gateup", "down", "head_norm", "lm_head", "topk"]
TAP_Q, TAP_ATTN, TAP_RESID, TAP_ACT, TAP_LOGITS = 0, 1, 2, 3, 4

STATUS = {0: "PIE_OK", -1: "PIE_EINVAL", -2: "PIE_ERANGE", -3: "PIE_EBATCH", -4: "PIE_ECONFLICT", -5: "PIE_ENOMEM",
          -6: "PIE_EHIP", -7: "PIE_EUNSUPPORTED"}


class PieError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class ModelDescC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("hidden", "n_q_heads", "n_kv_heads", "head_dim", "mlp_dim", "vocab",
                                          "page_size")] + [("rms_eps", C.c_float), ("rope_theta", C.c_float),
                                                           ("n_layers", C.c_int32)]


class PoolDescC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_kv_pages", "n_embeds", "max_batch_tokens", "max_batch_requests",
                                          "max_top_k", "max_dist_rows", "max_adapters", "max_lora_rank")]


class ForwardBatchC(C.Structure):
    _fields_ = [("n_requests", C.c_int32), ("n_tokens", C.c_int32), ("tok_indptr", C.c_void_p),
                ("in_embed_ids", C.c_void_p), ("out_embed_ids", C.c_void_p), ("positions", C.c_void_p),
                ("page_indptr", C.c_void_p), ("page_ids", C.c_void_p), ("kv_len", C.c_void_p),
                ("mask_indptr", C.c_void_p), ("mask_words", C.c_void_p), ("adapter_ids", C.c_void_p)]


class BeamSearchC(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("group_indptr", C.c_void_p), ("scores", C.c_void_p), ("finished", C.c_void_p),
                ("eos_token", C.c_int32), ("n_out", C.c_int32), ("temperature", C.c_float)]


_ROWS = struct.Struct("@Pi4xq")  # pie_rows: data, dtype, row_stride


class MxRowsC(C.Structure):
    _fields_ = [("format", C.c_int32), ("elements", C.c_void_p), ("row_bytes", C.c_int64), ("scales", C.c_void_p), ("scale_bytes", C.c_int64)]


def lib_path() -> str:
    return os.path.join(HERE, _LIB_NAME)


_lib = None


def load_library():
    """Load the built library; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: build it with `python -m paper_2510_24051_amd.build` "
                                "(or __graft_entry__.build()); the HIP path has no fallback")
    lib = C.CDLL(path)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    sigs = {
        "pie_create": [C.POINTER(ModelDescC), C.POINTER(PoolDescC), vp, C.POINTER(vp)],
        "pie_destroy": [vp],
        "pie_load_layer": [vp, i32] + [vp] * 9,
        "pie_load_head": [vp, vp, vp],
        "pie_embed_write": [vp, vp, i32, vp],
        "pie_embed_read": [vp, vp, i32, vp],
        "pie_kv_write": [vp, i32, vp, vp, i32, vp, vp],
        "pie_kv_read": [vp, i32, vp, vp, i32, vp, vp],
        "pie_batch_create": [vp, C.POINTER(ForwardBatchC), i32, C.POINTER(vp)],
        "pie_batch_destroy": [vp, vp],
        "pie_forward": [vp, i32, vp],
        "pie_forward_all": [vp, vp],
        "pie_load_embedding": [vp, vp],
        "pie_load_adapter": [vp, i32, i32, i32, i32, f32, vp, vp],
        "pie_embed_txt": [vp, vp, vp, i32, vp],
        "pie_mask_kvpage": [vp, vp, vp, i32],
        "pie_copy_kvpage": [vp, vp, vp, vp, vp, i32],
        "pie_fork_kvpage": [vp, vp, vp, i32],
        "pie_save_kvpage": [vp, vp, i32, vp],
        "pie_restore_kvpage": [vp, vp, i32, vp],
        "pie_compact_kvpage": [vp, i32] + [vp] * 7,
        "pie_beam_select": [vp, C.POINTER(BeamSearchC), vp, i32, i64, i32, vp, vp, vp],
        "pie_get_next_beams": [vp, C.POINTER(BeamSearchC), vp, vp, vp, vp],
        "pie_mx_quantise": [vp, vp, i32, i32, vp],
        "pie_mx_dequantise": [vp, vp, i32, i32, vp],
        "pie_mx_norm": [vp, vp, vp, vp, i32, i32, vp, vp],
        "pie_mx_weight_create": [vp, C.POINTER(MxRowsC), vp, i32, i32, i32, C.POINTER(vp)],
        "pie_mx_weight_destroy": [vp, vp],
        "pie_mx_product": [vp, vp, i32, vp, vp],
        "pie_mx_swiglu": [vp, vp, i32, vp, vp],
        "pie_mx_product_plan": [i32, i32, i32, i32, i32, i32, vp],
        "pie_load_layer_mx": [vp, i32, vp, vp, C.POINTER(MxRowsC)],
        "pie_forward_host": [vp, i32, C.POINTER(ForwardBatchC), i32],
        "pie_get_next_dist": [vp, vp, i32, i32, f32, vp, vp],
        "pie_get_next_dist_static": [vp, vp, i32, i32, f32, vp, vp],
        "pie_forward_dist": [vp, vp, vp, i32, i32, f32, vp, vp],
        "pie_synchronize": [vp],
        "pie_read_tap": [vp, i32, vp, i64],
        "pie_set_stage_timing": [vp, i32],
        "pie_stage_times": [vp, vp],
        "pie_batch_work": [vp, vp],
        "pie_batch_plan_info": [vp, vp],
        "pie_batch_plan_parts": [vp, vp],
        "pie_batch_prefill_work": [vp, vp, i32, vp],
        "pie_product_plan": [i32, i32, i32, i64, i32, vp],
        "pie_product_stream": [i32, i32, i32, i64, i32, vp],
        "pie_create_planner": [C.POINTER(ModelDescC), C.POINTER(PoolDescC), i32, C.POINTER(vp)],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = i32
    lib.pie_last_error.argtypes = [vp]
    lib.pie_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def product_plan(rows: int, n_out: int, k: int, workspace_floats: int, n_cus: int = 256) -> dict:
    """pie_product_plan: how a product would be cut into tiles."""
    out = np.zeros(4, dtype=np.int64)
    st = load_library().pie_product_plan(rows, n_out, k, workspace_floats, n_cus, _ptr(out))
    if st != 0:
        raise PieError(st, "pie_product_plan: bad argument")
    return {"tile_rows": int(out[0]), "splits": int(out[1]), "whole_rows": int(out[2]), "column_fetches": int(out[3])}


def product_stream(rows: int, n_out: int, k: int, workspace_floats: int, n_cus: int = 256) -> dict:
    """pie_product_stream: the streaming kernel's form where it takes a product (tile_rows 0: it does not)."""
    out = np.zeros(3, dtype=np.int64)
    st = load_library().pie_product_stream(rows, n_out, k, workspace_floats, n_cus, _ptr(out))
    if st != 0:
        raise PieError(st, "pie_product_stream: bad argument")
    return {"tile_rows": int(out[0]), "k_slices": int(out[1]), "splits": int(out[2])}


def mx_product_plan(rows: int, n: int, k: int, gated: bool = False, format: str = "mxfp8", n_cus: int = 256) -> dict:
    """pie_mx_product_plan: how a product of microscaled rows is taken."""
    out = np.zeros(5, dtype=np.int64)
    st = load_library().pie_mx_product_plan(rows, n, k, int(gated), MX_FORMATS.get(format, -1), n_cus, _ptr(out))
    if st != 0:
        raise PieError(st, "pie_mx_product_plan: bad argument")
    return {"tile_rows": int(out[0]), "tile_columns": int(out[1]), "k_slices": int(out[2]), "splits": int(out[3]), "rows": int(out[4])}


_INT32 = np.dtype(np.int32)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, _INT32)


def _ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


_NOTHING = C.c_int32(0)  # where an empty array is said to be: some pointers must not be null


def _at(a):
    """Address of an array that the caller keeps until the call has returned (_ptr keeps it itself and takes four times as long)."""
    if a is None:
        return None
    if a.size == 0:
        return C.addressof(_NOTHING)
    try:
        return C.addressof(C.c_char.from_buffer(a))
    except TypeError:  # a read-only array
        return a.__array_interface__["data"][0]


_row_types = {}  # numbers of the element types that rows may have, and of those that a product may leave


def _types(which: str) -> dict:
    if not _row_types:
        _row_types.update(any={torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}, product={torch.float32: 0, torch.bfloat16: 1})
    return _row_types[which]


MX_FORMATS = {"mxfp8": 0, "mxfp4": 1}


class MxRows:
    """Rows in a microscaled format: `elements` [rows, k] ("mxfp8", one byte each: uint8 or float8_e4m3fn) or [rows, k / 2] ("mxfp4", uint8, the
    first of two in the low half), `scales` (uint8 or float8_e8m0fnu) [rows, k / 32 up to the next multiple of 4].  Rows may be strided
    (elements by multiples of 16 bytes, scales of 4)."""

    def __init__(self, format: str, elements: torch.Tensor, scales: torch.Tensor):
        if format not in MX_FORMATS:
            raise ValueError(f"microscaled rows: format {format!r} is none of {', '.join(MX_FORMATS)}")
        for t, types in ((elements, (torch.uint8, torch.float8_e4m3fn) if format == "mxfp8" else (torch.uint8,)),
                         (scales, (torch.uint8, torch.float8_e8m0fnu))):
            if t.dtype not in types or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
                raise ValueError("microscaled rows: elements and scales are tensors [rows, bytes] of 8-bit types whose rows are contiguous")
        self.format, self.elements, self.scales = format, elements, scales
        self.rows, self.k = elements.shape[0], elements.shape[1] * (1 if format == "mxfp8" else 2)
        if self.k == 0 or self.k % 32 or scales.shape != (self.rows, (self.k // 32 + 3) // 4 * 4):
            raise ValueError("microscaled rows: k is a multiple of 32, and scales are [rows, k / 32 up to the next multiple of 4]")
        self._c = MxRowsC(MX_FORMATS[format], elements.data_ptr(), self._stride(elements), scales.data_ptr(), self._stride(scales))
        self._at = C.addressof(self._c)
        self._index = elements.get_device() if elements.device == scales.device else -1

    @staticmethod
    def _stride(t: torch.Tensor) -> int:
        return t.stride(0) if t.shape[0] > 1 else (t.shape[1] + 15) // 16 * 16

    @classmethod
    def empty(cls, rows: int, k: int, format: str, device="cuda") -> "MxRows":
        if k <= 0 or k % 32:
            raise ValueError("microscaled rows: k is a multiple of 32")
        return cls(format, torch.empty((rows, k // (2 if format == "mxfp4" else 1)), dtype=torch.uint8, device=device),
                   torch.empty((rows, (k // 32 + 3) // 4 * 4), dtype=torch.uint8, device=device))


class MxWeight:
    """Weights of products (pie_mx_weight_create): `n` output rows (of a gated weight: the gate's), `k` inputs.  destroy() frees it; one that is only
    dropped is freed when its context next makes a weight, synchronizes or is closed: Python drops things at any time, and freeing waits for the
    GPU, which ends a capture on whatever stream."""

    def __init__(self, owner: "Pie", handle, n: int, k: int, gated: bool):
        self.owner, self.handle, self.n, self.k, self.gated = owner, handle, n, k, gated

    def destroy(self):
        if self.handle is not None and self.owner.ctx is not None:
            self.owner._check(self.owner.lib.pie_mx_weight_destroy(self.owner.ctx, self.handle))
        self.handle = None

    def __del__(self):
        if self.handle is not None and getattr(self.owner, "ctx", None) is not None:
            self.owner.__dict__.setdefault("_dropped", []).append(self.handle)


class PieBatch:
    def __init__(self, owner: "Pie", handle, keepalive):
        self.owner, self.handle, self._keep = owner, handle, keepalive

    def work(self) -> dict:
        out = np.zeros(6, dtype=np.int64)
        self.owner._check(self.owner.lib.pie_batch_work(self.handle, _ptr(out)))
        return {"kv_bytes": int(out[0]), "kv_bytes_decode": int(out[1]), "attn_flops": int(out[2]),
                "visited_pages": int(out[3]), "kv_bytes_unique": int(out[4]), "kv_bytes_requested": int(out[5])}

    def plan_info(self) -> dict:
        out = np.zeros(8, dtype=np.int64)
        self.owner._check(self.owner.lib.pie_batch_plan_info(self.handle, _ptr(out)))
        return {"decode_waves": int(out[0]), "segments": int(out[1]), "max_pairs_per_wave": int(out[2]),
                "prefill_items": int(out[3]), "decode_requests": int(out[4]), "rows_cap": int(out[5]),
                "prefill_workgroups": int(out[6]), "prefill_workgroups_pair_weights": int(out[7])}

    def plan_parts(self) -> dict:
        out = np.zeros(4, dtype=np.int64)
        self.owner._check(self.owner.lib.pie_batch_plan_parts(self.handle, _ptr(out)))
        return {"cut_blocks": int(out[0]), "most_parts": int(out[1]), "wide_groups": int(out[2]), "most_wide_parts": int(out[3])}

    def prefill_work(self) -> np.ndarray:
        """[n, 3] int32 (request, query block, kv head) per workgroup of the two prefill launches, one after the
        other (sizes in plan_info); request -1 = empty."""
        n = C.c_int32(0)
        self.owner._check(self.owner.lib.pie_batch_prefill_work(self.handle, None, 0, C.byref(n)))
        out = np.zeros((max(n.value, 1), 3), dtype=np.int32)
        self.owner._check(self.owner.lib.pie_batch_prefill_work(self.handle, _ptr(out), n.value, C.byref(n)))
        return out[:n.value]

    def destroy(self):
        if self.handle is not None:
            self.owner.lib.pie_batch_destroy(self.owner.ctx, self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Pie:
    """One context = one GPU = one stream.  bf16 tensors cross this binding as uint16 numpy arrays (host)
    or torch.bfloat16 CUDA tensors (device)."""

    _dropped = ()  # handles of microscaled weights that nothing names any more (a list, once there is one)

    def __init__(self, model, n_kv_pages: int, n_embeds: int, max_batch_tokens: int, max_batch_requests: int,
                 max_top_k: int = 256, max_dist_rows: int = 0, n_layers: int = 1, device: str = "cuda:0",
                 stream: Optional[torch.cuda.Stream] = None, max_adapters: int = 0, max_lora_rank: int = 0):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the HIP path cannot run (there is no CPU fallback)")
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.Stream(device=self.device)
        self.model, self.n_layers, self._page_image = model, n_layers, self._image_of_page(model, n_layers)
        md = ModelDescC(model.hidden, model.n_q_heads, model.n_kv_heads, model.head_dim, model.mlp_dim, model.vocab,
                        model.page_size, model.rms_eps, model.rope_theta, n_layers)
        pd = PoolDescC(n_kv_pages, n_embeds, max_batch_tokens, max_batch_requests, max_top_k, max_dist_rows,
                       max_adapters, max_lora_rank)
        h = C.c_void_p()
        st = self.lib.pie_create(C.byref(md), C.byref(pd), C.c_void_p(self.stream.cuda_stream), C.byref(h))
        if st != 0:
            raise PieError(st, self.lib.pie_last_error(None).decode())
        self.ctx = h
        self._index, self._raw_stream = self.device.index, self.stream.cuda_stream
        self._before, self._after = torch.cuda.Event(), torch.cuda.Event()

    @classmethod
    def planner(cls, model, n_kv_pages: int, n_embeds: int, max_batch_tokens: int, max_batch_requests: int,
                n_layers: int = 1, max_adapters: int = 0, max_lora_rank: int = 0, wave_slots: int = 2048) -> "Pie":
        """A context that only deserialises and plans batches (pie_create_planner): needs no GPU.  batch_create,
        PieBatch.work / plan_info and mask_kvpage work on it; everything else raises PieError."""
        self = cls.__new__(cls)
        self.lib = load_library()
        self.device, self.stream, self.model, self.n_layers, self._page_image = None, None, model, n_layers, self._image_of_page(model, n_layers)
        md = ModelDescC(model.hidden, model.n_q_heads, model.n_kv_heads, model.head_dim, model.mlp_dim, model.vocab,
                        model.page_size, model.rms_eps, model.rope_theta, n_layers)
        pd = PoolDescC(n_kv_pages, n_embeds, max_batch_tokens, max_batch_requests, 0, 0, max_adapters, max_lora_rank)
        h = C.c_void_p()
        st = self.lib.pie_create_planner(C.byref(md), C.byref(pd), int(wave_slots), C.byref(h))
        if st != 0:
            raise PieError(st, self.lib.pie_last_error(None).decode())
        self.ctx = h
        return self

    # ---- helpers ----
    @staticmethod
    def _image_of_page(model, n_layers: int) -> tuple:
        return (n_layers, 2, model.page_size, model.n_kv_heads, model.head_dim)

    def _check(self, st: int):
        if st != 0:
            raise PieError(st, self.lib.pie_last_error(self.ctx).decode())

    def _ordered(self, call, *args):
        """A call that works on the caller's tensors: on the context's stream, behind what torch's current stream holds (what made them,
        what their memory was used for before), and in front of what that stream gets afterwards."""
        if torch._C._cuda_getCurrentRawStream(self._index) == self._raw_stream:
            st = call(*args)
            return self._check(st) if st != 0 else None
        if self._raw_stream == 0 and torch.cuda.is_current_stream_capturing():  # (waiting there for an event of the capture has ended the process)
            raise PieError(-6, "the context's stream is the device's default stream, which cannot be captured: give the context a stream of its own")
        current = torch.cuda.current_stream(self.device)
        self._before.record(current)
        self.stream.wait_event(self._before)
        st = call(*args)
        self._after.record(self.stream)
        current.wait_event(self._after)
        self._check(st)

    def _device(self) -> torch.device:
        """The context's device (a number belongs to it), as its tensors name it."""
        if self.device is None:
            raise PieError(-1, "the context only plans batches (pie_create_planner)")
        return self.device

    def _dev_bf16(self, bits) -> torch.Tensor:
        if isinstance(bits, torch.Tensor):
            assert bits.dtype == torch.bfloat16 and bits.is_cuda and bits.is_contiguous()
            return bits
        a = np.ascontiguousarray(bits, dtype=np.uint16)
        t = torch.from_numpy(a.view(np.int16)).to(self.device, non_blocking=False)
        return t.view(torch.bfloat16)

    def close(self):
        if getattr(self, "ctx", None) is not None:
            self.lib.pie_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- weights ----
    def load_layer(self, layer: int, w):
        names = ("g1", "wq", "wk", "wv", "wo", "g2", "wgate", "wup", "wdown")
        ts = [self._dev_bf16(getattr(w, n)) for n in names]
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_load_layer(self.ctx, layer, *[C.c_void_p(t.data_ptr()) for t in ts]))
        del ts

    def load_layer_mx(self, layer: int, w):
        """pie_load_layer_mx: w.g1 and w.g2 as for load_layer, w.wq, w.wk, w.wv, w.wo, w.wgate, w.wup and w.wdown MxRows in MXFP4."""
        m, dev = self.model, self._device()
        q, kv = m.n_q_heads * m.head_dim, m.n_kv_heads * m.head_dim
        shapes = {"wq": (q, m.hidden), "wk": (kv, m.hidden), "wv": (kv, m.hidden), "wo": (m.hidden, q), "wgate": (m.mlp_dim, m.hidden),
                  "wup": (m.mlp_dim, m.hidden), "wdown": (m.hidden, m.mlp_dim)}
        parts = [getattr(w, n) for n in self.PROJECTIONS]
        for n, p in zip(self.PROJECTIONS, parts):
            if not isinstance(p, MxRows) or p.format != "mxfp4" or (p.rows, p.k) != shapes[n] or p._index != self._index:
                raise ValueError(f"load_layer_mx: {n} is {shapes[n]} in mxfp4 on the context's device")
        g = [self._dev_bf16(x) for x in (w.g1, w.g2)]
        if any(x.numel() != m.hidden for x in g):
            raise ValueError("load_layer_mx: gains have one value per hidden dimension")
        torch.cuda.synchronize(dev)
        self._check(self.lib.pie_load_layer_mx(self.ctx, layer, g[0].data_ptr(), g[1].data_ptr(), (MxRowsC * 7)(*[p._c for p in parts])))

    def load_head(self, head):
        g = None if head.g_final is None else self._dev_bf16(head.g_final)
        w = self._dev_bf16(head.w_lm)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_load_head(self.ctx, None if g is None else C.c_void_p(g.data_ptr()),
                                           C.c_void_p(w.data_ptr())))

    def load_embedding(self, table_bits):
        t = self._dev_bf16(table_bits)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_load_embedding(self.ctx, C.c_void_p(t.data_ptr())))

    PROJECTIONS = ("wq", "wk", "wv", "wo", "wgate", "wup", "wdown")

    def load_adapter(self, adapter: int, layers):
        """`layers[l]` maps projection names to (A bits [rank, in], B bits [out, rank], scale)."""
        for l, d in enumerate(layers):
            for name, (a_bits, b_bits, scale) in d.items():
                a, b = self._dev_bf16(a_bits), self._dev_bf16(b_bits)
                torch.cuda.synchronize(self.device)
                self._check(self.lib.pie_load_adapter(self.ctx, adapter, l, self.PROJECTIONS.index(name), a.shape[0],
                                                      float(scale), C.c_void_p(a.data_ptr()), C.c_void_p(b.data_ptr())))

    # ---- resources ----
    def embed_txt(self, token_ids, positions, embed_ids):
        tok, pos, ids = _i32(token_ids), _i32(positions), _i32(embed_ids)
        if not (len(tok) == len(pos) == len(ids)):
            raise ValueError("embed_txt: token_ids, positions and embed_ids must have one length")
        self._check(self.lib.pie_embed_txt(self.ctx, _ptr(tok), _ptr(pos), len(tok), _ptr(ids)))

    def embed_write(self, embed_ids, bits):
        ids = _i32(embed_ids)
        t = self._dev_bf16(bits)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_embed_write(self.ctx, _ptr(ids), len(ids), C.c_void_p(t.data_ptr())))

    def embed_read(self, embed_ids) -> np.ndarray:
        ids = _i32(embed_ids)
        t = torch.empty((len(ids), self.model.hidden), dtype=torch.bfloat16, device=self.device)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_embed_read(self.ctx, _ptr(ids), len(ids), C.c_void_p(t.data_ptr())))
        return t.view(torch.int16).cpu().numpy().view(np.uint16)

    def kv_write(self, layer: int, page_ids, slots, k_bits, v_bits, chunk: int = 1 << 16):
        p, s = _i32(page_ids), _i32(slots)
        k_bits = np.ascontiguousarray(k_bits, dtype=np.uint16)
        v_bits = np.ascontiguousarray(v_bits, dtype=np.uint16)
        for a in range(0, len(p), chunk):  # bounded staging copies
            b = min(len(p), a + chunk)
            k, v = self._dev_bf16(k_bits[a:b]), self._dev_bf16(v_bits[a:b])
            torch.cuda.synchronize(self.device)
            self._check(self.lib.pie_kv_write(self.ctx, layer, _ptr(p[a:b].copy()), _ptr(s[a:b].copy()), b - a,
                                              C.c_void_p(k.data_ptr()), C.c_void_p(v.data_ptr())))

    def mask_kvpage(self, page_ids, visible_bits):
        p = _i32(page_ids)
        bits = np.ascontiguousarray(visible_bits, dtype=np.uint32)
        if len(p) != len(bits):
            raise ValueError("mask_kvpage: one mask per page")
        self._check(self.lib.pie_mask_kvpage(self.ctx, _ptr(p), _ptr(bits), len(p)))

    def copy_kvpage(self, src_pages, src_slots, dst_pages, dst_slots):
        a = [_i32(x) for x in (src_pages, src_slots, dst_pages, dst_slots)]
        if len({len(x) for x in a}) != 1:
            raise ValueError("copy_kvpage: four arrays of one length")
        self._check(self.lib.pie_copy_kvpage(self.ctx, *[_ptr(x) for x in a], len(a[0])))

    def fork_kvpage(self, src_pages, dst_pages):
        s, d = _i32(src_pages), _i32(dst_pages)
        if len(s) != len(d):
            raise ValueError("fork_kvpage: one destination per source")
        self._check(self.lib.pie_fork_kvpage(self.ctx, _at(s), _at(d), len(s)))

    def _move_image(self, call, page_ids, image: torch.Tensor):
        ids = np.ascontiguousarray(page_ids, _INT32)
        n = len(ids)
        if image.shape != (n, *self._page_image) or image.dtype is not torch.bfloat16 or image.device != self._device() or not image.is_contiguous():
            raise ValueError("an image of pages is a contiguous bfloat16 device tensor [pages, layers, 2, page_size, kv heads, head_dim]")
        self._ordered(call, self.ctx, ids.tobytes(), n, image.data_ptr())

    def save_kvpage(self, page_ids, image: torch.Tensor):
        """Enqueues the copy of the pages into `image` [pages, layers, 2, page_size, kv heads, head_dim]; torch's current stream sees it
        whole.  The pages' masks are not in it."""
        self._move_image(self.lib.pie_save_kvpage, page_ids, image)

    def restore_kvpage(self, page_ids, image: torch.Tensor):
        """Enqueues the copy of `image`, as torch's current stream leaves it, into the pages; that stream may write it again at once.
        The pages keep the masks that they have."""
        self._move_image(self.lib.pie_restore_kvpage, page_ids, image)

    def compact_kvpage(self, page_indptr, page_ids, kv_len, shifts=None, dst_page_indptr=None, dst_page_ids=None) -> np.ndarray:
        """Returns the sequences' new lengths; the moves are enqueued.  Pages left behind keep the masks that hid the evicted tokens: set
        them (mask_kvpage) before they are another's."""
        ip, ids, kl = _i32(page_indptr), _i32(page_ids), _i32(kv_len)
        sh = None if shifts is None else _i32(shifts)
        if (dst_page_indptr is None) != (dst_page_ids is None):
            raise ValueError("compact_kvpage: dst_page_indptr and dst_page_ids are given together")
        dp, di = (None, None) if dst_page_indptr is None else (_i32(dst_page_indptr), _i32(dst_page_ids))
        if len(ip) != len(kl) + 1 or ip[-1] != len(ids) or (sh is not None and len(sh) != kl.sum()) or \
                (dp is not None and (len(dp) != len(kl) + 1 or dp[-1] != len(di))):
            raise ValueError("compact_kvpage: arrays of lengths that do not belong together")
        out = np.zeros(len(kl), dtype=np.int32)
        self._check(self.lib.pie_compact_kvpage(self.ctx, len(kl), _at(ip), _at(ids), _at(kl), _at(dp), _at(di), _at(sh), _at(out)))
        return out

    def kv_read(self, layer: int, page_ids, slots):
        p, s = _i32(page_ids), _i32(slots)
        m = self.model
        k = torch.empty((len(p), m.n_kv_heads, m.head_dim), dtype=torch.bfloat16, device=self.device)
        v = torch.empty_like(k)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_kv_read(self.ctx, layer, _ptr(p), _ptr(s), len(p), C.c_void_p(k.data_ptr()),
                                         C.c_void_p(v.data_ptr())))
        f = lambda t: t.view(torch.int16).cpu().numpy().view(np.uint16)
        return f(k), f(v)

    # ---- forward ----
    def _batch_struct(self, b):
        arrs = dict(tok_indptr=_i32(b.tok_indptr), in_embed_ids=_i32(b.in_embed_ids),
                    out_embed_ids=_i32(b.out_embed_ids),
                    positions=None if b.positions is None else _i32(b.positions),
                    page_indptr=_i32(b.page_indptr), page_ids=_i32(b.page_ids), kv_len=_i32(b.kv_len))
        mi = None if b.mask_indptr is None else np.ascontiguousarray(b.mask_indptr, dtype=np.int64)
        mw = None if b.mask_words is None else np.ascontiguousarray(b.mask_words, dtype=np.uint32)
        ad = getattr(b, "adapter_ids", None)
        ad = None if ad is None else _i32(ad)
        fb = ForwardBatchC(int(b.n_requests), int(b.n_tokens), _ptr(arrs["tok_indptr"]), _ptr(arrs["in_embed_ids"]),
                           _ptr(arrs["out_embed_ids"]), _ptr(arrs["positions"]), _ptr(arrs["page_indptr"]),
                           _ptr(arrs["page_ids"]), _ptr(arrs["kv_len"]), _ptr(mi), _ptr(mw), _ptr(ad))
        return fb, (arrs, mi, mw, ad)

    def batch_create(self, batch, validate: bool = True) -> PieBatch:
        fb, keep = self._batch_struct(batch)
        h = C.c_void_p()
        self._check(self.lib.pie_batch_create(self.ctx, C.byref(fb), int(validate), C.byref(h)))
        return PieBatch(self, h, keep)

    def forward(self, layer: int, batch: PieBatch):
        self._check(self.lib.pie_forward(self.ctx, layer, batch.handle))

    def forward_all(self, batch: PieBatch):
        self._check(self.lib.pie_forward_all(self.ctx, batch.handle))

    def forward_host(self, layer: int, batch, validate: bool = True):
        fb, keep = self._batch_struct(batch)
        self._check(self.lib.pie_forward_host(self.ctx, layer, C.byref(fb), int(validate)))

    # ---- sample ----
    def get_next_dist_async(self, embed_ids, top_k: int, temperature: float, out_ids: torch.Tensor,
                            out_probs: torch.Tensor):
        ids = _i32(embed_ids)
        self._check(self.lib.pie_get_next_dist(self.ctx, _ptr(ids), len(ids), top_k, float(temperature),
                                               C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_probs.data_ptr())))

    def get_next_dist_static_async(self, embed_ids, top_k: int, temperature: float, out_ids: torch.Tensor,
                                   out_probs: torch.Tensor):
        """pie_get_next_dist_static: the allocation-free variant (at most 32 rows); outputs are caller tensors."""
        ids = _i32(embed_ids)
        self._check(self.lib.pie_get_next_dist_static(self.ctx, _ptr(ids), len(ids), top_k, float(temperature),
                                                      C.c_void_p(out_ids.data_ptr()), C.c_void_p(out_probs.data_ptr())))

    def forward_dist(self, batch: PieBatch, rows, top_k: int, temperature: float = 1.0):
        r = _i32(rows)
        oi = torch.empty((len(r), top_k), dtype=torch.int32, device=self.device)
        op = torch.empty((len(r), top_k), dtype=torch.float32, device=self.device)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_forward_dist(self.ctx, batch.handle, _ptr(r), len(r), top_k, float(temperature),
                                              C.c_void_p(oi.data_ptr()), C.c_void_p(op.data_ptr())))
        self.synchronize()
        return oi.cpu().numpy(), op.cpu().numpy()

    def get_next_dist(self, embed_ids, top_k: int, temperature: float = 1.0):
        n = len(embed_ids)
        oi = torch.empty((n, top_k), dtype=torch.int32, device=self.device)
        op = torch.empty((n, top_k), dtype=torch.float32, device=self.device)
        torch.cuda.synchronize(self.device)
        self.get_next_dist_async(embed_ids, top_k, temperature, oi, op)
        self.synchronize()
        return oi.cpu().numpy(), op.cpu().numpy()

    @staticmethod
    def _searches(group_indptr) -> np.ndarray:
        ip = _i32(group_indptr)
        if len(ip) < 1:
            raise ValueError("beam search: group_indptr has one entry more than there are searches")
        return ip

    def _beam_search(self, group_indptr, n_out, out_beams, out_tokens, out_scores, scores, finished, eos_token, temperature):
        ip = self._searches(group_indptr)
        G, n, dev = len(ip) - 1, int(ip[-1]), self._device()
        for t, dt in ((out_beams, torch.int32), (out_tokens, torch.int32), (out_scores, torch.float32)):
            if t.dtype != dt or t.device != dev or not t.is_contiguous() or t.numel() != G * n_out:
                raise ValueError("beam search: outputs are contiguous device tensors [groups, n_out] of int32, int32 and float32")
        for t, dts in ((scores, (torch.float32,)), (finished, (torch.uint8, torch.bool))):
            if t is not None and (t.dtype not in dts or t.device != dev or not t.is_contiguous() or t.numel() != n):
                raise ValueError("beam search: scores (float32) and finished (uint8 or bool) are contiguous device tensors [rows]")
        at = lambda t: None if t is None else t.data_ptr()
        return BeamSearchC(G, _at(ip), at(scores), at(finished), int(eos_token), int(n_out), float(temperature)), ip

    def beam_select_async(self, logits: torch.Tensor, group_indptr, n_out: int, out_beams: torch.Tensor, out_tokens: torch.Tensor,
                          out_scores: torch.Tensor, scores: Optional[torch.Tensor] = None, finished: Optional[torch.Tensor] = None,
                          eos_token: int = -1, temperature: float = 1.0):
        """pie_beam_select over `logits` [rows, vocab] (float32, bfloat16 or float16; rows may be strided); the outputs are the
        caller's tensors [groups, n_out], complete when the context's stream has got there.  Inputs are as torch's current stream
        leaves them, and what that stream gets afterwards sees the outputs."""
        b, keep = self._beam_search(group_indptr, n_out, out_beams, out_tokens, out_scores, scores, finished, eos_token, temperature)
        types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        if logits.dtype not in types or logits.device != self._device() or logits.dim() != 2 or logits.shape[0] != keep[-1] or \
                (logits.shape[1] > 1 and logits.stride(1) != 1):
            raise ValueError("beam_select: logits are a device tensor [rows, vocab] of float32, bfloat16 or float16 whose rows are contiguous")
        stride = logits.stride(0) if logits.shape[0] > 1 else logits.shape[1]
        self._ordered(self.lib.pie_beam_select, self.ctx, C.byref(b), logits.data_ptr(), types[logits.dtype], stride, logits.shape[1],
                      out_beams.data_ptr(), out_tokens.data_ptr(), out_scores.data_ptr())

    def get_next_beams_async(self, embed_ids, group_indptr, n_out: int, out_beams: torch.Tensor, out_tokens: torch.Tensor,
                             out_scores: torch.Tensor, scores: Optional[torch.Tensor] = None, finished: Optional[torch.Tensor] = None,
                             eos_token: int = -1, temperature: float = 1.0):
        """pie_get_next_beams; arguments and streams as for beam_select_async."""
        ids = _i32(embed_ids)
        b, keep = self._beam_search(group_indptr, n_out, out_beams, out_tokens, out_scores, scores, finished, eos_token, temperature)
        if len(ids) != keep[-1]:
            raise ValueError("get_next_beams: one Embed per row")
        self._ordered(self.lib.pie_get_next_beams, self.ctx, C.byref(b), _at(ids), out_beams.data_ptr(), out_tokens.data_ptr(), out_scores.data_ptr())

    def get_next_beams(self, embed_ids, group_indptr, n_out: int, scores=None, finished=None, eos_token: int = -1, temperature: float = 1.0):
        """The same with host arrays: (beams, tokens, scores) [groups, n_out], after the stream has been waited for."""
        G = len(self._searches(group_indptr)) - 1
        dev = lambda a, dt: None if a is None else torch.from_numpy(np.array(a, dtype=dt)).to(self.device)
        s, f = dev(scores, np.float32), dev(finished, np.uint8)
        ob, ot = (torch.empty((G, n_out), dtype=torch.int32, device=self.device) for _ in range(2))
        os_ = torch.empty((G, n_out), dtype=torch.float32, device=self.device)
        torch.cuda.synchronize(self.device)
        self.get_next_beams_async(embed_ids, group_indptr, n_out, ob, ot, os_, s, f, eos_token, temperature)
        self.synchronize()
        return ob.cpu().numpy(), ot.cpu().numpy(), os_.cpu().numpy()

    # ---- microscaled formats ----
    # Inputs are as torch's current stream leaves them, and what that stream gets afterwards sees the outputs.
    def _rows(self, t: torch.Tensor, rows: int, k: int, what: str, types: dict) -> bytes:
        """pie_rows of a tensor."""
        number, shape, strides = types.get(t.dtype), t.shape, t.stride()
        if number is None or len(shape) != 2 or shape[0] != rows or shape[1] != k or strides[1] != 1 or t.get_device() != self._index:
            raise ValueError(f"{what} is a tensor [{rows}, {k}] on the context's device whose rows are contiguous, of "
                             + ", ".join(str(x).replace("torch.", "") for x in types))
        return _ROWS.pack(t.data_ptr(), number, strides[0] if rows > 1 else k)

    def _mx_rows(self, r: MxRows, rows: int, k: int, what: str) -> int:
        """Address of r's pie_mx_rows."""
        if self.device is None:
            self._device()  # (says why)
        if not isinstance(r, MxRows) or r.rows != rows or r.k != k or r._index != self._index:
            raise ValueError(f"{what}: MxRows of {rows} rows of {k} on the context's device")
        return r._at

    def mx_quantise(self, x: torch.Tensor, out: MxRows):
        """pie_mx_quantise: out = x [rows, k] (float32, bfloat16 or float16; rows may be strided)."""
        rows, k = out.rows, out.k
        o = self._mx_rows(out, rows, k, "mx_quantise")
        self._ordered(self.lib.pie_mx_quantise, self.ctx, self._rows(x, rows, k, "mx_quantise: x", _types("any")), rows, k, o)

    def mx_dequantise(self, a: MxRows, out: torch.Tensor):
        """pie_mx_dequantise: out [rows, k] (float32, bfloat16 or float16; rows may be strided) = the values of a."""
        r = self._mx_rows(a, a.rows, a.k, "mx_dequantise")
        self._ordered(self.lib.pie_mx_dequantise, self.ctx, r, a.rows, a.k, self._rows(out, a.rows, a.k, "mx_dequantise: out", _types("any")))

    def mx_norm(self, x: torch.Tensor, gain: torch.Tensor, out: MxRows, delta: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None):
        """pie_mx_norm: h = x + delta, out = rmsnorm(h) * gain.  gain: bfloat16 [k]; h may be x."""
        rows, k, types = out.rows, out.k, _types("any")
        o = self._mx_rows(out, rows, k, "mx_norm")
        if gain.dtype is not torch.bfloat16 or gain.shape != (k,) or gain.get_device() != self._index or not gain.is_contiguous():
            raise ValueError("mx_norm: gain is a contiguous bfloat16 tensor [k] on the context's device")
        rx = self._rows(x, rows, k, "mx_norm: x", types)
        rd = None if delta is None else self._rows(delta, rows, k, "mx_norm: delta", types)
        if h is not None and h.dtype is not x.dtype:
            raise ValueError("mx_norm: h has x's type")
        rh = None if h is None else rx if h is x else self._rows(h, rows, k, "mx_norm: h", types)
        self._ordered(self.lib.pie_mx_norm, self.ctx, rx, rd, gain.data_ptr(), rows, k, rh, o)

    def mx_weight(self, parts, gated: bool = False) -> MxWeight:
        """pie_mx_weight_create: matrices in MXFP4, one below the other, or gate and up."""
        parts, dev = list(parts), self._device()
        if not parts or any(not isinstance(p, MxRows) or p.k != parts[0].k or p._index != self._index for p in parts):
            raise ValueError("mx_weight: MxRows of one k on the context's device")
        torch.cuda.synchronize(dev)
        self._free_dropped()
        n = np.array([p.rows for p in parts], _INT32)
        h = C.c_void_p()
        self._check(self.lib.pie_mx_weight_create(self.ctx, (MxRowsC * len(parts))(*[p._c for p in parts]), _ptr(n), len(parts), parts[0].k, int(gated),
                                                  C.byref(h)))
        return MxWeight(self, h, int(n[0] if gated else n.sum()), parts[0].k, gated)

    def _free_dropped(self):
        while self._dropped:
            self._check(self.lib.pie_mx_weight_destroy(self.ctx, self._dropped.pop()))

    def _mx_weight(self, w: MxWeight, a: MxRows, what: str) -> int:
        self._device()
        if not isinstance(w, MxWeight) or w.handle is None or w.owner.ctx is None:
            raise ValueError(f"{what}: the weight is an MxWeight that has not been destroyed, nor its context closed")
        return self._mx_rows(a, a.rows, w.k, what)

    def mx_product(self, a: MxRows, w: MxWeight, out: torch.Tensor):
        """pie_mx_product: out [rows, n] (bfloat16 or float32; rows may be strided) = a w^T."""
        r = self._mx_weight(w, a, "mx_product")
        self._ordered(self.lib.pie_mx_product, self.ctx, r, a.rows, w.handle,
                      self._rows(out, a.rows, w.n, "mx_product: out", _types("product")))

    def mx_swiglu(self, a: MxRows, w: MxWeight, out: MxRows):
        """pie_mx_swiglu: out [rows, n] = silu(a gate^T) * (a up^T) for a gated weight."""
        r = self._mx_weight(w, a, "mx_swiglu")
        self._ordered(self.lib.pie_mx_swiglu, self.ctx, r, a.rows, w.handle, self._mx_rows(out, a.rows, w.n, "mx_swiglu: out"))

    def synchronize(self):
        self._check(self.lib.pie_synchronize(self.ctx))
        self._free_dropped()

    # ---- observation ----
    def read_tap(self, which: int, rows: int) -> np.ndarray:
        m = self.model
        if which in (TAP_Q, TAP_ATTN):
            shape, dt = (rows, m.n_q_heads * m.head_dim), torch.bfloat16
        elif which == TAP_RESID:
            shape, dt = (rows, m.hidden), torch.float32
        elif which == TAP_ACT:
            shape, dt = (rows, m.mlp_dim), torch.bfloat16
        else:
            shape, dt = (rows, m.vocab), torch.float32
        t = torch.empty(shape, dtype=dt, device=self.device)
        torch.cuda.synchronize(self.device)
        self._check(self.lib.pie_read_tap(self.ctx, which, C.c_void_p(t.data_ptr()), t.numel()))
        if dt == torch.bfloat16:
            return t.view(torch.int16).cpu().numpy().view(np.uint16)
        return t.cpu().numpy()

    def set_stage_timing(self, enabled: bool):
        self._check(self.lib.pie_set_stage_timing(self.ctx, int(enabled)))

    def stage_times(self) -> dict:
        out = np.zeros(PIE_N_STAGES, dtype=np.float32)
        self._check(self.lib.pie_stage_times(self.ctx, _ptr(out)))
        return {STAGE_NAMES[i]: float(out[i]) for i in range(PIE_N_STAGES)}
