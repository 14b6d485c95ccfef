"""Python binding of libwq.so (include/wq.h): argument marshalling, and two helpers that
prepare arguments (rope_table, tree_mask).

Every function here converts torch tensors to device pointers and sizes,
calls the C ABI of the same name on the current CUDA stream, and raises
``WQError`` on a non-zero status.  All other arithmetic runs in the CUDA kernels;
there is no fallback: if the library is missing or no GPU is present the
calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

from . import _build

WQ_PRENORM = 1
WQ_LAUNCH_CHAIN = 2
WQ_LAUNCH_STACK = 4
WQ_HEAD_NORM = 8
WQ_BF16 = 0
WQ_F32 = 1

_STATUS = {0: "WQ_OK", -1: "WQ_ERR_ARG", -2: "WQ_ERR_SHAPE", -3: "WQ_ERR_ALIGN", -4: "WQ_ERR_UNSUPPORTED",
           -5: "WQ_ERR_CUDA", -6: "WQ_ERR_TIMEOUT", -7: "WQ_ERR_WORKSPACE"}


class WQError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


class _QWeight(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("meta", ctypes.c_void_p), ("n", ctypes.c_int32),
                ("k", ctypes.c_int32), ("group", ctypes.c_int32), ("bits", ctypes.c_int32)]


class _MLPLayer(ctypes.Structure):
    _fields_ = [("gate", _QWeight), ("up", _QWeight), ("down", _QWeight), ("lora_a", ctypes.c_void_p),
                ("lora_b_gate", ctypes.c_void_p), ("lora_b_up", ctypes.c_void_p), ("r", ctypes.c_int32),
                ("lora_scale", ctypes.c_float)]


class _DecoderLayer(ctypes.Structure):
    _fields_ = [("qkv", _QWeight), ("o", _QWeight), ("mlp", _MLPLayer), ("n_heads", ctypes.c_int32),
                ("n_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rope_theta", ctypes.c_float)]


class _MoELayer(ctypes.Structure):
    _fields_ = [("experts", _MLPLayer), ("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32)]


class _KVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_meta", ctypes.c_void_p),
                ("v_meta", ctypes.c_void_p), ("batch", ctypes.c_int32), ("n_kv", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("bits", ctypes.c_int32)]


_lib = None


def library_path() -> str:
    """libwq.so, or the bounds-checking debug build when WQ_DEBUG_LIB=1."""
    return _build.DEBUG_LIB_PATH if os.environ.get("WQ_DEBUG_LIB") == "1" else _build.LIB_PATH


def lib():
    """The loaded libwq.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(f"libwq.so not found at {path}: run __graft_entry__.build() first")
        L = ctypes.CDLL(path)
        P, I, S, F, U = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float, ctypes.c_uint
        QP = ctypes.POINTER(_QWeight)
        CP, L3 = ctypes.POINTER(_KVCache), ctypes.POINTER(ctypes.c_int64)
        sig = {
            "wq_packed_sizes": (I, [I, I, I, I, ctypes.POINTER(S), ctypes.POINTER(S)]),
            "wq_pack": (I, [P, I, I, I, I, QP, P, P]),
            "wq_pack_w2": (I, [P, I, I, I, QP, P, P]),
            "wq_pack_w4": (I, [P, I, I, I, QP, P, P]),
            "wq_merge_lora": (I, [QP, P, P, I, F, P, QP, P, P]),
            "wq_workspace_bytes": (S, [I, I, I, I]),
            "wq_workspace_init": (I, [P, S, P]),
            "wq_gateup_w2_lora": (I, [P, I, QP, QP, P, P, P, I, F, U, P, P, S, P]),
            "wq_gateup_w2_lora_noalloc": (I, [P, I, QP, QP, P, P, P, I, F, U, P, P]),
            "wq_gateup_w3_lora": (I, [P, I, QP, QP, P, P, P, I, F, U, P, P, S, P]),
            "wq_gateup_w4": (I, [P, I, QP, QP, U, P, P, S, P]),
            "wq_down_w4": (I, [P, I, QP, P, P, I, P, S, P]),
            "wq_down_bf16": (I, [P, I, P, I, I, P, P, I, P]),
            "wq_mlp_forward": (I, [P, I, ctypes.POINTER(_MLPLayer), I, U, P, P, S, P]),
            "wq_mlp_forward_states": (I, [P, I, ctypes.POINTER(_MLPLayer), I, U, P, P, P, P, S, P]),
            "wq_mlp_forward_info": (I, [I, ctypes.POINTER(_MLPLayer), I, U, ctypes.POINTER(ctypes.c_int64)]),
            "wq_plan_info": (I, [I, I, I, I, I, I, ctypes.POINTER(ctypes.c_int64)]),
            "wq_attn_workspace_bytes": (S, [I, I, I, I, I]),
            "wq_attn_decode": (I, [P, P, P, I, I, I, I, I, F, P, P, I, P, P, S, P]),
            "wq_decoder_workspace_bytes": (S, [I, ctypes.POINTER(_DecoderLayer), I]),
            "wq_decoder_layer_forward": (I, [P, I, P, ctypes.POINTER(_DecoderLayer), P, P, I, U, P, P, S, P]),
            "wq_kv_append": (I, [CP, P, P, I, I, L3, L3, P, P, P, I, P]),
            "wq_kv_read": (I, [CP, P, P, I, P, P, I, P]),
            "wq_qkv_rope": (I, [P, P, I, I, P, P, I, I, I, I, U, P, P, P, P]),
            "wq_attn_tree_workspace_bytes": (S, [I, I, I, I, I, I]),
            "wq_attn_tree": (I, [P, P, P, I, I, CP, P, P, P, F, P, P, S, P]),
            "wq_decoder_tree_workspace_bytes": (S, [I, I, ctypes.POINTER(_DecoderLayer), I]),
            "wq_decoder_tree_forward": (I, [P, I, P, P, ctypes.POINTER(_DecoderLayer), CP, P, I, P, P, U, P, P, P, P,
                                            S, P]),
            "wq_moe_workspace_bytes": (S, [I, ctypes.POINTER(_MoELayer), U]),
            "wq_moe_forward": (I, [P, I, P, ctypes.POINTER(_MoELayer), U, P, P, P, P, P, P, S, P]),
            "wq_wait_check": (I, [P]),
            "wq_last_error": (ctypes.c_char_p, []),
            "wq_device_status": (I, [ctypes.POINTER(I)]),
            "wq_version": (ctypes.c_char_p, []),
            "wq_debug_record": (I, [ctypes.POINTER(ctypes.c_longlong)]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise WQError(status, lib().wq_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _raw_stream() -> int:
    """The current stream's handle, without the Stream object that torch.cuda.current_stream() makes."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


@dataclass
class QWeight:
    """A packed group-quantized matrix [n, k] held in two device tensors."""
    codes: torch.Tensor   # int32 words
    meta: torch.Tensor    # int16 (binary16 bit patterns)
    n: int
    k: int
    group: int
    bits: int

    def c(self) -> _QWeight:
        return _QWeight(self.codes.data_ptr(), self.meta.data_ptr(), self.n, self.k, self.group, self.bits)

    @property
    def nbytes(self) -> int:
        return self.codes.numel() * 4 + self.meta.numel() * 2


def dense_weight(w: torch.Tensor) -> QWeight:
    """A dense bf16 [n, k] matrix as a down weight of wq_mlp_forward (bits 16;
    the BF16/W2-GateUp configuration)."""
    assert w.dtype == torch.bfloat16 and w.is_cuda and w.is_contiguous()
    n, k = w.shape
    return QWeight(w.view(torch.int16).view(-1), torch.zeros(8, dtype=torch.int16, device=w.device), n, k, 0, 16)


def packed_sizes(bits: int, n: int, k: int, group: int):
    cb, mb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().wq_packed_sizes(bits, n, k, group, ctypes.byref(cb), ctypes.byref(mb)))
    return cb.value, mb.value


def empty_qweight(n: int, k: int, group: int, bits: int, device="cuda") -> QWeight:
    cb, mb = packed_sizes(bits, n, k, group)
    return QWeight(torch.empty(cb // 4, dtype=torch.int32, device=device),
                   torch.empty(mb // 2, dtype=torch.int16, device=device), n, k, group, bits)


def pack(w: torch.Tensor, group: int, bits: int, nonfinite: torch.Tensor | None = None,
         out: QWeight | None = None) -> QWeight:
    """Quantize and pack an fp32 [n, k] device matrix (wq_pack)."""
    assert w.dtype == torch.float32 and w.is_cuda and w.is_contiguous()
    n, k = w.shape
    q = out if out is not None else empty_qweight(n, k, group, bits, device=w.device)
    cq = q.c()
    _check(lib().wq_pack(_ptr(w), n, k, group, bits, ctypes.byref(cq), _ptr(nonfinite), _stream()))
    return q


def pack_w2(w, group, nonfinite=None):
    return pack(w, group, 2, nonfinite)


def pack_w4(w, group, nonfinite=None):
    return pack(w, group, 4, nonfinite)


def merge_lora(src: QWeight, lora_b: torch.Tensor | None, lora_a: torch.Tensor | None, lora_scale: float,
               out: QWeight | None = None, w_merged: torch.Tensor | None = None,
               nonfinite: torch.Tensor | None = None) -> QWeight:
    """Merge an adapter into a packed matrix and quantize it again (wq_merge_lora).

    lora_b is bf16 [n, r] and lora_a bf16 [r, k], contiguous on the device (None
    for r = 0).  ``out=src`` merges in place; ``w_merged`` (fp32 [n, k]) receives
    the merged matrix before quantization.
    """
    r = 0 if lora_b is None else lora_b.shape[1]
    if r:
        assert lora_b.dtype == torch.bfloat16 and lora_a.dtype == torch.bfloat16
        assert lora_b.is_contiguous() and lora_a.is_contiguous()
        assert tuple(lora_b.shape) == (src.n, r) and tuple(lora_a.shape) == (r, src.k)
    if w_merged is None:
        w_merged = torch.empty(src.n, src.k, dtype=torch.float32, device=src.codes.device)
    q = out if out is not None else empty_qweight(src.n, src.k, src.group, src.bits, device=src.codes.device)
    cs, cq = src.c(), q.c()
    _check(lib().wq_merge_lora(ctypes.byref(cs), _ptr(lora_b) if r else None, _ptr(lora_a) if r else None, r,
                               float(lora_scale), _ptr(w_merged), ctypes.byref(cq), _ptr(nonfinite), _stream()))
    return q


def workspace_bytes(m: int, d: int, inter: int, r: int = 0) -> int:
    return int(lib().wq_workspace_bytes(m, d, inter, r))


def workspace(m: int, d: int, inter: int, r: int = 0, device="cuda") -> torch.Tensor:
    """A zero-initialised workspace tensor for up to m tokens of a (d, inter) layer."""
    nb = workspace_bytes(m, d, inter, r)
    if nb == 0:
        raise WQError(-2, f"no workspace size for m={m}, d={d}, inter={inter}")
    ws = torch.empty(nb, dtype=torch.uint8, device=device)
    _check(lib().wq_workspace_init(_ptr(ws), nb, _stream()))
    return ws


def gateup_w2_lora(x, gate: QWeight, up: QWeight, lora_a=None, lora_b_gate=None, lora_b_up=None,
                   lora_scale: float = 0.0, prenorm: bool = False, h=None, ws=None):
    m, d = x.shape
    r = 0 if lora_b_gate is None else lora_b_gate.shape[1]
    if h is None:
        h = torch.empty((m, gate.n), dtype=torch.bfloat16, device=x.device)
    if ws is None:
        ws = workspace(max(m, 1), d, gate.n, r, device=x.device)
    cg, cu = gate.c(), up.c()
    _check(lib().wq_gateup_w2_lora(_ptr(x), m, ctypes.byref(cg), ctypes.byref(cu), _ptr(lora_a), _ptr(lora_b_gate),
                                   _ptr(lora_b_up), r, float(lora_scale), WQ_PRENORM if prenorm else 0, _ptr(h),
                                   _ptr(ws), ws.numel(), _stream()))
    return h


def gateup_w3_lora(x, gate: QWeight, up: QWeight, lora_a=None, lora_b_gate=None, lora_b_up=None,
                   lora_scale: float = 0.0, prenorm: bool = False, h=None, ws=None):
    """wq_gateup_w3_lora: gateup_w2_lora with 3-bit gate/up codes (App. B)."""
    m, d = x.shape
    r = 0 if lora_b_gate is None else lora_b_gate.shape[1]
    if h is None:
        h = torch.empty((m, gate.n), dtype=torch.bfloat16, device=x.device)
    if ws is None:
        ws = workspace(max(m, 1), d, gate.n, r, device=x.device)
    cg, cu = gate.c(), up.c()
    _check(lib().wq_gateup_w3_lora(_ptr(x), m, ctypes.byref(cg), ctypes.byref(cu), _ptr(lora_a), _ptr(lora_b_gate),
                                   _ptr(lora_b_up), r, float(lora_scale), WQ_PRENORM if prenorm else 0, _ptr(h),
                                   _ptr(ws), ws.numel(), _stream()))
    return h


def gateup_w2_lora_noalloc(x, gate: QWeight, up: QWeight, lora_a=None, lora_b_gate=None, lora_b_up=None,
                           lora_scale: float = 0.0, prenorm: bool = False, h=None):
    """wq_gateup_w2_lora_noalloc: the same call with the library's built-in scratch.

    For callers that cannot allocate device memory; ``h`` may be passed in so
    that nothing is allocated on the Python side either.
    """
    m, d = x.shape
    r = 0 if lora_b_gate is None else lora_b_gate.shape[1]
    if h is None:
        h = torch.empty((m, gate.n), dtype=torch.bfloat16, device=x.device)
    cg, cu = gate.c(), up.c()
    _check(lib().wq_gateup_w2_lora_noalloc(_ptr(x), m, ctypes.byref(cg), ctypes.byref(cu), _ptr(lora_a),
                                           _ptr(lora_b_gate), _ptr(lora_b_up), r, float(lora_scale),
                                           WQ_PRENORM if prenorm else 0, _ptr(h), _stream()))
    return h


def gateup_w4(x, gate: QWeight, up: QWeight, prenorm: bool = False, h=None, ws=None):
    m, d = x.shape
    if h is None:
        h = torch.empty((m, gate.n), dtype=torch.bfloat16, device=x.device)
    if ws is None:
        ws = workspace(max(m, 1), d, gate.n, 0, device=x.device)
    cg, cu = gate.c(), up.c()
    _check(lib().wq_gateup_w4(_ptr(x), m, ctypes.byref(cg), ctypes.byref(cu), WQ_PRENORM if prenorm else 0, _ptr(h),
                              _ptr(ws), ws.numel(), _stream()))
    return h


def down_w4(h, down: QWeight, residual=None, out_f32: bool = False, y=None, ws=None):
    m, inter = h.shape
    if y is None:
        y = torch.empty((m, down.n), dtype=torch.float32 if out_f32 else torch.bfloat16, device=h.device)
    if ws is None:
        ws = workspace(max(m, 1), down.n, inter, 0, device=h.device)
    cd = down.c()
    _check(lib().wq_down_w4(_ptr(h), m, ctypes.byref(cd), _ptr(residual), _ptr(y), WQ_F32 if out_f32 else WQ_BF16,
                            _ptr(ws), ws.numel(), _stream()))
    return y


def down_bf16(h, wd, residual=None, out_f32: bool = False, y=None):
    """y = residual + h Wd^T with a bf16 Wd [d, inter] (wq_down_bf16)."""
    assert h.dtype == torch.bfloat16 and wd.dtype == torch.bfloat16 and h.is_contiguous() and wd.is_contiguous()
    m, inter = h.shape
    d = wd.shape[0]
    assert wd.shape[1] == inter
    if y is None:
        y = torch.empty((m, d), dtype=torch.float32 if out_f32 else torch.bfloat16, device=h.device)
    _check(lib().wq_down_bf16(_ptr(h), m, _ptr(wd), d, inter, _ptr(residual), _ptr(y), WQ_F32 if out_f32 else WQ_BF16,
                              _stream()))
    return y


@dataclass
class MLPLayer:
    gate: QWeight
    up: QWeight
    down: QWeight
    lora_a: torch.Tensor | None = None
    lora_b_gate: torch.Tensor | None = None
    lora_b_up: torch.Tensor | None = None
    lora_scale: float = 0.0

    @property
    def r(self) -> int:
        return 0 if self.lora_b_gate is None else self.lora_b_gate.shape[1]

    def c(self) -> _MLPLayer:
        return _MLPLayer(self.gate.c(), self.up.c(), self.down.c(),
                         None if self.lora_a is None else self.lora_a.data_ptr(),
                         None if self.lora_b_gate is None else self.lora_b_gate.data_ptr(),
                         None if self.lora_b_up is None else self.lora_b_up.data_ptr(),
                         self.r, float(self.lora_scale))


def merge_layer(layer: MLPLayer, w_merged: torch.Tensor | None = None) -> MLPLayer:
    """The layer with its gate and up adapters merged into new 2-bit codes
    (wq_merge_lora on each); the merged layer carries no adapter (r = 0)."""
    r = layer.r
    if r == 0:
        return MLPLayer(layer.gate, layer.up, layer.down)
    a = layer.lora_a
    gate = merge_lora(layer.gate, layer.lora_b_gate, a[:r], layer.lora_scale, w_merged=w_merged)
    up = merge_lora(layer.up, layer.lora_b_up, a[r:], layer.lora_scale, w_merged=w_merged)
    return MLPLayer(gate, up, layer.down)


class LayerTable:
    """The C array of wq_mlp_layer for a stack (kept alive for graph replays)."""

    def __init__(self, layers):
        self.layers = list(layers)
        self.array = (_MLPLayer * max(1, len(self.layers)))(*[l.c() for l in self.layers])


def _stack_flags(prenorm: bool, chain: bool, stack: bool = False) -> int:
    return (WQ_PRENORM if prenorm else 0) | (WQ_LAUNCH_CHAIN if chain else 0) | (WQ_LAUNCH_STACK if stack else 0)


def mlp_forward(x, layers, prenorm: bool = True, y=None, ws=None, table: LayerTable | None = None,
                chain: bool = False, stack: bool = False):
    """Stack of gated-MLP layers (wq_mlp_forward) on the current stream; chain=True
    asks for the per-layer launch chain (WQ_LAUNCH_CHAIN), stack=True for the
    single-launch stack kernel (WQ_LAUNCH_STACK)."""
    m, d = x.shape
    if table is None:
        table = LayerTable(layers)
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        l0 = table.layers[0]
        ws = workspace(max(m, 1), d, l0.gate.n, l0.r, device=x.device)
    _check(lib().wq_mlp_forward(_ptr(x), m, table.array, len(table.layers), _stack_flags(prenorm, chain, stack), _ptr(y),
                                _ptr(ws), ws.numel(), _stream()))
    return y


def mlp_forward_states(x, layers, prenorm: bool = True, states=None, h_states=None, y=None, ws=None,
                       table: LayerTable | None = None, chain: bool = False, with_h: bool = False,
                       stack: bool = False):
    """wq_mlp_forward_states: the stack plus every layer's output, bf16 [n_layers, m, d], and with
    with_h=True every layer's h, bf16 [n_layers, m, inter].  Returns (y, states, h_states)."""
    m, d = x.shape
    if table is None:
        table = LayerTable(layers)
    n = len(table.layers)
    inter = table.layers[0].gate.n
    if states is None:
        states = torch.empty((n, m, d), dtype=torch.bfloat16, device=x.device)
    if h_states is None and with_h:
        h_states = torch.empty((n, m, inter), dtype=torch.bfloat16, device=x.device)
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        l0 = table.layers[0]
        ws = workspace(max(m, 1), d, l0.gate.n, l0.r, device=x.device)
    _check(lib().wq_mlp_forward_states(_ptr(x), m, table.array, n, _stack_flags(prenorm, chain, stack), _ptr(y),
                                       _ptr(states), _ptr(h_states), _ptr(ws), ws.numel(), _stream()))
    return y, states, h_states


ROUTE_GEMV_CHAIN, ROUTE_GEMM_CHAIN, ROUTE_STACK = 0, 1, 2
_STEP_FIELDS = ("rb", "kp", "wk", "tpw", "panels", "ctas")


def mlp_forward_info(m: int, layers, prenorm: bool = True, table: LayerTable | None = None,
                     chain: bool = False, stack: bool = False) -> dict:
    """How wq_mlp_forward would run this stack (wq_mlp_forward_info)."""
    if table is None:
        table = LayerTable(layers)
    arr = (ctypes.c_int64 * 16)()
    _check(lib().wq_mlp_forward_info(m, table.array, len(table.layers), _stack_flags(prenorm, chain, stack), arr))
    v = list(arr)
    out = {"route": v[0]}
    if v[0] == ROUTE_STACK:
        out["stack"] = dict(zip(("ctas", "stages", "stage_bytes", "h_barrier", "warps_per_tile", "tiles_per_cta",
                                 "smem"), v[1:8]))
    if v[0] == ROUTE_GEMV_CHAIN:
        out["gateup"] = dict(zip(_STEP_FIELDS, v[1:7]))
        out["down"] = dict(zip(_STEP_FIELDS, v[7:13]))
        out["panel"] = bool(v[13])
    return out


PLAN_FIELDS = ("row_tiles", "kblocks", "rb", "kp", "wk", "panels", "ctas", "threads", "smem", "tok_chunk")
KIND_GATEUP_W2, KIND_GATEUP_W4, KIND_DOWN_W4, KIND_GATEUP_W3 = 0, 1, 2, 3


def plan_info(kind: int, n: int, k: int, m: int, group: int, r: int = 0) -> dict:
    """The launch decomposition the library would use on the current device."""
    arr = (ctypes.c_int64 * 10)()
    _check(lib().wq_plan_info(kind, n, k, m, group, r, arr))
    return dict(zip(PLAN_FIELDS, list(arr)))


def attn_workspace(batch: int, n_heads: int, n_kv: int, head_dim: int, max_len: int, device="cuda") -> torch.Tensor:
    nb = int(lib().wq_attn_workspace_bytes(batch, n_heads, n_kv, head_dim, max_len))
    if nb == 0:
        raise WQError(-2, "no attention workspace for these sizes")
    return torch.empty(nb, dtype=torch.uint8, device=device)


def attn_decode(qkv, x, lens, k_cache, v_cache, n_heads: int, n_kv: int, theta: float, o=None, ws=None):
    """wq_attn_decode: one decode step of grouped-query attention; the caches
    (bf16 [B, n_kv, max_len, head_dim]) gain position lens[b]."""
    b, d = x.shape
    _, hkv, max_len, hd = k_cache.shape
    assert hkv == n_kv and lens.dtype == torch.int32
    if o is None:
        o = torch.empty((b, n_heads * hd), dtype=torch.bfloat16, device=x.device)
    if ws is None:
        ws = attn_workspace(b, n_heads, n_kv, hd, max_len, device=x.device)
    _check(lib().wq_attn_decode(_ptr(qkv), _ptr(x), _ptr(lens), b, d, n_heads, n_kv, hd, float(theta), _ptr(k_cache),
                                _ptr(v_cache), max_len, _ptr(o), _ptr(ws), ws.numel(), _stream()))
    return o


@dataclass
class DecoderLayer:
    """A decoder layer: 4-bit qkv (rows of Wq, Wk, Wv) and o projections around an MLPLayer."""
    qkv: QWeight
    o: QWeight
    mlp: MLPLayer
    n_heads: int
    n_kv: int
    head_dim: int
    rope_theta: float = 1e6

    def c(self) -> _DecoderLayer:
        return _DecoderLayer(self.qkv.c(), self.o.c(), self.mlp.c(), self.n_heads, self.n_kv, self.head_dim,
                             float(self.rope_theta))


def decoder_workspace(batch: int, layer: DecoderLayer, max_len: int, device="cuda") -> torch.Tensor:
    cl = layer.c()
    nb = int(lib().wq_decoder_workspace_bytes(batch, ctypes.byref(cl), max_len))
    if nb == 0:
        raise WQError(-2, "no decoder workspace for these sizes")
    ws = torch.empty(nb, dtype=torch.uint8, device=device)
    _check(lib().wq_workspace_init(_ptr(ws), nb, _stream()))
    return ws


def decoder_layer_forward(x, lens, layer: DecoderLayer, k_cache, v_cache, prenorm: bool = True, y=None, ws=None,
                          c_layer=None):
    """wq_decoder_layer_forward: one decode step of the layer for x bf16 [B, d]."""
    b, d = x.shape
    max_len = k_cache.shape[2]
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = decoder_workspace(b, layer, max_len, device=x.device)
    cl = c_layer if c_layer is not None else layer.c()
    _check(lib().wq_decoder_layer_forward(_ptr(x), b, _ptr(lens), ctypes.byref(cl), _ptr(k_cache), _ptr(v_cache),
                                          max_len, WQ_PRENORM if prenorm else 0, _ptr(y), _ptr(ws), ws.numel(),
                                          _stream()))
    return y


class KVCache:
    """A KV cache [batch, n_kv, max_len, head_dim] of 16 (bf16), 8 or 4 bits (wq_kv_cache): k, v are
    bf16, or uint8 [batch, n_kv, max_len, head_dim * bits / 8] with int32 k_meta, v_meta
    [batch, n_kv, max_len] (scale and zero of a row).  The tensors are held; the C struct is made once."""
    __slots__ = ("_k", "_v", "_k_meta", "_v_meta", "batch", "n_kv", "max_len", "head_dim", "bits", "_c", "_ref")

    def __init__(self, k, v, k_meta, v_meta, head_dim: int, bits: int):
        want = torch.bfloat16 if bits == 16 else torch.uint8
        for t in (k, v):
            assert t.is_cuda and t.dtype == want and t.dim() == 4 and t.is_contiguous() and t.shape == k.shape
            assert t.shape[3] == (head_dim if bits == 16 else head_dim * bits // 8)
        for t in (k_meta, v_meta) if bits != 16 else ():
            assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.shape == k.shape[:3]
        self._k, self._v, self._k_meta, self._v_meta = k, v, k_meta, v_meta
        self.batch, self.n_kv, self.max_len = k.shape[:3]
        self.head_dim, self.bits = head_dim, bits
        meta = [None if t is None else t.data_ptr() for t in (k_meta, v_meta)]
        self._c = _KVCache(k.data_ptr(), v.data_ptr(), *meta, self.batch, self.n_kv, self.max_len, head_dim, bits)
        self._ref = ctypes.byref(self._c)

    k = property(lambda self: self._k)
    v = property(lambda self: self._v)
    k_meta = property(lambda self: self._k_meta)
    v_meta = property(lambda self: self._v_meta)


def kv_cache(batch: int, n_kv: int, max_len: int, head_dim: int, bits: int = 16, device="cuda") -> KVCache:
    """An empty (zero) cache; ``bits`` 16 (bf16), 8 or 4."""
    if bits == 16:
        k, v = (torch.zeros((batch, n_kv, max_len, head_dim), dtype=torch.bfloat16, device=device) for _ in range(2))
        return KVCache(k, v, None, None, head_dim, bits)
    if bits not in (8, 4):
        raise WQError(-4, f"cache bits {bits} not 16, 8 or 4")
    k, v = (torch.zeros((batch, n_kv, max_len, head_dim * bits // 8), dtype=torch.uint8, device=device)
            for _ in range(2))
    km, vm = (torch.zeros((batch, n_kv, max_len), dtype=torch.int32, device=device) for _ in range(2))
    return KVCache(k, v, km, vm, head_dim, bits)


@functools.lru_cache(maxsize=256)
def _strides(s):
    """The first three strides as the C ABI takes them."""
    return (ctypes.c_int64 * 3)(*s[:3])


def _out(t, dtype, shape, device, name):
    """An output tensor and its address: ``t`` checked, or a new one."""
    if t is not None:
        return t, _at(t, dtype, shape, name)
    t = torch.empty(shape, dtype=dtype, device=device)
    return t, t.data_ptr()


def _at(t, dtype, shape, name):
    """The address of a contiguous device tensor of this type and shape (None: NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise AssertionError(f"{name}: contiguous {dtype} {shape} on the device, not {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def kv_append(cache: KVCache, k, v, start, counts=None, index=None):
    """wq_kv_append: rows k, v (bf16 or fp32 [batch, T, n_kv, head_dim], any strides of the first
    three dimensions that are multiples of 16 bytes) quantized into the cache at positions
    start[b] + i; ``index`` [batch, n] picks the source token of row i, ``counts`` [batch] how many."""
    b, dt, shape = cache.batch, k.dtype, k.shape
    t = shape[1]
    assert dt is torch.bfloat16 or dt is torch.float32
    assert shape == (b, t, cache.n_kv, cache.head_dim) and v.shape == shape and v.dtype is dt
    ks, vs = k.stride(), v.stride()
    assert ks[3] == 1 and vs[3] == 1 and k.is_cuda and v.is_cuda
    n = t if index is None else index.shape[1]
    i32 = torch.int32
    _check(lib().wq_kv_append(cache._ref, k.data_ptr(), v.data_ptr(), 1 if dt is torch.float32 else 0, t,
                              _strides(ks), _strides(vs), _at(start, i32, (b,), "start"),
                              _at(counts, i32, (b,), "counts"), _at(index, i32, (b, n), "index"), n, _raw_stream()))


def kv_read(cache: KVCache, start, n: int, counts=None, dtype=torch.bfloat16, k=None, v=None):
    """wq_kv_read: (k, v) [batch, n, n_kv, head_dim] of positions start[b] .. start[b] + n - 1 in bf16 or fp32."""
    assert dtype is torch.bfloat16 or dtype is torch.float32
    b = cache.batch
    shape = (b, n, cache.n_kv, cache.head_dim)
    dev = cache._k.device
    k, kp = _out(k, dtype, shape, dev, "k")
    v, vp = _out(v, dtype, shape, dev, "v")
    _check(lib().wq_kv_read(cache._ref, _at(start, torch.int32, (b,), "start"), _at(counts, torch.int32, (b,), "counts"),
                            n, kp, vp, 1 if dtype is torch.float32 else 0, _raw_stream()))
    return k, v


def rope_table(n_pos: int, head_dim: int, theta: float = 1e6, device="cuda") -> torch.Tensor:
    """fp32 [n_pos, head_dim / 2, 2]: cosine and sine of position * theta^(-2i / head_dim), from fp64 angles."""
    f = theta ** (-2.0 * torch.arange(head_dim // 2, dtype=torch.float64, device=device) / head_dim)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
    return torch.stack([torch.cos(a), torch.sin(a)], -1).to(torch.float32)


def qkv_rope(qkv, positions, table, n_heads: int, n_kv: int, x=None, head_norm: bool = True, q=None, k=None, v=None):
    """wq_qkv_rope: bf16 (q [m, n_heads, hd], k, v [m, n_kv, hd]) from fp32 projections [m, (n_heads + 2 n_kv) hd]."""
    m, n_pos, hd = qkv.shape[0], table.shape[0], 2 * table.shape[1]
    bf, f32, dev = torch.bfloat16, torch.float32, qkv.device
    q, qp = _out(q, bf, (m, n_heads, hd), dev, "q")
    k, kp = _out(k, bf, (m, n_kv, hd), dev, "k")
    v, vp = _out(v, bf, (m, n_kv, hd), dev, "v")
    d = 0 if x is None else x.shape[1]
    _check(lib().wq_qkv_rope(_at(qkv, f32, (m, (n_heads + 2 * n_kv) * hd), "qkv"), _at(x, bf, (m, d), "x"), m, d,
                             _at(positions, torch.int32, (m,), "positions"), _at(table, f32, (n_pos, hd // 2, 2), "table"),
                             n_pos, n_heads, n_kv, hd, WQ_HEAD_NORM if head_norm else 0, qp, kp, vp, _raw_stream()))
    return q, k, v


def tree_mask(parents: torch.Tensor) -> torch.Tensor:
    """The mask of wq_attn_tree for int32 parents [batch, T]: parents[b, i] < i is draft i's parent, -1 the
    context's last token.  int32 [batch, T, ceil(T / 32)]; draft i sees its ancestors and itself.
    Made on the host: parents on the device are copied there (a synchronisation, not for stream capture), and 32 x 128
    drafts take milliseconds.  A loop whose trees keep their shape makes it once; one that draws a tree a step is better
    served by a mask that it writes itself."""
    b, t = parents.shape
    up = parents.cpu().tolist()
    words = (t + 31) // 32
    out = []
    for row in up:
        see = []
        for i, p in enumerate(row):
            assert -1 <= p < i, f"draft {i}: parent {p}"
            see.append((see[p] if p >= 0 else 0) | 1 << i)
        out.append([[(s >> (32 * w)) & 0xffffffff for w in range(words)] for s in see])
    m = torch.tensor(out, dtype=torch.int64).view(b, t, words)
    return torch.where(m >= 2 ** 31, m - 2 ** 32, m).to(torch.int32).to(parents.device)


def attn_tree_workspace(batch: int, n_draft: int, n_heads: int, n_kv: int, head_dim: int, max_len: int,
                        device="cuda") -> torch.Tensor:
    nb = int(lib().wq_attn_tree_workspace_bytes(batch, n_draft, n_heads, n_kv, head_dim, max_len))
    if nb == 0:
        raise WQError(-2, "no attention workspace for these sizes")
    return torch.empty(nb, dtype=torch.uint8, device=device)


def attn_tree(q, k_new, v_new, cache: KVCache, lens, mask=None, counts=None, scale: float | None = None, o=None, ws=None):
    """wq_attn_tree: attention of drafts q [batch, T, n_heads, hd] over the cache's first lens[b] positions
    and the drafts k_new, v_new [batch, T, n_kv, hd] that ``mask`` (int32 [batch, T, ceil(T/32)], see
    tree_mask; None: a chain) lets them see."""
    t, h = q.shape[1], q.shape[2]
    b, hkv, hd = cache.batch, cache.n_kv, cache.head_dim
    bf, i32 = torch.bfloat16, torch.int32
    rows, kv = (b, t, h, hd), (b, t, hkv, hd)
    if o is None:
        o = torch.empty(rows, dtype=bf, device=q.device)
    if ws is None:
        ws = attn_tree_workspace(b, max(t, 1), h, hkv, hd, cache.max_len, device=q.device)
    assert ws.is_cuda
    _check(lib().wq_attn_tree(_at(q, bf, rows, "q"), _at(k_new, bf, kv, "k_new"), _at(v_new, bf, kv, "v_new"), t, h,
                              cache._ref, _at(lens, i32, (b,), "lens"), _at(counts, i32, (b,), "counts"),
                              _at(mask, i32, (b, t, (t + 31) // 32), "mask"), hd ** -0.5 if scale is None else scale,
                              _at(o, bf, rows, "o"), ws.data_ptr(), ws.numel(), _raw_stream()))
    return o


def decoder_tree_workspace(batch: int, n_draft: int, layer: DecoderLayer, max_len: int, device="cuda") -> torch.Tensor:
    cl = layer.c()
    nb = int(lib().wq_decoder_tree_workspace_bytes(batch, n_draft, ctypes.byref(cl), max_len))
    if nb == 0:
        raise WQError(-2, "no decoder workspace for these sizes")
    ws = torch.empty(nb, dtype=torch.uint8, device=device)
    _check(lib().wq_workspace_init(_ptr(ws), nb, _stream()))
    return ws


def decoder_tree_forward(x, lens, positions, layer: DecoderLayer, cache: KVCache, table, mask=None, counts=None,
                         prenorm: bool = True, k_new=None, v_new=None, y=None, ws=None, c_layer=None):
    """wq_decoder_tree_forward: the verify step of a layer for x bf16 [batch, T, d].  Returns
    (y, k_new, v_new); kv_append(cache, k_new, v_new, lens, counts=.., index=..) then keeps the accepted path."""
    b, t, d = x.shape
    bf, i32 = torch.bfloat16, torch.int32
    assert b == cache.batch and d == layer.qkv.k
    kv = (b, t, cache.n_kv, cache.head_dim)
    k_new = torch.empty(kv, dtype=bf, device=x.device) if k_new is None else k_new
    v_new = torch.empty(kv, dtype=bf, device=x.device) if v_new is None else v_new
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = decoder_tree_workspace(b, max(t, 1), layer, cache.max_len, device=x.device)
    assert ws.is_cuda
    n_pos = table.shape[0]
    cl = c_layer if c_layer is not None else layer.c()
    _check(lib().wq_decoder_tree_forward(
        _at(x, bf, (b, t, d), "x"), t, _at(lens, i32, (b,), "lens"), _at(positions, i32, (b, t), "positions"),
        ctypes.byref(cl), cache._ref, _at(table, torch.float32, (n_pos, cache.head_dim // 2, 2), "table"), n_pos,
        _at(counts, i32, (b,), "counts"), _at(mask, i32, (b, t, (t + 31) // 32), "mask"), WQ_PRENORM if prenorm else 0,
        _at(k_new, bf, kv, "k_new"), _at(v_new, bf, kv, "v_new"), _at(y, bf, (b, t, d), "y"), ws.data_ptr(), ws.numel(),
        _raw_stream()))
    return y, k_new, v_new


@dataclass
class MoELayer:
    """A mixture-of-experts block: the experts' matrices stacked row-wise in one
    MLPLayer (gate/up [E*inter, d], down [E*d, inter], lora_a [E*2r, d],
    lora_b_* [E*inter, r]), n_experts experts, top_k of them per token."""
    experts: MLPLayer
    n_experts: int
    top_k: int

    def c(self) -> _MoELayer:
        return _MoELayer(self.experts.c(), self.n_experts, self.top_k)


def moe_workspace(m: int, layer: MoELayer, prenorm: bool = True, device="cuda") -> torch.Tensor:
    cl = layer.c()
    nb = int(lib().wq_moe_workspace_bytes(m, ctypes.byref(cl), WQ_PRENORM if prenorm else 0))
    if nb == 0:
        raise WQError(-2, "no MoE workspace for these sizes")
    ws = torch.empty(nb, dtype=torch.uint8, device=device)
    _check(lib().wq_workspace_init(_ptr(ws), nb, _stream()))
    return ws


def moe_forward(x, logits, layer: MoELayer, prenorm: bool = True, y=None, ws=None, with_slots: bool = False,
                c_layer=None):
    """wq_moe_forward for x bf16 [m, d] and router logits fp32 [m, E].  Returns y,
    or with with_slots (y, expert_idx [m, k], expert_w [m, k], h [m*k, inter], y_slots [m*k, d])."""
    m, d = x.shape
    k = layer.top_k
    inter = layer.experts.gate.n // layer.n_experts
    if y is None:
        y = torch.empty_like(x)
    if ws is None:
        ws = moe_workspace(m, layer, prenorm, device=x.device)
    idx = wt = hs = ys = None
    if with_slots:
        idx = torch.empty((m, k), dtype=torch.int32, device=x.device)
        wt = torch.empty((m, k), dtype=torch.float32, device=x.device)
        hs = torch.empty((m * k, inter), dtype=torch.bfloat16, device=x.device)
        ys = torch.empty((m * k, d), dtype=torch.float32, device=x.device)
    cl = c_layer if c_layer is not None else layer.c()
    _check(lib().wq_moe_forward(_ptr(x), m, _ptr(logits), ctypes.byref(cl), WQ_PRENORM if prenorm else 0, _ptr(y),
                                _ptr(idx), _ptr(wt), _ptr(hs), _ptr(ys), _ptr(ws), ws.numel(), _stream()))
    return (y, idx, wt, hs, ys) if with_slots else y


def wait_check():
    """wq_wait_check: a launch whose bounded waits run out (WQ_ERR_TIMEOUT in the device status)."""
    _check(lib().wq_wait_check(_stream()))


def device_status() -> int:
    v = ctypes.c_int(0)
    _check(lib().wq_device_status(ctypes.byref(v)))
    return v.value


def debug_record():
    """Debug build: (site, line, value, count) of the first failed in-kernel check."""
    rec = (ctypes.c_longlong * 4)()
    _check(lib().wq_debug_record(rec))
    return tuple(rec)


def version() -> str:
    return lib().wq_version().decode()
