"""Thin ctypes binding of libllep.so (include/llep.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels. Tensors are torch tensors on the GPU (torch supplies device memory
and streams); each function passes their data pointers and the current HIP
stream. The library must be built (``__graft_entry__.build()``); nothing
here falls back to another implementation when it is missing.
"""

from __future__ import annotations

import ctypes
import operator
import os
from typing import Optional

from ._build import LIB_PATH

LLEP_OK = 0
LLEP_E_ARG = -1
LLEP_E_WORKSPACE = -2
LLEP_E_DTYPE = -3
LLEP_E_HIP = -4
LLEP_F32 = 0
LLEP_BF16 = 1
LLEP_MODE_LLEP = 0
LLEP_MODE_EP = 1
LLEP_STATUS_BAD_EXPERT_ID = 1
LLEP_STATUS_FFN_WAIT = 2
LLEP_MAX_EXPERTS = 512
LLEP_MAX_DEVICES = 64
LLEP_MAX_FFN_DIM = 65536
LLEP_MAX_NORM_DIM = 8192
LLEP_GATE_NONE, LLEP_GATE_CHANNEL, LLEP_GATE_TOKEN, LLEP_GATE_FULL = range(4)
LLEP_SCORE_SOFTMAX, LLEP_SCORE_SIGMOID = range(2)
LLEP_GROUP_MAX, LLEP_GROUP_TOP2 = range(2)
LLEP_MAX_ROUTE_TOPK = 64
LLEP_MAX_ROUTE_GROUPS = 64

EXPORTED = [
    "llep_plan", "llep_permute", "llep_grouped_ffn", "llep_combine",
    "llep_pack_weights", "llep_plan_max_chunks", "llep_plan_rank_base_elems",
    "llep_grouped_ffn_workspace_bytes", "llep_packed_gate_up_bytes",
    "llep_packed_down_bytes", "llep_last_error", "llep_combine_backward",
    "llep_pack_weights_backward", "llep_grouped_ffn_backward_workspace_bytes",
    "llep_grouped_ffn_backward", "llep_grouped_ffn_train", "llep_grouped_ffn_noalloc",
    "llep_zero_absent_gradients", "llep_block_norm",
    "llep_block_norm_backward_workspace_bytes", "llep_block_norm_backward",
    "llep_clip_gradients_workspace_bytes", "llep_gradient_norm", "llep_clip_gradients",
    "llep_int8_row_bytes", "llep_quantize_rows", "llep_packed_int8_bytes", "llep_pack_int8",
    "llep_int8_matmul_workspace_bytes", "llep_int8_matmul",
    "llep_grouped_ffn_int8_workspace_bytes", "llep_grouped_ffn_int8",
    "llep_grouped_ffn_int8_f32", "llep_combine_to_bf16",
    "llep_route", "llep_route_backward", "llep_mxfp4_row_bytes", "llep_mxfp4_scale_bytes",
    "llep_quantize_rows_mxfp4", "llep_dequantize_rows_mxfp4", "llep_packed_mxfp4_bytes",
    "llep_pack_mxfp4", "llep_mxfp4_matmul", "llep_grouped_ffn_mxfp4_workspace_bytes",
    "llep_grouped_ffn_mxfp4",
]
LLEP_NOALLOC_SCRATCH_BYTES = 64 << 20


class llep_plan_params(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("K", ctypes.c_int32), ("E", ctypes.c_int32),
                ("P", ctypes.c_int32), ("min_chunk", ctypes.c_int32),
                ("capacity", ctypes.c_int64), ("lam", ctypes.c_double),
                ("mode", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class llep_plan_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "status", "n_chunks", "n_groups", "n_xfers", "bypassed", "forced",
        "max_device", "total_rows")]


_P = ctypes.c_void_p


class llep_plan_buffers(ctypes.Structure):
    _fields_ = [(n, _P) for n in (
        "loads", "chunks", "chunk_row", "expert_chunk_begin", "groups",
        "group_begin", "device_rows", "xfers", "rank_base", "info")]


class llep_gradient(ctypes.Structure):
    _fields_ = [("data", _P), ("out", _P), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


_DTYPE_OF, _IS_CUDA = operator.attrgetter("dtype"), operator.attrgetter("is_cuda")


class llep_route_params(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64)] + [
        (n, ctypes.c_int32) for n in ("K", "E", "score", "groups", "top_groups", "group_score",
                                      "renormalize")] + [("scale", ctypes.c_float)]


class LLEPError(RuntimeError):
    def __init__(self, code: int, where: str, msg: str):
        super().__init__(f"{where} failed with code {code}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load libllep.so (once). Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        pp = ctypes.POINTER(llep_plan_params)
        pb = ctypes.POINTER(llep_plan_buffers)
        pg = ctypes.POINTER(llep_gradient)
        pr = ctypes.POINTER(llep_route_params)
        i32, i64, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        f32 = ctypes.c_float
        sigs = {
            "llep_plan_max_chunks": (i32, [pp]),
            "llep_plan_rank_base_elems": (i64, [pp]),
            "llep_plan": (ctypes.c_int, [pp, _P, pb, _P]),
            "llep_permute": (ctypes.c_int, [pp, pb, _P, _P, _P, i32, ctypes.c_int, _P, _P,
                                            _P, _P, _P]),
            "llep_packed_gate_up_bytes": (sz, [i32, i32, i32, ctypes.c_int]),
            "llep_packed_down_bytes": (sz, [i32, i32, i32, ctypes.c_int]),
            "llep_pack_weights": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, _P, _P, _P, _P,
                                                 _P, _P]),
            "llep_grouped_ffn_workspace_bytes": (sz, [pp, i32, ctypes.c_int]),
            "llep_grouped_ffn": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, i32, i32,
                                                ctypes.c_int, _P, _P, sz, _P]),
            "llep_grouped_ffn_train": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, i32, i32,
                                                      ctypes.c_int, _P, _P, _P, sz, _P]),
            "llep_grouped_ffn_noalloc": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, i32, i32,
                                                        ctypes.c_int, _P, _P]),
            "llep_combine": (ctypes.c_int, [pp, _P, _P, _P, i32, ctypes.c_int, _P, _P]),
            "llep_combine_backward": (ctypes.c_int, [pp, _P, _P, _P, _P, i32, ctypes.c_int, _P,
                                                     _P, _P]),
            "llep_pack_weights_backward": (ctypes.c_int, [i32, i32, i32, ctypes.c_int, _P, _P,
                                                          _P, _P, _P, _P]),
            "llep_grouped_ffn_backward_workspace_bytes": (sz, [pp, i32, i32, ctypes.c_int]),
            "llep_grouped_ffn_backward": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, _P, _P, _P,
                                                         i32, i32, ctypes.c_int, _P, _P, _P, _P,
                                                         _P, sz, _P]),
            "llep_zero_absent_gradients": (ctypes.c_int, [pp, pb, i32, i32, i32, _P, _P, _P, _P]),
            "llep_block_norm": (ctypes.c_int, [i64, i32, ctypes.c_int, _P, _P, _P, ctypes.c_int,
                                               _P, _P, f32, f32, _P, _P, _P, _P, i32, _P]),
            "llep_block_norm_backward_workspace_bytes": (sz, [i64, i32]),
            "llep_block_norm_backward": (ctypes.c_int, [i64, i32, ctypes.c_int, _P, _P, _P,
                                                        ctypes.c_int, _P, _P, f32, f32, _P, _P,
                                                        _P, _P, _P, _P, _P, _P, sz, _P]),
            "llep_int8_row_bytes": (i32, [i32]),
            "llep_quantize_rows": (ctypes.c_int, [i64, i32, ctypes.c_int, _P, _P, i32, _P, _P]),
            "llep_packed_int8_bytes": (sz, [i32, i32, i32]),
            "llep_pack_int8": (ctypes.c_int, [i32, i32, i32, _P, _P, _P, _P]),
            "llep_int8_matmul_workspace_bytes": (sz, [i64, i32, i32]),
            "llep_int8_matmul": (ctypes.c_int, [i64, i32, i32, _P, i32, _P, _P, _P, ctypes.c_int,
                                                _P, _P, sz, _P]),
            "llep_grouped_ffn_int8_workspace_bytes": (sz, [pp, i32]),
            "llep_grouped_ffn_int8": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, _P, _P, _P, _P, _P,
                                                     i32, i32, _P, _P, sz, _P]),
            "llep_grouped_ffn_int8_f32": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, _P, _P, _P, _P,
                                                         _P, i32, i32, _P, _P, sz, _P]),
            "llep_combine_to_bf16": (ctypes.c_int, [pp, _P, _P, _P, i32, _P, _P]),
            "llep_route": (ctypes.c_int, [pr, ctypes.c_int, _P, _P, _P, _P, _P]),
            "llep_route_backward": (ctypes.c_int, [pr, ctypes.c_int, _P, _P, _P, _P, _P, _P]),
            "llep_mxfp4_row_bytes": (i32, [i32]),
            "llep_mxfp4_scale_bytes": (i32, [i32]),
            "llep_quantize_rows_mxfp4": (ctypes.c_int, [i64, i32, ctypes.c_int, _P, _P, i32, _P,
                                                        i32, _P]),
            "llep_dequantize_rows_mxfp4": (ctypes.c_int, [i64, i32, ctypes.c_int, _P, i32, _P,
                                                          i32, _P, _P]),
            "llep_packed_mxfp4_bytes": (sz, [i32, i32, i32]),
            "llep_pack_mxfp4": (ctypes.c_int, [i32, i32, i32, _P, _P, _P, _P, i32, i32, _P, _P]),
            "llep_mxfp4_matmul": (ctypes.c_int, [i64, i32, i32, _P, i32, _P, i32, _P,
                                                 ctypes.c_int, _P, _P]),
            "llep_grouped_ffn_mxfp4_workspace_bytes": (sz, [pp, i32]),
            "llep_grouped_ffn_mxfp4": (ctypes.c_int, [pp, pb, i32, _P, _P, _P, i32, i32,
                                                      ctypes.c_int, _P, _P, sz, _P]),
            "llep_clip_gradients_workspace_bytes": (sz, []),
            "llep_gradient_norm": (ctypes.c_int, [i32, pg, _P, _P, sz, _P]),
            "llep_clip_gradients": (ctypes.c_int, [i32, pg, f32, _P, _P, sz, _P]),
            "llep_last_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sigs.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def last_error() -> str:
    return lib().llep_last_error().decode()


def _check(rc: int, where: str):
    if rc != LLEP_OK:
        raise LLEPError(rc, where, last_error())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream=None) -> int:
    import torch
    if stream is not None:
        return stream.cuda_stream
    # torch.cuda.current_stream().cuda_stream without the Stream object (3 us less)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _empty(shape, dtype, device, stream=None):
    """torch.empty for a call on `stream` (None: the current one). The memory is that stream's, as
    the current stream's could still be in use by what is enqueued there, and is not given away,
    once freed, before the current stream is done with it too."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream())
    return t


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return LLEP_BF16
    if t.dtype == torch.float32:
        return LLEP_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def make_params(T: int, K: int, E: int, P: int, capacity: int, min_chunk: int = 1,
                lam: float = 0.0, mode: str = "llep") -> llep_plan_params:
    return llep_plan_params(T=T, K=K, E=E, P=P, min_chunk=min_chunk, capacity=capacity,
                            lam=lam, mode=LLEP_MODE_EP if mode == "ep" else LLEP_MODE_LLEP,
                            reserved=0)


# ---- size queries ----------------------------------------------------------

def llep_plan_max_chunks(params: llep_plan_params) -> int:
    n = lib().llep_plan_max_chunks(ctypes.byref(params))
    if n < 0:
        raise LLEPError(LLEP_E_ARG, "llep_plan_max_chunks", last_error())
    return n


def llep_plan_rank_base_elems(params: llep_plan_params) -> int:
    n = lib().llep_plan_rank_base_elems(ctypes.byref(params))
    if n < 0:
        raise LLEPError(LLEP_E_ARG, "llep_plan_rank_base_elems", last_error())
    return n


def llep_grouped_ffn_workspace_bytes(params: llep_plan_params, F: int, dtype_code: int) -> int:
    return lib().llep_grouped_ffn_workspace_bytes(ctypes.byref(params), F, dtype_code)


def llep_grouped_ffn_backward_workspace_bytes(params: llep_plan_params, D: int, F: int,
                                              dtype_code: int) -> int:
    return lib().llep_grouped_ffn_backward_workspace_bytes(ctypes.byref(params), D, F,
                                                           dtype_code)


# ---- plan buffers (device tensors) --------------------------------------------

class PlanBuffers:
    """Device tensors for llep_plan's tables, sized from the params."""

    def __init__(self, params: llep_plan_params, device="cuda"):
        import torch
        C = llep_plan_max_chunks(params)
        E, P = params.E, params.P
        i32 = dict(dtype=torch.int32, device=device)
        self.loads = torch.zeros(E, **i32)
        self.chunks = torch.zeros(C, 4, **i32)
        self.chunk_row = torch.zeros(C, **i32)
        self.expert_chunk_begin = torch.zeros(E + 1, **i32)
        self.groups = torch.zeros(C, 4, **i32)
        self.group_begin = torch.zeros(P + 1, **i32)
        self.device_rows = torch.zeros(P, **i32)
        self.xfers = torch.zeros(C, 3, **i32)
        self.rank_base = torch.zeros(max(1, llep_plan_rank_base_elems(params)), **i32)
        self.info = torch.zeros(8, **i32)
        self.struct = llep_plan_buffers(*[t.data_ptr() for t in (
            self.loads, self.chunks, self.chunk_row, self.expert_chunk_begin, self.groups,
            self.group_begin, self.device_rows, self.xfers, self.rank_base, self.info)])

    def info_dict(self) -> dict:
        v = self.info.cpu().tolist()
        return dict(zip(("status", "n_chunks", "n_groups", "n_xfers", "bypassed", "forced",
                         "max_device", "total_rows"), v))


# ---- the four steps and weight packing -----------------------------------------

def llep_plan(params: llep_plan_params, topk_ids, bufs: PlanBuffers, stream=None):
    _check(lib().llep_plan(ctypes.byref(params), _ptr(topk_ids), ctypes.byref(bufs.struct),
                           _stream(stream)), "llep_plan")


def llep_permute(params: llep_plan_params, bufs: PlanBuffers, topk_ids, topk_gates, x,
                 x_perm, gate_perm, row_pair, pair_row, stream=None):
    _check(lib().llep_permute(ctypes.byref(params), ctypes.byref(bufs.struct), _ptr(topk_ids),
                              _ptr(topk_gates), _ptr(x), x.shape[-1], _dtype_code(x),
                              _ptr(x_perm), _ptr(gate_perm), _ptr(row_pair), _ptr(pair_row),
                              _stream(stream)), "llep_permute")


def llep_pack_weights(w_gate, w_up, w_down, stream=None, out=None):
    """Packed copies of the expert weights (see llep.h); returns (gate_up, down).
    `out` = (gate_up, down) packs into those (contiguous) tensors instead, e.g.
    slices of a larger packed set filled a few experts at a time."""
    E, D, F = w_gate.shape
    code = _dtype_code(w_gate)
    if out is None:
        gu = _empty((E, 2 * F, D), w_gate.dtype, w_gate.device, stream)
        dn = _empty((E, D, F), w_gate.dtype, w_gate.device, stream)
    else:
        gu, dn = out
        if (gu.numel() != E * 2 * F * D or dn.numel() != E * D * F or not gu.is_contiguous()
                or not dn.is_contiguous() or gu.dtype != w_gate.dtype or dn.dtype != w_gate.dtype):
            raise ValueError("out tensors do not match the weights")
    _check(lib().llep_pack_weights(E, D, F, code, _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                   _ptr(gu), _ptr(dn), _stream(stream)), "llep_pack_weights")
    return gu, dn


def llep_grouped_ffn(params: llep_plan_params, bufs: PlanBuffers, device: int, x_perm,
                     w_gate_up, w_down, out_perm, workspace, stream=None):
    D = x_perm.shape[-1]
    F = w_down.shape[-1]
    _check(lib().llep_grouped_ffn(ctypes.byref(params), ctypes.byref(bufs.struct), device,
                                  _ptr(x_perm), _ptr(w_gate_up), _ptr(w_down), D, F,
                                  _dtype_code(x_perm), _ptr(out_perm), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(),
                                  _stream(stream)), "llep_grouped_ffn")


def llep_grouped_ffn_train(params: llep_plan_params, bufs: PlanBuffers, device: int, x_perm,
                           w_gate_up, w_down, out_perm, gate_up, workspace, stream=None):
    """llep_grouped_ffn that also keeps g and u ([T*K, 2F], interleaved per
    32 columns) for llep_grouped_ffn_backward."""
    D = x_perm.shape[-1]
    F = w_down.shape[-1]
    _check(lib().llep_grouped_ffn_train(ctypes.byref(params), ctypes.byref(bufs.struct), device,
                                        _ptr(x_perm), _ptr(w_gate_up), _ptr(w_down), D, F,
                                        _dtype_code(x_perm), _ptr(out_perm), _ptr(gate_up),
                                        _ptr(workspace),
                                        workspace.numel() * workspace.element_size(),
                                        _stream(stream)), "llep_grouped_ffn_train")


def llep_grouped_ffn_noalloc(params: llep_plan_params, bufs: PlanBuffers, device: int, x_perm,
                             w_gate_up, w_down, out_perm, stream=None):
    """llep_grouped_ffn with the library's own workspace array (no caller
    workspace; at most LLEP_NOALLOC_SCRATCH_BYTES)."""
    D = x_perm.shape[-1]
    F = w_down.shape[-1]
    _check(lib().llep_grouped_ffn_noalloc(ctypes.byref(params), ctypes.byref(bufs.struct),
                                          device, _ptr(x_perm), _ptr(w_gate_up), _ptr(w_down),
                                          D, F, _dtype_code(x_perm), _ptr(out_perm),
                                          _stream(stream)), "llep_grouped_ffn_noalloc")


def llep_combine(params: llep_plan_params, out_perm, pair_row, topk_gates, y, stream=None):
    _check(lib().llep_combine(ctypes.byref(params), _ptr(out_perm), _ptr(pair_row),
                              _ptr(topk_gates), out_perm.shape[-1], _dtype_code(out_perm),
                              _ptr(y), _stream(stream)), "llep_combine")


# ---- backward ------------------------------------------------------------------

def llep_combine_backward(params: llep_plan_params, out_perm, pair_row, topk_gates, dy,
                          d_out_perm, d_gates, stream=None):
    _check(lib().llep_combine_backward(ctypes.byref(params), _ptr(out_perm), _ptr(pair_row),
                                       _ptr(topk_gates), _ptr(dy), dy.shape[-1],
                                       _dtype_code(dy), _ptr(d_out_perm), _ptr(d_gates),
                                       _stream(stream)), "llep_combine_backward")


def llep_pack_weights_backward(w_gate, w_up, w_down, stream=None):
    """Packed weights of the backward GEMMs (see llep.h); returns
    (gate_up_t, down_t)."""
    E, D, F = w_gate.shape
    gut = _empty((E, D, 2 * F), w_gate.dtype, w_gate.device, stream)
    dnt = _empty((E, F, D), w_gate.dtype, w_gate.device, stream)
    _check(lib().llep_pack_weights_backward(E, D, F, _dtype_code(w_gate), _ptr(w_gate),
                                            _ptr(w_up), _ptr(w_down), _ptr(gut), _ptr(dnt),
                                            _stream(stream)), "llep_pack_weights_backward")
    return gut, dnt


def llep_grouped_ffn_backward(params: llep_plan_params, bufs: PlanBuffers, device: int, x_perm,
                              d_out_perm, w_gate_up, w_gate_up_t, w_down_t, dx_perm, dw_gate,
                              dw_up, dw_down, workspace, stream=None, gate_up=None):
    """gate_up: the llep_grouped_ffn_train output (None: recompute g and u)."""
    D = x_perm.shape[-1]
    F = w_down_t.shape[-2]
    _check(lib().llep_grouped_ffn_backward(
        ctypes.byref(params), ctypes.byref(bufs.struct), device, _ptr(x_perm), _ptr(d_out_perm),
        _ptr(w_gate_up), _ptr(w_gate_up_t), _ptr(w_down_t), _ptr(gate_up), D, F,
        _dtype_code(x_perm),
        _ptr(dx_perm), _ptr(dw_gate), _ptr(dw_up), _ptr(dw_down), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)),
        "llep_grouped_ffn_backward")


def llep_zero_absent_gradients(params: llep_plan_params, bufs: PlanBuffers, device: int, dw_gate,
                               dw_up, dw_down, stream=None):
    """Zeros for the experts that llep_grouped_ffn_backward leaves unwritten."""
    D, F = dw_gate.shape[-2:]
    _check(lib().llep_zero_absent_gradients(
        ctypes.byref(params), ctypes.byref(bufs.struct), device, D, F, _ptr(dw_gate),
        _ptr(dw_up), _ptr(dw_down), _stream(stream)), "llep_zero_absent_gradients")


# ---- around the block ------------------------------------------------------------

def _dense(what: str, t, shape, dtype):
    """t, if it is a dense GPU tensor of this shape and type (or None)."""
    if t is None or (t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.is_cuda):
        return t
    if t.dtype != dtype:
        raise TypeError(f"{what} is {t.dtype}, not {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{what} is not contiguous")
    if not t.is_cuda:
        raise ValueError(f"{what} is not on a GPU")
    return t


def _all_dense(shape, dtype, tensors) -> bool:
    """Whether _dense takes all of them (one pass over a call's tensors: a call for one token takes
    the GPU 4 us)."""
    for t in tensors:
        if t is not None and not (t.dtype is dtype and t.shape == shape and t.is_contiguous()
                                  and t.is_cuda):
            return False
    return True


def _list(what: str, t, n: int, dtype):
    """t, if it is a dense GPU tensor of this type with at least n elements along its only axis."""
    if t is None:
        raise ValueError(f"{what} is None")
    _dense(what, t, t.shape, dtype)
    if t.dim() != 1 or t.shape[0] < n:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, not [{n}] or longer")
    return t


def _pairs(what: str, t, params: llep_plan_params, dtype):
    """t, if it is a dense GPU tensor of this type with a value for every token-expert pair:
    [T, K], or one after another."""
    if t is None:
        raise ValueError(f"{what} is None")
    flat = t.dim() == 1
    return _dense(what, t, (params.T * params.K,) if flat else (params.T, params.K), dtype)


def _workspace(ws):
    """Pointer and bytes of a dense GPU tensor used as a workspace (or None)."""
    if ws is None:
        return None, 0
    if not ws.is_contiguous() or not ws.is_cuda:
        raise ValueError("the workspace is not a contiguous GPU tensor")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _gate_shape(gate, T: int, D: int, shape) -> int:
    """LLEP_GATE_* of a gate of shape [1, D] or [D], [T, 1], or [T, D] (or None); `shape`, where
    given, has to fit it."""
    if gate is None:
        if shape is not None and shape != LLEP_GATE_NONE and T > 0:
            raise ValueError("gate_shape without a gate")
        return LLEP_GATE_NONE
    if shape is not None:
        fits = {LLEP_GATE_CHANNEL: ((1, D), (D,)), LLEP_GATE_TOKEN: ((T, 1),),
                LLEP_GATE_FULL: ((T, D),)}.get(shape, ())
        if tuple(gate.shape) not in fits:
            raise ValueError(f"gate of shape {tuple(gate.shape)} does not fit gate_shape {shape}")
        return shape
    if gate.shape == (1, D) or gate.shape == (D,):
        return LLEP_GATE_CHANNEL
    if gate.shape == (T, 1):
        return LLEP_GATE_TOKEN
    if gate.shape == (T, D):
        return LLEP_GATE_FULL
    raise ValueError(f"gate of shape {tuple(gate.shape)} fits no rows of [{T}, {D}]")


def llep_block_norm(x, b, gate, w_post, w_pre, alpha: float, eps: float, r, h=None, h_q=None,
                    h_scale=None, stream=None, gate_shape=None):
    """r = x + alpha * gate * norm(b) * w_post, h = norm(r) * w_pre (see llep.h). x, b, r, h
    [T, D]; gate None, [1, D], [T, 1] or [T, D] (gate_shape: LLEP_GATE_*, where the shape alone
    leaves it open); h_q [T, bytes] int8 with h_scale [T]: h as 8-bit rows. Any of b, gate,
    w_post, w_pre, and outputs, may be None."""
    T, D = size = x.shape
    dt = x.dtype
    code = _dtype_code(x)
    shape = _gate_shape(gate, T, D, gate_shape)
    if not _all_dense(size, dt, (x, b, r, h)):
        for what, t in (("x", x), ("b", b), ("r", r), ("h", h)):
            _dense(what, t, (T, D), dt)
    if not _all_dense((D,), dt, (w_post, w_pre)):
        for what, t in (("w_post", w_post), ("w_pre", w_pre)):
            _dense(what, t, (D,), dt)
    if gate is not None:
        _dense("gate", gate, gate.shape, dt)
    q_bytes = 0
    if h_q is not None:
        import torch
        q_bytes = h_q.shape[-1]
        _dense("h_q", h_q, (T, q_bytes), torch.int8)
        _dense("h_scale", h_scale, (T,), torch.float32)
    _check(lib().llep_block_norm(T, D, code, _ptr(x), _ptr(b), _ptr(gate), shape, _ptr(w_post),
                                 _ptr(w_pre), alpha, eps, _ptr(r), _ptr(h), _ptr(h_q),
                                 _ptr(h_scale), q_bytes, _stream(stream)), "llep_block_norm")


def llep_block_norm_backward_workspace_bytes(T: int, D: int) -> int:
    return lib().llep_block_norm_backward_workspace_bytes(T, D)


def llep_block_norm_backward(r, b, gate, w_post, w_pre, alpha: float, eps: float, d_r, d_h, dx,
                             db, d_gate, dw_post, dw_pre, workspace, stream=None,
                             gate_shape=None):
    """Every gradient of llep_block_norm (see llep.h): dx, db in x's type; d_gate (the gate's
    shape), dw_post, dw_pre float32; None for inputs that the forward had not."""
    import torch
    T, D = size = d_r.shape
    dt = d_r.dtype
    code = _dtype_code(d_r)
    shape = _gate_shape(gate, T, D, gate_shape)
    if not _all_dense(size, dt, (r, b, d_r, d_h, dx, db)):
        for what, t in (("r", r), ("b", b), ("d_r", d_r), ("d_h", d_h), ("dx", dx), ("db", db)):
            _dense(what, t, (T, D), dt)
    if not _all_dense((D,), dt, (w_post, w_pre)):
        for what, t in (("w_post", w_post), ("w_pre", w_pre)):
            _dense(what, t, (D,), dt)
    if not _all_dense((D,), torch.float32, (dw_post, dw_pre)):
        for what, t in (("dw_post", dw_post), ("dw_pre", dw_pre)):
            _dense(what, t, (D,), torch.float32)
    if gate is not None:
        _dense("gate", gate, gate.shape, dt)
        _dense("d_gate", d_gate, gate.shape, torch.float32)
    _check(lib().llep_block_norm_backward(
        T, D, code, _ptr(r), _ptr(b), _ptr(gate), shape, _ptr(w_post), _ptr(w_pre), alpha, eps,
        _ptr(d_r), _ptr(d_h), _ptr(dx), _ptr(db), _ptr(d_gate), _ptr(dw_post), _ptr(dw_pre),
        *_workspace(workspace), _stream(stream)), "llep_block_norm_backward")


def llep_clip_gradients_workspace_bytes() -> int:
    return lib().llep_clip_gradients_workspace_bytes()


def _gradients(grads, out):
    """The llep_gradient array of dense bf16 / float32 tensors (in whole-list steps: a model has
    hundreds of them)."""
    import array
    import torch
    T = torch.Tensor
    if len(out) != len(grads):
        raise ValueError("as many outputs as gradients")
    n = len(grads)
    sizes = list(map(T.numel, grads))
    types = list(map(_DTYPE_OF, grads))
    codes = list(map({torch.float32: LLEP_F32, torch.bfloat16: LLEP_BF16}.get, types))
    both = (grads,) if out is grads else (grads, out)
    if (None in codes or not all(all(map(T.is_contiguous, ts)) and all(map(_IS_CUDA, ts))
                                 for ts in both)
            or (out is not grads and (not all(map(T.is_same_size, out, grads))
                                      or list(map(_DTYPE_OF, out)) != types))):
        for i, (g, o) in enumerate(zip(grads, out)):
            _dtype_code(g)
            _dense(f"gradient {i}", g, g.shape, g.dtype)
            _dense(f"output {i}", o, g.shape, g.dtype)
        raise ValueError("gradients and outputs do not match")
    words = [0] * (4 * max(n, 1))  # a llep_gradient is four 8-byte words
    words[0:4 * n:4] = map(T.data_ptr, grads)
    words[1:4 * n:4] = map(T.data_ptr, out)
    words[2:4 * n:4] = sizes
    words[3:4 * n:4] = codes
    return (llep_gradient * max(n, 1)).from_buffer(array.array("q", words))


def llep_gradient_norm(grads, norm, workspace, stream=None):
    """norm [1] float32 = the 2-norm over all elements of the tensors."""
    import torch
    _dense("norm", norm, (1,), torch.float32)
    _check(lib().llep_gradient_norm(len(grads), _gradients(grads, grads), _ptr(norm),
                                    *_workspace(workspace), _stream(stream)),
           "llep_gradient_norm")


def llep_clip_gradients(grads, max_norm: float, norm, workspace, out=None, stream=None):
    """llep_gradient_norm, then every gradient times min(1, max_norm / norm), in place or into
    `out` (tensors of the same shapes and types)."""
    import torch
    _dense("norm", norm, (1,), torch.float32)
    _check(lib().llep_clip_gradients(len(grads), _gradients(grads, grads if out is None else out),
                                     max_norm, _ptr(norm), *_workspace(workspace),
                                     _stream(stream)), "llep_clip_gradients")


# ---- 8-bit products ----------------------------------------------------------------

def llep_int8_row_bytes(D: int) -> int:
    """Bytes of an 8-bit row of D values."""
    n = lib().llep_int8_row_bytes(D)
    if n < 0:
        raise LLEPError(LLEP_E_ARG, "llep_int8_row_bytes", "D outside [1, LLEP_MAX_FFN_DIM]")
    return n


def llep_quantize_rows(x, q, scale, stream=None):
    """x [R, D] to 8 bits by row: q [R, bytes] int8 (bytes a multiple of 64, at least D; zeros
    past D) and scale [R] float32."""
    import torch
    R, D = x.shape
    code = _dtype_code(x)
    _dense("x", x, (R, D), x.dtype)
    _dense("q", q, (R, q.shape[-1]), torch.int8)
    _dense("scale", scale, (R,), torch.float32)
    _check(lib().llep_quantize_rows(R, D, code, _ptr(x), _ptr(q), q.shape[-1], _ptr(scale),
                                    _stream(stream)), "llep_quantize_rows")


def llep_pack_matrix_int8(w, w_up=None, stream=None):
    """Packed copy of 8-bit weights [N, K] or [E, N, K], rows = output channels; with w_up (the
    same shape) of gate and up rows together (see llep.h). Returns an int8 tensor [E, bytes]."""
    import torch
    if w.dim() not in (2, 3):
        raise ValueError("weights are [N, K] or [E, N, K]")
    E, N, K = (1, *w.shape) if w.dim() == 2 else w.shape
    _dense("w", w, w.shape, torch.int8)
    _dense("w_up", w_up, w.shape, torch.int8)
    nbytes = lib().llep_packed_int8_bytes(E, N, K) * (1 if w_up is None else 2)
    if nbytes == 0:
        raise LLEPError(LLEP_E_ARG, "llep_pack_matrix_int8", "E, N or K outside its range")
    out = _empty((E, nbytes // E), torch.int8, w.device, stream)
    _check(lib().llep_pack_int8(E, N, K, _ptr(w), _ptr(w_up), _ptr(out), _stream(stream)),
           "llep_pack_int8")
    return out


def llep_int8_matmul_workspace_bytes(M: int, N: int, K: int) -> int:
    return lib().llep_int8_matmul_workspace_bytes(M, N, K)


def llep_int8_matmul(x, x_scale, w_packed, w_scale, out, K: int, workspace=None, stream=None):
    """out [M, N] (bf16 or float32) = x_scale w_scale (x w^T): x [M, bytes] int8 rows of K values
    (llep_quantize_rows), w_packed from llep_pack_matrix_int8, x_scale [M], w_scale [N]."""
    import torch
    M, N = out.shape
    code = _dtype_code(out)
    _dense("x", x, (M, x.shape[-1]), torch.int8)
    _dense("x_scale", x_scale, (M,), torch.float32)
    _dense("w_packed", w_packed, (1, lib().llep_packed_int8_bytes(1, N, K)), torch.int8)
    _dense("w_scale", w_scale, (N,), torch.float32)
    _dense("out", out, (M, N), out.dtype)
    _check(lib().llep_int8_matmul(M, N, K, _ptr(x), x.shape[-1], _ptr(x_scale), _ptr(w_packed),
                                  _ptr(w_scale), code, _ptr(out), *_workspace(workspace),
                                  _stream(stream)), "llep_int8_matmul")


def llep_grouped_ffn_int8_workspace_bytes(params: llep_plan_params, F: int) -> int:
    return lib().llep_grouped_ffn_int8_workspace_bytes(ctypes.byref(params), F)


def llep_grouped_ffn_int8(params: llep_plan_params, bufs: PlanBuffers, device: int, x_perm,
                          x_scale, row_pair, w_gate_up, gate_scale, up_scale, w_down, down_scale,
                          out_perm, workspace, stream=None):
    """The grouped FFN on 8-bit rows and weights (see llep.h): x_perm [T*K, D] int8, x_scale [T]
    with row_pair [T*K] int32, or [T*K] with row_pair None; weights from llep_pack_matrix_int8,
    scales [E, F], [E, F] and [E, D]; out_perm [T*K, D] bf16, or float32
    (llep_grouped_ffn_int8_f32)."""
    import torch
    R = params.T * params.K
    D, F, E = x_perm.shape[-1], gate_scale.shape[-1], params.E
    if x_perm.shape[0] < R or out_perm.shape[0] < R:
        raise ValueError("x_perm and out_perm need T * K rows")
    _dense("x_perm", x_perm, (x_perm.shape[0], D), torch.int8)
    _list("x_scale", x_scale, R if row_pair is None else params.T, torch.float32)
    if row_pair is not None:
        _list("row_pair", row_pair, R, torch.int32)
    for what, t, n in (("gate_scale", gate_scale, F), ("up_scale", up_scale, F),
                       ("down_scale", down_scale, D)):
        _dense(what, t, (E, n), torch.float32)
    _dense("w_gate_up", w_gate_up, (E, 2 * F * D), torch.int8)
    _dense("w_down", w_down, (E, D * F), torch.int8)
    wide = out_perm.dtype is torch.float32
    _dense("out_perm", out_perm, (out_perm.shape[0], D), torch.float32 if wide else torch.bfloat16)
    name = "llep_grouped_ffn_int8_f32" if wide else "llep_grouped_ffn_int8"
    _check(getattr(lib(), name)(
        ctypes.byref(params), ctypes.byref(bufs.struct), device, _ptr(x_perm), _ptr(x_scale),
        _ptr(row_pair), _ptr(w_gate_up), _ptr(gate_scale), _ptr(up_scale), _ptr(w_down),
        _ptr(down_scale), D, F, _ptr(out_perm), *_workspace(workspace), _stream(stream)), name)


def llep_combine_to_bf16(params: llep_plan_params, out_perm, pair_row, topk_gates, y, stream=None):
    """llep_combine of float32 rows out_perm [T*K, D] into y [T, D] bf16: pair_row [T*K] int32,
    topk_gates [T, K] float32 (or None: the pairs' sum)."""
    import torch
    D = out_perm.shape[-1]
    _dense("out_perm", out_perm, (out_perm.shape[0], D), torch.float32)
    _dense("y", y, (params.T, D), torch.bfloat16)
    _list("pair_row", pair_row, params.T * params.K, torch.int32)
    if topk_gates is not None:
        _pairs("topk_gates", topk_gates, params, torch.float32)
    if out_perm.shape[0] < params.T * params.K:
        raise ValueError("out_perm needs T * K rows")
    _check(lib().llep_combine_to_bf16(ctypes.byref(params), _ptr(out_perm), _ptr(pair_row),
                                      _ptr(topk_gates), D, _ptr(y), _stream(stream)),
           "llep_combine_to_bf16")


# ---- routing -----------------------------------------------------------------------

def _here(*tensors):
    """Refuses tensors of another device than the current one, whose stream a call goes to."""
    import torch
    current = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != current:
            raise ValueError(f"a tensor is on {t.device}, the current device is {current}")


_torch = None  # the module, once a call below has needed it (an import statement is 0.2 us)


def _type_code(t):
    """_dtype_code(t), and torch."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    dtype = t.dtype
    return (LLEP_BF16 if dtype is _torch.bfloat16 else
            LLEP_F32 if dtype is _torch.float32 else _dtype_code(t)), _torch


def _arguments(stream, *specs):
    """The call's stream, if all of the specs (what, tensor or None, shape, dtype) are dense tensors
    on the current device; refuses others as _dense and _here do. In one pass: a call for one token
    takes the GPU 3 to 6 us."""
    dev = specs[0][1].get_device()
    for _, t, shape, dtype in specs:
        if t is not None and (t.get_device() != dev or t.dtype is not dtype or t.shape != shape
                              or not t.is_contiguous()):
            break
    else:
        if dev >= 0 and _torch._C._cuda_getDevice() == dev:
            if stream is not None:
                return stream.cuda_stream
            return _torch._C._cuda_getCurrentRawStream(dev)
    for what, t, shape, dtype in specs:
        _dense(what, t, shape, dtype)
    _here(*(t for _, t, _, _ in specs))
    return _stream(stream)


def make_route(T: int, K: int, E: int, score: str = "softmax", groups: int = 1,
               top_groups: int = 1, group_score: str = "max", renormalize: bool = True,
               scale: float = 1.0) -> llep_route_params:
    """Parameters of llep_route (see llep.h). score: "softmax" or "sigmoid"; group_score: "max" or
    "top2"."""
    scores = {"softmax": LLEP_SCORE_SOFTMAX, "sigmoid": LLEP_SCORE_SIGMOID}
    kinds = {"max": LLEP_GROUP_MAX, "top2": LLEP_GROUP_TOP2}
    if score not in scores:
        raise ValueError(f"score is {score!r}, not 'softmax' or 'sigmoid'")
    if group_score not in kinds:
        raise ValueError(f"group_score is {group_score!r}, not 'max' or 'top2'")
    return llep_route_params(T=T, K=K, E=E, score=scores[score], groups=groups,
                             top_groups=top_groups, group_score=kinds[group_score],
                             renormalize=int(bool(renormalize)), scale=scale)


def llep_route(params: llep_route_params, logits, bias, ids, gates, stream=None):
    """Router logits [T, E] (bf16 or float32) to ids [T, K] int32 and gates [T, K] float32 (see
    llep.h); bias [E] float32 or None."""
    T, K, E = params.T, params.K, params.E
    code, torch = _type_code(logits)
    at = _arguments(stream, ("logits", logits, (T, E), logits.dtype),
                    ("bias", bias, (E,), torch.float32), ("ids", ids, (T, K), torch.int32),
                    ("gates", gates, (T, K), torch.float32))
    rc = lib().llep_route(ctypes.byref(params), code, logits.data_ptr(), _ptr(bias),
                          ids.data_ptr(), gates.data_ptr(), at)
    if rc:
        _check(rc, "llep_route")


def llep_route_backward(params: llep_route_params, logits, ids, gates, d_gates, d_logits,
                        stream=None):
    """d_logits [T, E] (bf16 or float32) from d_gates [T, K] float32 and llep_route's inputs and
    outputs; logits (of d_logits' type) may be None for the renormalized softmax."""
    T, K, E = params.T, params.K, params.E
    code, torch = _type_code(d_logits)
    at = _arguments(stream, ("d_logits", d_logits, (T, E), d_logits.dtype),
                    ("logits", logits, (T, E), d_logits.dtype), ("ids", ids, (T, K), torch.int32),
                    ("gates", gates, (T, K), torch.float32),
                    ("d_gates", d_gates, (T, K), torch.float32))
    rc = lib().llep_route_backward(ctypes.byref(params), code, _ptr(logits), ids.data_ptr(),
                                   gates.data_ptr(), d_gates.data_ptr(), d_logits.data_ptr(), at)
    if rc:
        _check(rc, "llep_route_backward")


# ---- 4-bit rows and products ---------------------------------------------------------

def llep_mxfp4_row_bytes(D: int) -> int:
    """Bytes of the values of a 4-bit row of D values."""
    n = lib().llep_mxfp4_row_bytes(D)
    if n < 0:
        raise LLEPError(LLEP_E_ARG, "llep_mxfp4_row_bytes", "D outside [1, LLEP_MAX_FFN_DIM]")
    return n


def llep_mxfp4_scale_bytes(D: int) -> int:
    """Bytes of the exponents of a 4-bit row of D values."""
    n = lib().llep_mxfp4_scale_bytes(D)
    if n < 0:
        raise LLEPError(LLEP_E_ARG, "llep_mxfp4_scale_bytes", "D outside [1, LLEP_MAX_FFN_DIM]")
    return n


def _mxfp4_bytes(D: int):
    """(llep_mxfp4_row_bytes(D), llep_mxfp4_scale_bytes(D))"""
    slices = (D + 127) >> 7
    if 1 <= D <= LLEP_MAX_FFN_DIM:
        return slices * 64, (slices + 3 >> 2) * 16
    return llep_mxfp4_row_bytes(D), llep_mxfp4_scale_bytes(D)


def _byte_rows(what: str, t, R: int, least: int, dev: int) -> int:
    """The bytes from one row of t to the next: t [R, >= least] uint8 on GPU dev, whose rows may be
    parts of longer ones (a view of a buffer's columns)."""
    if t.dtype is not _torch.uint8:
        raise TypeError(f"{what} is {t.dtype}, not {_torch.uint8}")
    shape = t.shape
    if len(shape) != 2 or shape[0] != R or shape[1] < least:
        raise ValueError(f"{what} has shape {tuple(shape)}, not [{R}, {least}] or wider")
    if t.get_device() != dev:
        raise ValueError(f"{what} is on {t.device}, not on GPU {dev}")
    pitch, step = t.stride()
    if step != 1 or (R > 1 and pitch < shape[1]):
        raise ValueError(f"{what} is not made of rows of bytes")
    if R <= 1:  # the stride of an only row means nothing
        return least
    if pitch >= 1 << 31:
        raise ValueError(f"{what} has rows {pitch} bytes apart, 2^31 or more")
    return pitch


def llep_quantize_rows_mxfp4(x, q, scale, stream=None):
    """x [R, D] (bf16 or float32) to 4-bit rows: q [R, llep_mxfp4_row_bytes(D)] and scale [R,
    llep_mxfp4_scale_bytes(D)] uint8 (rows a multiple of 16 bytes apart, at most
    LLEP_MAX_FFN_DIM)."""
    R, D = x.shape
    code, _ = _type_code(x)
    at = _arguments(stream, ("x", x, (R, D), x.dtype))
    q_bytes, s_bytes = _mxfp4_bytes(D)
    dev = x.get_device()
    q_pitch, s_pitch = _byte_rows("q", q, R, q_bytes, dev), _byte_rows("scale", scale, R, s_bytes, dev)
    rc = lib().llep_quantize_rows_mxfp4(R, D, code, x.data_ptr(), q.data_ptr(), q_pitch,
                                        scale.data_ptr(), s_pitch, at)
    if rc:
        _check(rc, "llep_quantize_rows_mxfp4")


def llep_dequantize_rows_mxfp4(q, scale, out, stream=None):
    """out [R, D] (bf16 or float32) = what the 4-bit rows q, scale stand for."""
    R, D = out.shape
    code, _ = _type_code(out)
    at = _arguments(stream, ("out", out, (R, D), out.dtype))
    q_bytes, s_bytes = _mxfp4_bytes(D)
    dev = out.get_device()
    q_pitch, s_pitch = _byte_rows("q", q, R, q_bytes, dev), _byte_rows("scale", scale, R, s_bytes, dev)
    rc = lib().llep_dequantize_rows_mxfp4(R, D, code, q.data_ptr(), q_pitch, scale.data_ptr(),
                                          s_pitch, out.data_ptr(), at)
    if rc:
        _check(rc, "llep_dequantize_rows_mxfp4")


def llep_pack_matrix_mxfp4(w, scale, w_up=None, up_scale=None, K: int = None, stream=None):
    """Packed copy of 4-bit weights: w [N, bytes] or [E, N, bytes] uint8 (two values a byte), rows
    = output channels, with exponents scale [.., N, blocks] uint8; with w_up and up_scale (the same
    shapes) of gate and up rows together. K: values of a row (2 * bytes, where it is not given).
    Returns a uint8 tensor [E, bytes]."""
    import torch
    if w.dim() not in (2, 3):
        raise ValueError("weights are [N, bytes] or [E, N, bytes]")
    E, N, w_bytes = (1, *w.shape) if w.dim() == 2 else w.shape
    if K is None:
        K = 2 * w_bytes
    if max(E, N, w_bytes, scale.shape[-1], K) >= 1 << 31:
        raise ValueError("weights have 2^31 or more matrices, rows, or bytes or values of a row")
    if w_bytes < (K + 1) // 2 or scale.shape[-1] < (K + 31) // 32:
        raise ValueError(f"rows of {w_bytes} bytes and {scale.shape[-1]} exponents hold no {K} values")
    _dense("w", w, w.shape, torch.uint8)
    _dense("scale", scale, (*w.shape[:-1], scale.shape[-1]), torch.uint8)
    if (w_up is None) != (up_scale is None):
        raise ValueError("w_up and up_scale: both or none")
    _dense("w_up", w_up, w.shape, torch.uint8)
    _dense("up_scale", up_scale, scale.shape, torch.uint8)
    _here(w, scale, w_up, up_scale)
    nbytes = lib().llep_packed_mxfp4_bytes(E, N if w_up is None else 2 * N, K)
    if nbytes == 0:
        raise LLEPError(LLEP_E_ARG, "llep_pack_matrix_mxfp4", "E, N or K outside its range")
    out = _empty((E, nbytes // E), torch.uint8, w.device, stream)
    _check(lib().llep_pack_mxfp4(E, N, K, _ptr(w), _ptr(scale), _ptr(w_up), _ptr(up_scale),
                                 w_bytes, scale.shape[-1], _ptr(out), _stream(stream)),
           "llep_pack_mxfp4")
    return out


def llep_mxfp4_matmul(x, x_scale, w_packed, out, K: int, stream=None):
    """out [M, N] (bf16 or float32) = x w^T: x, x_scale 4-bit rows of K values
    (llep_quantize_rows_mxfp4), w_packed one matrix of llep_pack_matrix_mxfp4."""
    M, N = out.shape
    code, torch = _type_code(out)
    q_bytes, s_bytes = _mxfp4_bytes(K)
    at = _arguments(stream, ("out", out, (M, N), out.dtype),
                    ("w_packed", w_packed, (1, (N + 15) // 16 * 16 * (q_bytes + s_bytes)),
                     torch.uint8))
    dev = out.get_device()
    q_pitch = _byte_rows("x", x, M, q_bytes, dev)
    s_pitch = _byte_rows("x_scale", x_scale, M, s_bytes, dev)
    rc = lib().llep_mxfp4_matmul(M, N, K, x.data_ptr(), q_pitch, x_scale.data_ptr(), s_pitch,
                                 w_packed.data_ptr(), code, out.data_ptr(), at)
    if rc:
        _check(rc, "llep_mxfp4_matmul")


def llep_grouped_ffn_mxfp4_workspace_bytes(params: llep_plan_params, F: int) -> int:
    return lib().llep_grouped_ffn_mxfp4_workspace_bytes(ctypes.byref(params), F)


def llep_grouped_ffn_mxfp4(params: llep_plan_params, bufs: PlanBuffers, device: int, x_perm,
                           w_gate_up, w_down, D: int, F: int, out_perm, workspace, stream=None):
    """The grouped FFN on 4-bit rows and weights (see llep.h): x_perm [T*K, bytes] uint8, values
    and then exponents of each row (llep_mxfp4_row_bytes(D) + llep_mxfp4_scale_bytes(D) bytes);
    weights from llep_pack_matrix_mxfp4; out_perm [T*K, D] bf16 or float32."""
    import torch
    R, E = params.T * params.K, params.E
    if x_perm.shape[0] < R or out_perm.shape[0] < R:
        raise ValueError("x_perm and out_perm need T * K rows")
    code = _dtype_code(out_perm)
    _dense("x_perm", x_perm,
           (x_perm.shape[0], llep_mxfp4_row_bytes(D) + llep_mxfp4_scale_bytes(D)), torch.uint8)
    L = lib()
    for what, t, n, k in (("w_gate_up", w_gate_up, 2 * F, D), ("w_down", w_down, D, F)):
        _dense(what, t, (E, L.llep_packed_mxfp4_bytes(1, n, k)), torch.uint8)
    _dense("out_perm", out_perm, (out_perm.shape[0], D), out_perm.dtype)
    _here(x_perm, w_gate_up, w_down, out_perm, workspace)
    _check(L.llep_grouped_ffn_mxfp4(
        ctypes.byref(params), ctypes.byref(bufs.struct), device, _ptr(x_perm), _ptr(w_gate_up),
        _ptr(w_down), D, F, code, _ptr(out_perm), *_workspace(workspace), _stream(stream)),
        "llep_grouped_ffn_mxfp4")
