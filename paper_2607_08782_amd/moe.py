"""Thin Python binding of libmoe.so (the C ABI in include/moe.h).

Argument marshalling only: every function checks that tensors live on the
GPU with the expected dtype and layout, allocates missing outputs with torch
(device memory is all torch is used for), and calls the C entry point of the
same name on torch's current HIP stream.  All arithmetic runs in the HIP
kernels.  If the library is not built this module raises; there is no
fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe.so")

MOE_F32, MOE_BF16 = 0, 1
MOE_OK, MOE_ERR_ARG, MOE_ERR_PLACEMENT, MOE_ERR_SHAPE, MOE_ERR_DEVICE = 0, 1, 2, 3, 4
MOE_RENORM, MOE_LOGITS_IN = 1, 2
MOE_FFN_GATE_UP, MOE_FFN_DOWN, MOE_FFN_SMALL_GROUPS, MOE_FFN_LARGE_GROUPS = 1, 2, 4, 8
MOE_MAX_E, MOE_MAX_K, MOE_MAX_G, MOE_MAX_GROUPS = 256, 16, 64, 128
MOE_PERMUTE_NOALLOC_MAX_WS = 4 << 20

EXPORTS = ("moe_status_string", "moe_route_topk", "moe_route_topk_ws_bytes",
           "moe_expert_histogram", "moe_permute_ws_bytes",
           "moe_permute", "moe_permute_noalloc", "moe_route_package", "moe_grouped_ffn_ws_bytes", "moe_grouped_ffn",
           "moe_grouped_ffn_products", "moe_grouped_ffn_combine",
           "moe_grouped_ffn_rows", "moe_grouped_ffn_rows_products", "moe_grouped_ffn_rows_shared",
           "moe_combine", "moe_combine_shared",
           "moe_quantize_e4m3", "moe_route_topk_e4m3",
           "moe_quantize_mxfp4", "moe_dequantize_mxfp4", "moe_mxfp4_lay_out",
           "moe_grouped_ffn_mxfp4_ws_bytes", "moe_grouped_ffn_mxfp4",
           "moe_combine_backward", "moe_permute_backward", "moe_route_topk_backward_ws_bytes",
           "moe_route_topk_backward", "moe_route_topk_backward_aux",
           "moe_quantize_int8", "moe_dequantize_int8",
           "moe_grouped_ffn_int8_ws_bytes", "moe_grouped_ffn_int8",
           "moe_rmsnorm", "moe_rmsnorm_backward_ws_bytes", "moe_rmsnorm_backward",
           "moe_balance_loss_ws_bytes", "moe_balance_loss", "moe_balance_loss_backward",
           "moe_grad_norm_ws_bytes", "moe_grad_norm", "moe_clip_grads")

_lib = None


class MoeError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (fn, status_string(status), status))


def load_library(path: str = LIB_PATH):
    """Load libmoe.so and declare every exported signature."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("libmoe.so is not built (%s); run __graft_entry__.build()" % path)
    lib = ctypes.CDLL(path)
    P, I, L, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    lib.moe_status_string.argtypes = [I]
    lib.moe_status_string.restype = ctypes.c_char_p
    lib.moe_route_topk.argtypes = [P, I, P, P, L, I, I, I, I, P, P, P, P, S, P]
    lib.moe_route_topk.restype = I
    lib.moe_route_topk_ws_bytes.argtypes = [I, L, I, I, I]
    lib.moe_route_topk_ws_bytes.restype = S
    lib.moe_expert_histogram.argtypes = [P, L, I, I, P, P, P]
    lib.moe_expert_histogram.restype = I
    lib.moe_permute_ws_bytes.argtypes = [L, I, I]
    lib.moe_permute_ws_bytes.restype = S
    lib.moe_permute.argtypes = [P, I, P, P, P, L, I, I, I, P, I, I, I, P, L, P, P, P, P, P, P, S, P]
    lib.moe_permute.restype = I
    lib.moe_permute_noalloc.argtypes = [P, I, P, P, P, L, I, I, I, P, I, I, I, P, L, P, P, P, P, P,
                                        P]
    lib.moe_permute_noalloc.restype = I
    lib.moe_route_package.argtypes = [P, I, P, P, L, I, I, I, I, P, P, P, P, S, P, P, P, I, I, I, P,
                                      L, P, P, P, P, P, P, S, P]
    lib.moe_route_package.restype = I
    lib.moe_grouped_ffn_ws_bytes.argtypes = [I, L, I, I, I]
    lib.moe_grouped_ffn_ws_bytes.restype = S
    lib.moe_grouped_ffn.argtypes = [P, I, P, I, P, P, I, I, L, P, P, S, P]
    lib.moe_grouped_ffn.restype = I
    lib.moe_grouped_ffn_products.argtypes = [P, I, P, I, P, P, I, I, L, P, P, S, I, P]
    lib.moe_grouped_ffn_products.restype = I
    lib.moe_grouped_ffn_combine.argtypes = [P, I, P, I, P, P, I, I, L, P, P, P, L, I, P, P, S, P]
    lib.moe_grouped_ffn_combine.restype = I
    lib.moe_grouped_ffn_rows.argtypes = [P, L, P, I, P, I, P, P, I, I, L, P, P, S, P]
    lib.moe_grouped_ffn_rows.restype = I
    lib.moe_grouped_ffn_rows_products.argtypes = [P, L, P, I, P, I, P, P, I, I, L, P, P, S, I, P]
    lib.moe_grouped_ffn_rows_products.restype = I
    lib.moe_grouped_ffn_rows_shared.argtypes = [P, L, P, I, P, I, I, P, P, I, I, L, P, P, S, I, P]
    lib.moe_grouped_ffn_rows_shared.restype = I
    lib.moe_combine.argtypes = [P, I, P, P, P, L, I, I, P, P]
    lib.moe_combine.restype = I
    lib.moe_combine_shared.argtypes = [P, I, P, P, P, I, L, I, I, P, P]
    lib.moe_combine_shared.restype = I
    lib.moe_quantize_e4m3.argtypes = [P, I, L, I, P, P, P]
    lib.moe_quantize_e4m3.restype = I
    lib.moe_route_topk_e4m3.argtypes = [P, P, P, P, P, L, I, I, I, I, P, P, P, P]
    lib.moe_route_topk_e4m3.restype = I
    lib.moe_quantize_mxfp4.argtypes = [P, I, L, I, P, P, P]
    lib.moe_quantize_mxfp4.restype = I
    lib.moe_dequantize_mxfp4.argtypes = [P, P, L, I, I, P, P]
    lib.moe_dequantize_mxfp4.restype = I
    lib.moe_mxfp4_lay_out.argtypes = [P, P, L, I, P, P, P]
    lib.moe_mxfp4_lay_out.restype = I
    lib.moe_grouped_ffn_mxfp4_ws_bytes.argtypes = [L, L, I, I, I]
    lib.moe_grouped_ffn_mxfp4_ws_bytes.restype = S
    lib.moe_grouped_ffn_mxfp4.argtypes = [P, L, P, P, I, I, P, P, P, P, I, I, L, P, P, S, P]
    lib.moe_grouped_ffn_mxfp4.restype = I
    lib.moe_combine_backward.argtypes = [P, P, I, P, P, L, I, I, P, P, P]
    lib.moe_combine_backward.restype = I
    lib.moe_permute_backward.argtypes = [P, I, P, P, L, I, I, P, P]
    lib.moe_permute_backward.restype = I
    lib.moe_route_topk_backward_ws_bytes.argtypes = [I, L, I, I, I, I]
    lib.moe_route_topk_backward_ws_bytes.restype = S
    lib.moe_route_topk_backward.argtypes = [P, P, P, P, P, P, I, L, I, I, I, I, P, P, P, P, P, S, P]
    lib.moe_route_topk_backward.restype = I
    lib.moe_route_topk_backward_aux.argtypes = [P, P, P, P, P, P, P, I, L, I, I, I, I, P, P, P, P, P, S, P]
    lib.moe_route_topk_backward_aux.restype = I
    F = ctypes.c_float
    lib.moe_quantize_int8.argtypes = [P, I, L, I, P, P, P]
    lib.moe_quantize_int8.restype = I
    lib.moe_dequantize_int8.argtypes = [P, P, L, I, I, P, P]
    lib.moe_dequantize_int8.restype = I
    lib.moe_grouped_ffn_int8_ws_bytes.argtypes = [L, I, I, I]
    lib.moe_grouped_ffn_int8_ws_bytes.restype = S
    lib.moe_grouped_ffn_int8.argtypes = [P, P, L, P, P, I, I, P, P, P, P, I, I, L, P, P, S, P]
    lib.moe_grouped_ffn_int8.restype = I
    lib.moe_rmsnorm.argtypes = [P, P, I, P, F, L, I, P, P, P, P, P, P]
    lib.moe_rmsnorm.restype = I
    lib.moe_rmsnorm_backward_ws_bytes.argtypes = [I, L, I]
    lib.moe_rmsnorm_backward_ws_bytes.restype = S
    lib.moe_rmsnorm_backward.argtypes = [P, P, I, P, P, P, L, I, P, P, P, S, P]
    lib.moe_rmsnorm_backward.restype = I
    lib.moe_balance_loss_ws_bytes.argtypes = [L, I]
    lib.moe_balance_loss_ws_bytes.restype = S
    lib.moe_balance_loss.argtypes = [P, P, P, L, I, I, P, P, P, P, P, S, P]
    lib.moe_balance_loss.restype = I
    lib.moe_balance_loss_backward.argtypes = [P, P, P, P, L, I, I, F, P, P]
    lib.moe_balance_loss_backward.restype = I
    lib.moe_grad_norm_ws_bytes.argtypes = [P, I]
    lib.moe_grad_norm_ws_bytes.restype = S
    lib.moe_grad_norm.argtypes = [P, P, P, I, P, P, S, P]
    lib.moe_grad_norm.restype = I
    lib.moe_clip_grads.argtypes = [P, P, P, I, P, F, P, P]
    lib.moe_clip_grads.restype = I
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().moe_status_string(int(status)).decode()


def _check(fn: str, status: int):
    if status != MOE_OK:
        raise MoeError(fn, status)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return MOE_BF16
    if t.dtype == torch.float32:
        return MOE_F32
    raise TypeError("unsupported element type %s (float32 or bfloat16)" % t.dtype)


def _dev(t: Optional[torch.Tensor], name: str, dtype=None):
    """Device pointer of a contiguous GPU tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return t.data_ptr()


def _holds(t: Optional[torch.Tensor], name: str, *shape: int):
    """t (None passes) holds at least the elements of this shape."""
    want = 1
    for n in shape:
        want *= n
    if t is not None and t.numel() < want:
        raise ValueError("%s must hold %s elements, got %s" % (name, tuple(shape), tuple(t.shape)))


# the current stream's handle without the Stream object around it, which takes longer to
# make (2.7 us) than the rest of a short call's marshalling
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _of(stream, make):
    """`make`, which allocates a tensor, for a call on this stream: in that stream's memory, so
    that nothing queued on another stream still uses it, and what the call drops is used again
    only behind the call."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))

    def on_stream(*args, **kw):
        with torch.cuda.stream(stream):
            return make(*args, **kw)
    return on_stream


def _empty(shape, dtype, device, stream=None):
    make = torch.empty if stream is None else _of(stream, torch.empty)
    return make(shape, dtype=dtype, device=device)


def moe_route_topk(x: Optional[torch.Tensor], w_router: Optional[torch.Tensor],
                   bias: Optional[torch.Tensor], k: int, *, E: Optional[int] = None,
                   renorm: bool = True, logits: Optional[torch.Tensor] = None,
                   logits_in: bool = False, want_logits: bool = True,
                   topk_idx: Optional[torch.Tensor] = None,
                   topk_gate: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                   stream=None):
    """Gate scores + top-k.  Returns (logits or None, topk_idx, topk_gate)."""
    lib = load_library()
    if logits_in:
        if logits is None:
            raise ValueError("logits_in needs logits")
        T, E_ = logits.shape
        d = 0 if x is None else x.shape[1]
        dtype = MOE_F32 if x is None else _dtype_code(x)
        device = logits.device
    else:
        T, d = x.shape
        E_ = w_router.shape[0]
        dtype = _dtype_code(x)
        if w_router.dtype != x.dtype or w_router.shape[1] != d:
            raise ValueError("w_router must be [E, d] of x's dtype")
        device = x.device
        if logits is None and want_logits:
            logits = _empty((T, E_), torch.float32, device, stream)
    if E is not None and E != E_:
        raise ValueError("E mismatch")
    if topk_idx is None:
        topk_idx = _empty((T, k), torch.int32, device, stream)
    if topk_gate is None:
        topk_gate = _empty((T, k), torch.float32, device, stream)
    flags = (MOE_RENORM if renorm else 0) | (MOE_LOGITS_IN if logits_in else 0)
    need = moe_route_topk_ws_bytes(dtype, T, d, E_, flags)
    if need and ws is None:
        ws = workspace(need, device, stream)
    st = lib.moe_route_topk(_dev(x, "x"), dtype, _dev(w_router, "w_router"),
                            _dev(bias, "bias", torch.float32), T, d, E_, k, flags,
                            _dev(logits, "logits", torch.float32),
                            _dev(topk_idx, "topk_idx", torch.int32),
                            _dev(topk_gate, "topk_gate", torch.float32), _dev(ws, "ws"),
                            0 if ws is None else ws.numel(), _stream(stream))
    _check("moe_route_topk", st)
    return logits, topk_idx, topk_gate


def moe_quantize_e4m3(x: torch.Tensor, *, q: Optional[torch.Tensor] = None,
                      scales: Optional[torch.Tensor] = None, stream=None):
    """Per-row E4M3 codes (uint8 [rows, cols]) and fp32 scales ([rows]) of x."""
    lib = load_library()
    rows, cols = x.shape
    if q is None:
        q = _empty((rows, cols), torch.uint8, x.device, stream)
    if scales is None:
        scales = _empty((rows,), torch.float32, x.device, stream)
    st = lib.moe_quantize_e4m3(_dev(x, "x"), _dtype_code(x), rows, cols, _dev(q, "q", torch.uint8),
                               _dev(scales, "scales", torch.float32), _stream(stream))
    _check("moe_quantize_e4m3", st)
    return q, scales


def moe_route_topk_e4m3(xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor,
                        w_scale: torch.Tensor, bias: Optional[torch.Tensor], k: int, *,
                        renorm: bool = True, logits: Optional[torch.Tensor] = None,
                        topk_idx: Optional[torch.Tensor] = None,
                        topk_gate: Optional[torch.Tensor] = None, stream=None):
    """Quantized-predictor scores + top-k.  Returns (logits, topk_idx, topk_gate)."""
    lib = load_library()
    T, d = xq.shape
    E = wq.shape[0]
    if wq.shape[1] != d:
        raise ValueError("wq must be [E, d]")
    if logits is None:
        logits = _empty((T, E), torch.float32, xq.device, stream)
    if topk_idx is None:
        topk_idx = _empty((T, k), torch.int32, xq.device, stream)
    if topk_gate is None:
        topk_gate = _empty((T, k), torch.float32, xq.device, stream)
    st = lib.moe_route_topk_e4m3(_dev(xq, "xq", torch.uint8), _dev(x_scale, "x_scale", torch.float32),
                                 _dev(wq, "wq", torch.uint8), _dev(w_scale, "w_scale", torch.float32),
                                 _dev(bias, "bias", torch.float32), T, d, E, k,
                                 MOE_RENORM if renorm else 0,
                                 _dev(logits, "logits", torch.float32),
                                 _dev(topk_idx, "topk_idx", torch.int32),
                                 _dev(topk_gate, "topk_gate", torch.float32), _stream(stream))
    _check("moe_route_topk_e4m3", st)
    return logits, topk_idx, topk_gate


def moe_route_topk_ws_bytes(dtype: int, T: int, d: int, E: int, flags: int) -> int:
    return int(load_library().moe_route_topk_ws_bytes(dtype, T, d, E, flags))


def moe_expert_histogram(topk_idx: torch.Tensor, E: int, *, counts: Optional[torch.Tensor] = None,
                         coact: Optional[torch.Tensor] = None, want_coact: bool = False,
                         stream=None):
    """Per-expert counts (and co-activation).  Returns (counts, coact or None)."""
    lib = load_library()
    T, k = topk_idx.shape
    if counts is None:
        counts = _empty((E,), torch.int32, topk_idx.device, stream)
    if coact is None and want_coact:
        coact = _empty((E, E), torch.int32, topk_idx.device, stream)
    st = lib.moe_expert_histogram(_dev(topk_idx, "topk_idx", torch.int32), T, k, E,
                                  _dev(counts, "counts", torch.int32),
                                  _dev(coact, "coact", torch.int32), _stream(stream))
    _check("moe_expert_histogram", st)
    return counts, coact


def moe_permute_ws_bytes(T: int, k: int, E: int) -> int:
    return int(load_library().moe_permute_ws_bytes(T, k, E))


def moe_grouped_ffn_ws_bytes(dtype: int, cap_rows: int, d: int, f: int, n_groups: int) -> int:
    return int(load_library().moe_grouped_ffn_ws_bytes(dtype, cap_rows, d, f, n_groups))


def workspace(nbytes: int, device, stream=None) -> torch.Tensor:
    """A 256-byte aligned device workspace (torch's caching allocator aligns to 512 B) for calls
    on this stream (None: the current one)."""
    make = torch.empty if stream is None else _of(stream, torch.empty)
    ws = make(max(int(nbytes), 256), dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws


def moe_permute(x: torch.Tensor, topk_idx: torch.Tensor, topk_gate: torch.Tensor,
                counts: torch.Tensor, placement: np.ndarray, dev: int, *, E: int,
                cap_rows: Optional[int] = None, c_max: int = 0, out: Optional[dict] = None,
                ws: Optional[torch.Tensor] = None, want_send_counts: bool = True,
                copy_rows: bool = True, stream=None, noalloc: bool = False):
    """Package tokens for the experts on GPU `dev`.  Returns a dict of device tensors
    (x_perm, group_offsets, row_token, row_gate, token_row, send_counts).  With
    copy_rows=False only the row maps are produced (x_perm is not written; for
    moe_grouped_ffn_rows).  noalloc=True calls moe_permute_noalloc (no workspace:
    the library's own scratch); outputs missing from `out` are still allocated here."""
    lib = load_library()
    T, d = x.shape
    k = topk_idx.shape[1]
    placement = np.ascontiguousarray(placement, dtype=np.uint8)
    if placement.ndim != 2 or placement.shape[0] != E:
        raise ValueError("placement must be a [E, G] array")
    G = placement.shape[1]
    n_local = int((placement[:, dev] != 0).sum()) if 0 <= dev < G else 0
    if cap_rows is None:
        cap_rows = T * min(k, n_local)
    device = x.device
    o = {} if out is None else out
    if "group_offsets" not in o:
        if copy_rows:
            o["x_perm"] = _empty((max(cap_rows, 1), d), x.dtype, device, stream)
        o["group_offsets"] = _empty((n_local + 1,), torch.int32, device, stream)
        o["row_token"] = _empty((max(cap_rows, 1),), torch.int32, device, stream)
        o["row_gate"] = _empty((max(cap_rows, 1),), torch.float32, device, stream)
        o["token_row"] = _empty((T, k), torch.int32, device, stream)
        o["send_counts"] = _empty((G,), torch.int32, device, stream) if want_send_counts else None
    args = [_dev(x, "x") if copy_rows else None, _dtype_code(x),
            _dev(topk_idx, "topk_idx", torch.int32), _dev(topk_gate, "topk_gate", torch.float32),
            _dev(counts, "counts", torch.int32), T, d if copy_rows else 0, k, E,
            placement.ctypes.data_as(ctypes.c_void_p), G, dev, c_max,
            _dev(o["x_perm"], "x_perm", x.dtype) if copy_rows else None, cap_rows,
            _dev(o["group_offsets"], "group_offsets", torch.int32),
            _dev(o["row_token"], "row_token", torch.int32),
            _dev(o["row_gate"], "row_gate", torch.float32),
            _dev(o["token_row"], "token_row", torch.int32),
            _dev(o.get("send_counts"), "send_counts", torch.int32)]
    if noalloc:
        _check("moe_permute_noalloc", lib.moe_permute_noalloc(*args, _stream(stream)))
        return o
    if ws is None:
        ws = workspace(moe_permute_ws_bytes(T, k, E), device, stream)
    _check("moe_permute", lib.moe_permute(*args, _dev(ws, "ws"), ws.numel(), _stream(stream)))
    return o


def moe_route_package(x: torch.Tensor, w_router: Optional[torch.Tensor],
                      bias: Optional[torch.Tensor], placement: np.ndarray, dev: int, *,
                      logits: Optional[torch.Tensor], topk_idx: torch.Tensor,
                      topk_gate: torch.Tensor, ws_route: Optional[torch.Tensor],
                      counts: torch.Tensor, coact: Optional[torch.Tensor], out: dict,
                      ws_perm: torch.Tensor, cap_rows: int, renorm: bool = True,
                      logits_in: bool = False, copy_rows: bool = True, c_max: int = 0, stream=None):
    """moe_route_topk, moe_expert_histogram and moe_permute of one batch in one call,
    into the caller's buffers (`out` as moe_permute's; copy_rows=False: row maps only).
    Every buffer's size is checked: the kernels write T, k, E and cap_rows entries."""
    lib = load_library()
    T, d = x.shape
    k = topk_idx.shape[1]
    E = counts.numel()
    dtype = _dtype_code(x)
    if not logits_in and (w_router is None or w_router.dtype != x.dtype
                          or tuple(w_router.shape) != (E, d)):
        raise ValueError("w_router must be [E, d] of x's dtype")
    if logits_in and (logits is None or tuple(logits.shape) != (T, E)):
        raise ValueError("logits_in needs logits [T, E]")
    placement = np.ascontiguousarray(placement, dtype=np.uint8)
    if placement.ndim != 2 or placement.shape[0] != E:
        raise ValueError("placement must be a [E, G] array")
    G = placement.shape[1]
    n_local = int(np.count_nonzero(placement[:, dev])) if 0 <= dev < G else 0
    _holds(bias, "bias", E)
    _holds(logits, "logits", T, E)
    _holds(topk_idx, "topk_idx", T, k)
    _holds(topk_gate, "topk_gate", T, k)
    _holds(coact, "coact", E, E)
    _holds(out["token_row"], "token_row", T, k)
    _holds(out["group_offsets"], "group_offsets", n_local + 1)
    _holds(out["row_token"], "row_token", cap_rows)
    _holds(out["row_gate"], "row_gate", cap_rows)
    _holds(out.get("send_counts"), "send_counts", G)
    if copy_rows:
        _holds(out["x_perm"], "x_perm", cap_rows, d)
    flags = (MOE_RENORM if renorm else 0) | (MOE_LOGITS_IN if logits_in else 0)
    st = lib.moe_route_package(
        _dev(x, "x"), dtype, None if logits_in else _dev(w_router, "w_router"),
        _dev(bias, "bias", torch.float32), T, d, E, k, flags, _dev(logits, "logits", torch.float32),
        _dev(topk_idx, "topk_idx", torch.int32), _dev(topk_gate, "topk_gate", torch.float32),
        _dev(ws_route, "ws_route"), 0 if ws_route is None else ws_route.numel(),
        _dev(counts, "counts", torch.int32), _dev(coact, "coact", torch.int32),
        placement.ctypes.data_as(ctypes.c_void_p), G, dev, c_max,
        _dev(out["x_perm"], "x_perm", x.dtype) if copy_rows else None, cap_rows,
        _dev(out["group_offsets"], "group_offsets", torch.int32),
        _dev(out["row_token"], "row_token", torch.int32),
        _dev(out["row_gate"], "row_gate", torch.float32),
        _dev(out["token_row"], "token_row", torch.int32),
        _dev(out.get("send_counts"), "send_counts", torch.int32), _dev(ws_perm, "ws_perm"),
        ws_perm.numel(), _stream(stream))
    _check("moe_route_package", st)


class WeightTable:
    """Host arrays of per-slot device pointers, as moe_grouped_ffn takes them."""

    def __init__(self, w13: Sequence[torch.Tensor], w2: Sequence[torch.Tensor]):
        if len(w13) != len(w2) or not len(w13):
            raise ValueError("need one (w13, w2) pair per group")
        self.w13 = list(w13)
        self.w2 = list(w2)
        self.f = w13[0].shape[0] // 2
        self.d = w13[0].shape[1]
        self.dtype = w13[0].dtype
        for a, b in zip(self.w13, self.w2):
            _dev(a, "w13", self.dtype)
            _dev(b, "w2", self.dtype)
            if tuple(a.shape) != (2 * self.f, self.d) or tuple(b.shape) != (self.d, self.f):
                raise ValueError("w13 must be [2f, d] and w2 [d, f] for every group")
        n = len(self.w13)
        self.p13 = (ctypes.c_void_p * n)(*[a.data_ptr() for a in self.w13])
        self.p2 = (ctypes.c_void_p * n)(*[b.data_ptr() for b in self.w2])

    def __len__(self):
        return len(self.w13)


def moe_grouped_ffn(x_perm: torch.Tensor, group_offsets: torch.Tensor, weights: WeightTable, *,
                    cap_rows: Optional[int] = None, y_perm: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, stream=None,
                    products: int = 3) -> torch.Tensor:
    """SwiGLU FFN of every group.  Returns y_perm [cap_rows, d].  products=1 or 2
    runs one product (moe_grouped_ffn_products: gate/up into the workspace, or down
    from it; the down call must follow a gate/up call with the same ws)."""
    lib = load_library()
    if cap_rows is None:
        cap_rows = x_perm.shape[0]
    d, f = weights.d, weights.f
    dtype = _dtype_code(x_perm)
    if x_perm.dtype != weights.dtype or x_perm.shape[1] != d:
        raise ValueError("x_perm must be [rows, d] of the weights' dtype")
    if group_offsets.numel() != len(weights) + 1:
        raise ValueError("group_offsets must hold n_groups + 1 entries")
    if y_perm is None:
        y_perm = _empty((max(cap_rows, 1), d), x_perm.dtype, x_perm.device, stream)
    if ws is None:
        ws = workspace(moe_grouped_ffn_ws_bytes(dtype, cap_rows, d, f, len(weights)), x_perm.device, stream)
    args = [_dev(x_perm, "x_perm"), dtype, _dev(group_offsets, "group_offsets", torch.int32),
            len(weights), ctypes.cast(weights.p13, ctypes.c_void_p),
            ctypes.cast(weights.p2, ctypes.c_void_p), d, f, cap_rows,
            _dev(y_perm, "y_perm", x_perm.dtype), _dev(ws, "ws"), ws.numel()]
    if products == MOE_FFN_GATE_UP | MOE_FFN_DOWN:
        _check("moe_grouped_ffn", lib.moe_grouped_ffn(*args, _stream(stream)))
    else:
        _check("moe_grouped_ffn_products",
               lib.moe_grouped_ffn_products(*args, products, _stream(stream)))
    return y_perm


def moe_grouped_ffn_combine(x_perm: torch.Tensor, group_offsets: torch.Tensor,
                            weights: WeightTable, token_row: torch.Tensor, topk_gate: torch.Tensor,
                            y_shared: Optional[torch.Tensor], *, cap_rows: int, T: int,
                            y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """Grouped FFN and weighted combine in one call (every group at most 256 rows).
    Returns y [T, d]."""
    lib = load_library()
    d, f = weights.d, weights.f
    dtype = _dtype_code(x_perm)
    if x_perm.dtype != weights.dtype or x_perm.shape[1] != d:
        raise ValueError("x_perm must be [rows, d] of the weights' dtype")
    k = token_row.shape[1]
    if y is None:
        y = _empty((max(T, 1), d), x_perm.dtype, x_perm.device, stream)
    if ws is None:
        ws = workspace(moe_grouped_ffn_ws_bytes(dtype, cap_rows, d, f, len(weights)), x_perm.device, stream)
    st = lib.moe_grouped_ffn_combine(
        _dev(x_perm, "x_perm"), dtype, _dev(group_offsets, "group_offsets", torch.int32),
        len(weights), ctypes.cast(weights.p13, ctypes.c_void_p),
        ctypes.cast(weights.p2, ctypes.c_void_p), d, f, cap_rows,
        _dev(token_row, "token_row", torch.int32), _dev(topk_gate, "topk_gate", torch.float32),
        _dev(y_shared, "y_shared", x_perm.dtype), T, k, _dev(y, "y", x_perm.dtype),
        _dev(ws, "ws"), ws.numel(), _stream(stream))
    _check("moe_grouped_ffn_combine", st)
    return y


def moe_grouped_ffn_rows(x: torch.Tensor, row_token: torch.Tensor, group_offsets: torch.Tensor,
                         weights: WeightTable, *, cap_rows: int,
                         y_perm: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                         stream=None, products: int = 3) -> torch.Tensor:
    """moe_grouped_ffn reading row p from x[row_token[p]] (no x_perm).  Returns y_perm.
    products other than 3 (single products, hints) call moe_grouped_ffn_rows_products."""
    lib = load_library()
    T = x.shape[0]
    d, f = weights.d, weights.f
    dtype = _dtype_code(x)
    if x.dtype != weights.dtype or x.shape[1] != d:
        raise ValueError("x must be [T, d] of the weights' dtype")
    if group_offsets.numel() != len(weights) + 1:
        raise ValueError("group_offsets must hold n_groups + 1 entries")
    if y_perm is None:
        y_perm = _empty((max(cap_rows, 1), d), x.dtype, x.device, stream)
    if ws is None:
        ws = workspace(moe_grouped_ffn_ws_bytes(dtype, cap_rows, d, f, len(weights)), x.device, stream)
    args = [_dev(x, "x"), T, _dev(row_token, "row_token", torch.int32), dtype,
            _dev(group_offsets, "group_offsets", torch.int32), len(weights),
            ctypes.cast(weights.p13, ctypes.c_void_p), ctypes.cast(weights.p2, ctypes.c_void_p), d, f,
            cap_rows, _dev(y_perm, "y_perm", x.dtype), _dev(ws, "ws"), ws.numel()]
    if products == MOE_FFN_GATE_UP | MOE_FFN_DOWN:
        _check("moe_grouped_ffn_rows", lib.moe_grouped_ffn_rows(*args, _stream(stream)))
    else:
        _check("moe_grouped_ffn_rows_products",
               lib.moe_grouped_ffn_rows_products(*args, products, _stream(stream)))
    return y_perm


def moe_grouped_ffn_rows_shared(x: torch.Tensor, row_token: torch.Tensor,
                                group_offsets: torch.Tensor, weights: WeightTable, n_shared: int, *,
                                cap_rows: int, y_perm: Optional[torch.Tensor] = None,
                                ws: Optional[torch.Tensor] = None, stream=None,
                                products: int = 3) -> torch.Tensor:
    """moe_grouped_ffn_rows_products with n_shared leading groups of T rows each
    (the shared experts, weights[0 .. n_shared-1]); the routed groups follow, their
    rows counted from n_shared * T.  Returns y_perm [n_shared * T + cap_rows, d]."""
    lib = load_library()
    T = x.shape[0]
    d, f = weights.d, weights.f
    dtype = _dtype_code(x)
    if x.dtype != weights.dtype or x.shape[1] != d:
        raise ValueError("x must be [T, d] of the weights' dtype")
    n_groups = len(weights) - n_shared
    if n_shared < 0 or n_groups < 0 or group_offsets.numel() != n_groups + 1:
        raise ValueError("group_offsets must hold n_groups + 1 entries for the routed groups")
    rows = n_shared * T + cap_rows
    if row_token.numel() < rows:
        raise ValueError("row_token must hold n_shared * T + cap_rows entries")
    if y_perm is None:
        y_perm = _empty((max(rows, 1), d), x.dtype, x.device, stream)
    if ws is None:
        ws = workspace(moe_grouped_ffn_ws_bytes(dtype, rows, d, f, len(weights)), x.device, stream)
    st = lib.moe_grouped_ffn_rows_shared(
        _dev(x, "x"), T, _dev(row_token, "row_token", torch.int32), dtype,
        _dev(group_offsets, "group_offsets", torch.int32), n_groups, n_shared,
        ctypes.cast(weights.p13, ctypes.c_void_p), ctypes.cast(weights.p2, ctypes.c_void_p), d, f,
        cap_rows, _dev(y_perm, "y_perm", x.dtype), _dev(ws, "ws"), ws.numel(), products,
        _stream(stream))
    _check("moe_grouped_ffn_rows_shared", st)
    return y_perm


def moe_combine(y_perm: torch.Tensor, token_row: torch.Tensor, topk_gate: torch.Tensor,
                y_shared: Optional[torch.Tensor], *, T: int, d: int,
                y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gate-weighted sum back in token order (+ shared experts).  Returns y [T, d]."""
    lib = load_library()
    k = token_row.shape[1] if token_row.dim() == 2 else 1
    dtype = _dtype_code(y_perm)
    if y is None:
        y = _empty((T, d), y_perm.dtype, y_perm.device, stream)
    st = lib.moe_combine(_dev(y_perm, "y_perm", y.dtype), dtype,
                         _dev(token_row, "token_row", torch.int32),
                         _dev(topk_gate, "topk_gate", torch.float32),
                         _dev(y_shared, "y_shared", y.dtype), T, d, k,
                         _dev(y, "y", y.dtype), _stream(stream))
    _check("moe_combine", st)
    return y


def moe_combine_shared(y_perm: torch.Tensor, token_row: torch.Tensor, topk_gate: torch.Tensor,
                       y_shared: Optional[torch.Tensor], n_shared: int, *, T: int, d: int,
                       y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """moe_combine with the shared experts' output in n_shared [T, d] slices
    (y_shared [n_shared, T, d], added in slice order).  Returns y [T, d]."""
    lib = load_library()
    k = token_row.shape[1] if token_row.dim() == 2 else 1
    dtype = _dtype_code(y_perm)
    if y is None:
        y = _empty((T, d), y_perm.dtype, y_perm.device, stream)
    if y_shared is not None and n_shared > 0 and y_shared.numel() < n_shared * T * d:
        raise ValueError("y_shared must hold n_shared slices of [T, d]")
    st = lib.moe_combine_shared(_dev(y_perm, "y_perm", y.dtype), dtype,
                                _dev(token_row, "token_row", torch.int32),
                                _dev(topk_gate, "topk_gate", torch.float32),
                                _dev(y_shared, "y_shared", y.dtype), n_shared, T, d, k,
                                _dev(y, "y", y.dtype), _stream(stream))
    _check("moe_combine_shared", st)
    return y


def mxfp4_cols(cols: int) -> int:
    """Columns of an MXFP4 row: `cols` padded to a multiple of 128 (MOE_MXFP4_COLS)."""
    return (int(cols) + 127) // 128 * 128


def moe_quantize_mxfp4(x: torch.Tensor, *, q: Optional[torch.Tensor] = None,
                       scales: Optional[torch.Tensor] = None, stream=None):
    """x [rows, cols] as an MXFP4 matrix.  Returns (codes uint8 [rows, P / 2], scales uint8
    [rows, P / 32]), P = mxfp4_cols(cols)."""
    lib = load_library()
    rows, cols = x.shape
    P = mxfp4_cols(cols)
    if q is None:
        q = _empty((rows, P // 2), torch.uint8, x.device, stream)
    if scales is None:
        scales = _empty((rows, P // 32), torch.uint8, x.device, stream)
    _holds(q, "q", rows, P // 2)
    _holds(scales, "scales", rows, P // 32)
    st = lib.moe_quantize_mxfp4(_dev(x, "x"), _dtype_code(x), rows, cols, _dev(q, "q", torch.uint8),
                                _dev(scales, "scales", torch.uint8), _stream(stream))
    _check("moe_quantize_mxfp4", st)
    return q, scales


def moe_dequantize_mxfp4(q: torch.Tensor, scales: torch.Tensor, cols: int, *,
                         dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """The values [rows, cols] that an MXFP4 matrix holds, in `dtype` (float32 or bfloat16)."""
    lib = load_library()
    rows, P = q.shape[0], mxfp4_cols(cols)
    if cols < 1 or tuple(q.shape) != (rows, P // 2) or tuple(scales.shape) != (rows, P // 32):
        raise ValueError("an MXFP4 matrix of %d columns has codes [rows, %d] and scales [rows, %d]"
                         % (cols, P // 2, P // 32))
    if out is None:
        out = _empty((rows, cols), dtype, q.device, stream)
    _holds(out, "out", rows, cols)
    st = lib.moe_dequantize_mxfp4(_dev(q, "q", torch.uint8), _dev(scales, "scales", torch.uint8),
                                  rows, cols, _dtype_code(out), _dev(out, "out", dtype),
                                  _stream(stream))
    _check("moe_dequantize_mxfp4", st)
    return out


def moe_mxfp4_lay_out(q: torch.Tensor, scales: torch.Tensor, cols: int, *, stream=None):
    """An MXFP4 matrix (codes [rows, P / 2], scales [rows, P / 32]) as the FFN reads a
    weight's, step-major.  Returns (codes uint8 [P / 128, rows, 64], scales int32 [P / 128,
    rows] of four scale bytes each)."""
    lib = load_library()
    rows, P = q.shape[0], mxfp4_cols(cols)
    if cols < 1 or tuple(q.shape) != (rows, P // 2) or tuple(scales.shape) != (rows, P // 32):
        raise ValueError("an MXFP4 matrix of %d columns has codes [rows, %d] and scales [rows, %d]"
                         % (cols, P // 2, P // 32))
    steps = _empty((P // 128, rows, 64), torch.uint8, q.device, stream)
    words = _empty((P // 128, rows), torch.int32, q.device, stream)
    st = lib.moe_mxfp4_lay_out(_dev(q, "q", torch.uint8), _dev(scales, "scales", torch.uint8), rows, cols,
                               _dev(steps, "step_codes"), _dev(words, "step_scales"), _stream(stream))
    _check("moe_mxfp4_lay_out", st)
    return steps, words


class MxWeightTable:
    """Experts whose weights are MXFP4 matrices, as moe_grouped_ffn_mxfp4 takes them: w13 and
    w2 hold one (codes, scales) pair per group, as moe_quantize_mxfp4 gives them for [2f, d]
    and [d, f].  Keeps step-major copies (moe_mxfp4_lay_out), not what it was given."""

    def __init__(self, w13: Sequence, w2: Sequence, d: int, f: int):
        if len(w13) != len(w2) or not len(w13):
            raise ValueError("need one (w13, w2) pair per group")
        self.d, self.f = int(d), int(f)
        self.w13, self.s13 = self._lay_out(w13, 2 * self.f, self.d, "w13")
        self.w2, self.s2 = self._lay_out(w2, self.d, self.f, "w2")
        n = len(self.w13)
        self._arrays = [(ctypes.c_void_p * n)(*[t.data_ptr() for t in ts])
                        for ts in (self.w13, self.s13, self.w2, self.s2)]
        self.pointers = [ctypes.cast(a, ctypes.c_void_p) for a in self._arrays]

    @classmethod
    def quantized(cls, w13: Sequence[torch.Tensor], w2: Sequence[torch.Tensor]) -> "MxWeightTable":
        """The experts of a WeightTable (w13 [2f, d], w2 [d, f], bf16 or fp32), quantized."""
        if not len(w13):
            raise ValueError("need one (w13, w2) pair per group")
        return cls([moe_quantize_mxfp4(w) for w in w13], [moe_quantize_mxfp4(w) for w in w2],
                   w13[0].shape[1], w13[0].shape[0] // 2)

    @staticmethod
    def _lay_out(pairs, rows: int, cols: int, name: str):
        P = mxfp4_cols(cols)
        codes, words = [], []
        for q, s in pairs:
            if tuple(q.shape) != (rows, P // 2) or tuple(s.shape) != (rows, P // 32):
                raise ValueError("%s must be MXFP4 matrices of %d rows and %d columns" % (name, rows, cols))
            step_codes, step_scales = moe_mxfp4_lay_out(q, s, cols)
            codes.append(step_codes)
            words.append(step_scales)
        return codes, words

    def __len__(self):
        return len(self.w13)


def moe_grouped_ffn_mxfp4_ws_bytes(T: int, cap_rows: int, d: int, f: int, n_groups: int) -> int:
    return int(load_library().moe_grouped_ffn_mxfp4_ws_bytes(T, cap_rows, d, f, n_groups))


def moe_grouped_ffn_mxfp4(x: torch.Tensor, group_offsets: torch.Tensor, weights: MxWeightTable, *,
                          row_token: Optional[torch.Tensor] = None, n_shared: int = 0,
                          cap_rows: Optional[int] = None, y_perm: Optional[torch.Tensor] = None,
                          ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """SwiGLU FFN of every group with 4-bit weights and activations; x [T, d] bf16, read
    through row_token (as moe_grouped_ffn_rows_shared's, n_shared leading groups included)
    or, without it, the packaged rows.  Returns y_perm [n_shared * T + cap_rows, d]."""
    lib = load_library()
    T = x.shape[0]
    d, f = weights.d, weights.f
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.shape[1] != d:
        raise ValueError("x must be bfloat16 [rows, %d]" % d)
    if cap_rows is None:
        if row_token is not None:
            raise ValueError("row_token needs cap_rows")
        cap_rows = T
    n_groups = len(weights) - n_shared
    if n_shared < 0 or n_groups < 0 or group_offsets.numel() != n_groups + 1:
        raise ValueError("group_offsets must hold n_groups + 1 entries for the routed groups")
    rows = n_shared * T + cap_rows
    _holds(row_token, "row_token", rows)
    if y_perm is None:
        y_perm = _empty((max(rows, 1), d), x.dtype, x.device, stream)
    _holds(y_perm, "y_perm", rows, d)
    if ws is None:
        ws = workspace(moe_grouped_ffn_mxfp4_ws_bytes(T, rows, d, f, len(weights)), x.device, stream)
    st = lib.moe_grouped_ffn_mxfp4(
        _dev(x, "x"), T, _dev(row_token, "row_token", torch.int32),
        _dev(group_offsets, "group_offsets", torch.int32), n_groups, n_shared, *weights.pointers,
        d, f, cap_rows, _dev(y_perm, "y_perm", torch.bfloat16), _dev(ws, "ws"), ws.numel(),
        _stream(stream))
    _check("moe_grouped_ffn_mxfp4", st)
    return y_perm


def _same(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, *shape: int):
    """t (None passes) is of this type and shape."""
    if t is not None and (t.dtype != dtype or t.shape != shape):
        raise ValueError("%s must be %s %s, got %s %s" % (name, dtype, shape, t.dtype, tuple(t.shape)))


def moe_combine_backward(dy: torch.Tensor, y_perm: Optional[torch.Tensor], token_row: torch.Tensor,
                         topk_gate: Optional[torch.Tensor], *, dy_perm: Optional[torch.Tensor] = None,
                         dgate: Optional[torch.Tensor] = None, want_dy_perm: bool = True,
                         want_dgate: bool = True, stream=None):
    """Gradient of moe_combine.  Returns (dy_perm of y_perm's shape or None, dgate [T, k] or
    None); rows of dy_perm that token_row does not name are left as they were."""
    lib = load_library()
    T, d = dy.shape
    k = token_row.shape[1]
    if token_row.shape[0] != T:
        raise ValueError("token_row must be [T, k]")
    _same(topk_gate, "topk_gate", torch.float32, T, k)
    if y_perm is not None and (y_perm.dtype != dy.dtype or y_perm.dim() != 2 or y_perm.shape[1] != d):
        raise ValueError("y_perm must be [rows, d] of dy's dtype")
    # (quicker than by a shape)
    like = torch.empty_like if stream is None else _of(stream, torch.empty_like)
    if want_dy_perm and dy_perm is None:
        if y_perm is None:
            raise ValueError("dy_perm's rows are y_perm's: give one of them")
        dy_perm = like(y_perm)
    if want_dgate and dgate is None:
        dgate = _empty((T, k), torch.float32, dy.device, stream) if topk_gate is None else like(topk_gate)
    if dy_perm is not None and (dy_perm.dtype != dy.dtype or dy_perm.dim() != 2 or dy_perm.shape[1] != d):
        raise ValueError("dy_perm must be [rows, d] of dy's dtype")
    if dy_perm is not None and y_perm is not None and dy_perm.shape[0] < y_perm.shape[0]:
        raise ValueError("dy_perm must hold y_perm's rows")
    _same(dgate, "dgate", torch.float32, T, k)
    # no rows have no address: any stands for one that no token_row leads to
    at_rows = _dev(y_perm, "y_perm") or (None if y_perm is None else dy.data_ptr())
    st = lib.moe_combine_backward(_dev(dy, "dy"), at_rows, _dtype_code(dy),
                                  _dev(token_row, "token_row", torch.int32), _dev(topk_gate, "topk_gate"),
                                  T, d, k, _dev(dy_perm, "dy_perm"), _dev(dgate, "dgate"), _stream(stream))
    _check("moe_combine_backward", st)
    return dy_perm, dgate


def moe_permute_backward(dx_perm: torch.Tensor, token_row: torch.Tensor, *,
                         dx_add: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """Gradient of moe_permute's row copy, on top of dx_add.  Returns dx [T, d]."""
    lib = load_library()
    d = dx_perm.shape[1]
    T, k = token_row.shape
    if dx is None:
        like = torch.empty_like if stream is None else _of(stream, torch.empty_like)
        dx = _empty((T, d), dx_perm.dtype, dx_perm.device, stream) if dx_add is None else like(dx_add)
    _same(dx_add, "dx_add", dx_perm.dtype, T, d)
    _same(dx, "dx", dx_perm.dtype, T, d)
    at_rows = _dev(dx_perm, "dx_perm") or dx.data_ptr()  # (as moe_combine_backward)
    st = lib.moe_permute_backward(at_rows, _dtype_code(dx_perm),
                                  _dev(token_row, "token_row", torch.int32), _dev(dx_add, "dx_add"),
                                  T, d, k, _dev(dx, "dx"), _stream(stream))
    _check("moe_permute_backward", st)
    return dx


def moe_route_topk_backward_ws_bytes(dtype: int, T: int, d: int, E: int, k: int, flags: int) -> int:
    return int(load_library().moe_route_topk_backward_ws_bytes(dtype, T, d, E, k, flags))


def moe_route_topk_backward(dgate: torch.Tensor, topk_gate: torch.Tensor, topk_idx: torch.Tensor,
                            x: torch.Tensor, w_router: torch.Tensor, *,
                            logits: Optional[torch.Tensor] = None, renorm: bool = True,
                            want_dlogits: bool = True, want_dx: bool = True, want_dw: bool = True,
                            want_dbias: bool = True, dlogits: Optional[torch.Tensor] = None,
                            dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None,
                            dbias: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                            dlogits_add: Optional[torch.Tensor] = None, stream=None):
    """Gradient of moe_route_topk.  Returns (dlogits [T, E], dx [T, d] of x's dtype, dw [E, d],
    dbias [E]), float32 but dx, None for what is not wanted.  renorm=False needs logits.
    dlogits_add [T, E] (moe_route_topk_backward_aux): what reaches the scores another way."""
    lib = load_library()
    T, d = x.shape
    E, k = w_router.shape[0], topk_idx.shape[1]
    if w_router.dtype != x.dtype or w_router.shape[1] != d:
        raise ValueError("w_router must be [E, d] of x's dtype")
    if not renorm and logits is None:
        raise ValueError("gates without renormalisation need logits")
    f32 = torch.float32
    _same(dgate, "dgate", f32, T, k)
    _same(topk_gate, "topk_gate", f32, T, k)
    _same(topk_idx, "topk_idx", torch.int32, T, k)
    _same(logits, "logits", f32, T, E)
    like, new = torch.empty_like, dgate.new_empty
    if stream is not None:
        like, new = _of(stream, like), _of(stream, new)
    if want_dlogits and dlogits is None:
        dlogits = new(T, E)
    if want_dx and dx is None:
        dx = like(x)
    if want_dw and dw is None:
        dw = like(w_router, dtype=f32)
    if want_dbias and dbias is None:
        dbias = new(E)
    _same(dlogits, "dlogits", f32, T, E)
    _same(dx, "dx", x.dtype, T, d)
    _same(dw, "dw", f32, E, d)
    _same(dbias, "dbias", f32, E)
    dtype, flags = _dtype_code(x), MOE_RENORM if renorm else 0
    if ws is None:
        ws = workspace(moe_route_topk_backward_ws_bytes(dtype, T, d, E, k, flags), x.device, stream)
    _same(dlogits_add, "dlogits_add", f32, T, E)
    scores = (None if renorm else _dev(logits, "logits"),)
    if dlogits_add is not None:
        scores += (_dev(dlogits_add, "dlogits_add"),)
    call = lib.moe_route_topk_backward if dlogits_add is None else lib.moe_route_topk_backward_aux
    st = call(_dev(dgate, "dgate"), _dev(topk_gate, "topk_gate"), _dev(topk_idx, "topk_idx"), *scores,
              _dev(x, "x"), _dev(w_router, "w_router"), dtype, T, d, E, k, flags, _dev(dlogits, "dlogits"),
              _dev(dx, "dx"), _dev(dw, "dw"), _dev(dbias, "dbias"), _dev(ws, "ws"), ws.numel(), _stream(stream))
    _check("moe_route_topk_backward", st)
    return dlogits, dx, dw, dbias


_current_gpu = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _arg(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, *shape: int):
    """Device pointer of a contiguous tensor of this type and shape on the current GPU, where the
    call's stream is (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError("%s must be %s %s, got %s %s" % (name, dtype, shape, t.dtype, tuple(t.shape)))
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if t.get_device() != _current_gpu():
        raise ValueError("%s must be on the current GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def int8_cols(cols: int) -> int:
    """Columns of an 8-bit row: `cols` padded to a multiple of 128 (MOE_INT8_COLS)."""
    return (int(cols) + 127) // 128 * 128


def moe_quantize_int8(x: torch.Tensor, *, q: Optional[torch.Tensor] = None,
                      scales: Optional[torch.Tensor] = None, stream=None):
    """The rows of x [rows, cols] in 8 bits.  Returns (codes int8 [rows, int8_cols(cols)], scales
    float32 [rows])."""
    lib = load_library()
    rows, cols = x.shape
    at_x = _arg(x, "x", x.dtype, rows, cols)
    new = x.new_empty if stream is None else _of(stream, x.new_empty)
    if q is None:
        q = new((rows, int8_cols(cols)), dtype=torch.int8)
    if scales is None:
        scales = new(rows, dtype=torch.float32)
    st = lib.moe_quantize_int8(at_x, _dtype_code(x), rows, cols,
                               _arg(q, "q", torch.int8, rows, int8_cols(cols)),
                               _arg(scales, "scales", torch.float32, rows), _stream(stream))
    _check("moe_quantize_int8", st)
    return q, scales


def moe_dequantize_int8(q: torch.Tensor, scales: torch.Tensor, cols: int, *,
                        dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """The values [rows, cols] that 8-bit rows hold, in `dtype` (float32 or bfloat16)."""
    lib = load_library()
    rows = q.shape[0]
    if cols < 1:
        raise ValueError("cols must be positive")
    at_q, at_scales = _arg(q, "q", torch.int8, rows, int8_cols(cols)), _arg(scales, "scales", torch.float32, rows)
    if out is None:
        new = q.new_empty if stream is None else _of(stream, q.new_empty)
        out = new((rows, cols), dtype=dtype)
        at_out = out.data_ptr()
    else:
        at_out = _arg(out, "out", dtype, rows, cols)
    st = lib.moe_dequantize_int8(at_q, at_scales, rows, cols, _dtype_code(out), at_out, _stream(stream))
    _check("moe_dequantize_int8", st)
    return out


class Int8WeightTable:
    """Experts whose weights are 8-bit rows, as moe_grouped_ffn_int8 takes them: w13 and w2 hold one
    (codes, scales) pair per group, as moe_quantize_int8 gives them for [2f, d] and [d, f]."""

    def __init__(self, w13: Sequence, w2: Sequence, d: int, f: int):
        if len(w13) != len(w2) or not len(w13):
            raise ValueError("need one (w13, w2) pair per group")
        self.d, self.f = int(d), int(f)
        self.w13, self.w2 = [tuple(p) for p in w13], [tuple(p) for p in w2]
        for pairs, rows, cols, name in ((self.w13, 2 * self.f, self.d, "w13"), (self.w2, self.d, self.f, "w2")):
            for q, s in pairs:
                _arg(q, name + " codes", torch.int8, rows, int8_cols(cols))
                _arg(s, name + " scales", torch.float32, rows)
        n = len(self.w13)
        self._arrays = [(ctypes.c_void_p * n)(*[p[i].data_ptr() for p in pairs])
                        for pairs in (self.w13, self.w2) for i in (0, 1)]
        self.pointers = [ctypes.cast(a, ctypes.c_void_p) for a in self._arrays]

    @classmethod
    def quantized(cls, w13: Sequence[torch.Tensor], w2: Sequence[torch.Tensor]) -> "Int8WeightTable":
        """The experts of a WeightTable (w13 [2f, d], w2 [d, f], bf16 or fp32), quantized."""
        if not len(w13):
            raise ValueError("need one (w13, w2) pair per group")
        return cls([moe_quantize_int8(w) for w in w13], [moe_quantize_int8(w) for w in w2],
                   w13[0].shape[1], w13[0].shape[0] // 2)

    def __len__(self):
        return len(self.w13)


def moe_grouped_ffn_int8_ws_bytes(cap_rows: int, d: int, f: int, n_groups: int) -> int:
    return int(load_library().moe_grouped_ffn_int8_ws_bytes(cap_rows, d, f, n_groups))


def moe_grouped_ffn_int8(xq: torch.Tensor, x_scale: torch.Tensor, group_offsets: torch.Tensor,
                         weights: Int8WeightTable, *, row_token: Optional[torch.Tensor] = None,
                         n_shared: int = 0, cap_rows: Optional[int] = None,
                         y_perm: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """SwiGLU FFN of every group in 8-bit integers; xq [T, int8_cols(d)] with x_scale [T], read
    through row_token (as moe_grouped_ffn_rows_shared's, n_shared leading groups included) or,
    without it, the packaged rows.  Returns y_perm [n_shared * T + cap_rows, d] bf16."""
    lib = load_library()
    T = xq.shape[0]
    d, f = weights.d, weights.f
    at_x, at_scale = _arg(xq, "xq", torch.int8, T, int8_cols(d)), _arg(x_scale, "x_scale", torch.float32, T)
    if cap_rows is None:
        if row_token is not None:
            raise ValueError("row_token needs cap_rows")
        cap_rows = T
    n_groups = len(weights) - n_shared
    if n_shared < 0 or n_groups < 0 or group_offsets.numel() != n_groups + 1:
        raise ValueError("group_offsets must hold n_groups + 1 entries for the routed groups")
    rows = n_shared * T + cap_rows
    _holds(row_token, "row_token", rows)
    if weights.w13[0][0].device != xq.device:
        raise ValueError("the experts must be on the current GPU")
    if y_perm is None:
        y_perm = _empty((max(rows, 1), d), torch.bfloat16, xq.device, stream)
    _holds(y_perm, "y_perm", rows, d)
    if ws is None:
        ws = workspace(moe_grouped_ffn_int8_ws_bytes(rows, d, f, len(weights)), xq.device, stream)
    st = lib.moe_grouped_ffn_int8(
        at_x, at_scale, T, _dev(row_token, "row_token", torch.int32),
        _dev(group_offsets, "group_offsets", torch.int32), n_groups, n_shared, *weights.pointers,
        d, f, cap_rows, _dev(y_perm, "y_perm", torch.bfloat16), _dev(ws, "ws"), ws.numel(),
        _stream(stream))
    _check("moe_grouped_ffn_int8", st)
    return y_perm


def moe_rmsnorm(x: torch.Tensor, weight: torch.Tensor, *, residual: Optional[torch.Tensor] = None,
                eps: float = 1e-6, h: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                want_y: bool = True, rstd: Optional[torch.Tensor] = None, want_rstd: bool = False,
                q: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                want_q: bool = False, stream=None):
    """Root-mean-square norm of the rows of x [T, d] (+ residual).  Returns (h = the sum, or x
    itself without a residual; y; rstd [T]; q, scales: y in 8 bits), None for what is not wanted."""
    lib = load_library()
    T, d = x.shape
    dt, f32, P = x.dtype, torch.float32, int8_cols(d)
    at_x, at_weight = _arg(x, "x", dt, T, d), _arg(weight, "weight", dt, d)
    at_residual, at_h = _arg(residual, "residual", dt, T, d), _arg(h, "h", dt, T, d)
    at_y, at_rstd = _arg(y, "y", dt, T, d), _arg(rstd, "rstd", f32, T)
    at_q, at_scales = _arg(q, "q", torch.int8, T, P), _arg(scales, "scales", f32, T)
    if (q is None) != (scales is None):
        raise ValueError("q and scales go together")
    like, new = torch.empty_like, x.new_empty
    if stream is not None:
        like, new = _of(stream, like), _of(stream, new)
    if residual is None:
        if h is not None:
            raise ValueError("h is x itself without a residual")
    elif h is None:
        h = like(x)
        at_h = h.data_ptr()
    if want_y and y is None:
        y = like(x)
        at_y = y.data_ptr()
    if want_rstd and rstd is None:
        rstd = new(T, dtype=f32)
        at_rstd = rstd.data_ptr()
    if want_q and q is None:
        q, scales = new((T, P), dtype=torch.int8), new(T, dtype=f32)
        at_q, at_scales = q.data_ptr(), scales.data_ptr()
    # (no rows have no address: nothing is written)
    st = lib.moe_rmsnorm(at_x, at_residual, _dtype_code(x), at_weight, eps, T, d, at_h, at_y, at_rstd, at_q or None,
                         at_scales or None, _stream(stream))
    _check("moe_rmsnorm", st)
    return (x if residual is None else h), y, rstd, q, scales


def moe_rmsnorm_backward_ws_bytes(dtype: int, T: int, d: int) -> int:
    return int(load_library().moe_rmsnorm_backward_ws_bytes(dtype, T, d))


def moe_rmsnorm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, *,
                         dh_add: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None,
                         dw: Optional[torch.Tensor] = None, want_dh: bool = True, want_dw: bool = True,
                         ws: Optional[torch.Tensor] = None, stream=None):
    """Gradient of moe_rmsnorm's y, on top of dh_add.  Returns (dh [T, d], of x and of the residual;
    dw [d] float32), None for what is not wanted."""
    lib = load_library()
    T, d = dy.shape
    dt, dtype = dy.dtype, _dtype_code(dy)
    at_dy, at_h, at_weight = _arg(dy, "dy", dt, T, d), _arg(h, "h", dt, T, d), _arg(weight, "weight", dt, d)
    at_rstd, at_add = _arg(rstd, "rstd", torch.float32, T), _arg(dh_add, "dh_add", dt, T, d)
    at_dh, at_dw = _arg(dh, "dh", dt, T, d), _arg(dw, "dw", torch.float32, d)
    like, new = torch.empty_like, dy.new_empty
    if stream is not None:
        like, new = _of(stream, like), _of(stream, new)
    if want_dh and dh is None:
        dh = like(dy)
        at_dh = dh.data_ptr()
    if want_dw and dw is None:
        dw = new(d, dtype=torch.float32)
        at_dw = dw.data_ptr()
    if dw is not None and ws is None:
        ws = new(moe_rmsnorm_backward_ws_bytes(dtype, T, d), dtype=torch.uint8)
    st = lib.moe_rmsnorm_backward(at_dy, at_h, dtype, at_weight, at_rstd, at_add, T, d, at_dh, at_dw,
                                  _dev(ws, "ws"), 0 if ws is None else ws.numel(), _stream(stream))
    _check("moe_rmsnorm_backward", st)
    return dh, dw


def _mask(mask: Optional[torch.Tensor], T: int):
    """Device pointer of a token mask (bool or uint8 [T]; None -> NULL)."""
    if mask is not None and mask.dtype is not torch.bool and mask.dtype is not torch.uint8:
        raise ValueError("mask must be bool or uint8 [%d]" % T)
    return None if mask is None else _arg(mask, "mask", mask.dtype, T)


def moe_balance_loss_ws_bytes(T: int, E: int) -> int:
    return int(load_library().moe_balance_loss_ws_bytes(T, E))


def moe_balance_loss(logits: torch.Tensor, topk_idx: torch.Tensor, *, mask: Optional[torch.Tensor] = None,
                     loss: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None,
                     prob_sum: Optional[torch.Tensor] = None, n_tokens: Optional[torch.Tensor] = None,
                     ws: Optional[torch.Tensor] = None, stream=None):
    """Balance loss of a routing over the tokens where mask [T] is not 0.  Returns (loss [1],
    counts [E] int32, prob_sum [E], n_tokens [1] int32), on the device."""
    lib = load_library()
    T, E = logits.shape
    k = topk_idx.shape[1]
    f32, i32 = torch.float32, torch.int32
    at_logits, at_idx, at_mask = _arg(logits, "logits", f32, T, E), _arg(topk_idx, "topk_idx", i32, T, k), _mask(mask, T)
    at_loss, at_n = _arg(loss, "loss", f32, 1), _arg(n_tokens, "n_tokens", i32, 1)
    at_counts, at_sums = _arg(counts, "counts", i32, E), _arg(prob_sum, "prob_sum", f32, E)
    new = logits.new_empty if stream is None else _of(stream, logits.new_empty)
    if loss is None:
        loss = new(1)
        at_loss = loss.data_ptr()
    if counts is None:
        counts = new(E, dtype=i32)
        at_counts = counts.data_ptr()
    if prob_sum is None:
        prob_sum = new(E)
        at_sums = prob_sum.data_ptr()
    if n_tokens is None:
        n_tokens = new(1, dtype=i32)
        at_n = n_tokens.data_ptr()
    if ws is None:
        ws = new(moe_balance_loss_ws_bytes(T, E), dtype=torch.uint8)
    st = lib.moe_balance_loss(at_logits, at_idx, at_mask, T, E, k, at_counts, at_sums, at_n, at_loss,
                              _dev(ws, "ws"), ws.numel(), _stream(stream))
    _check("moe_balance_loss", st)
    return loss, counts, prob_sum, n_tokens


def moe_balance_loss_backward(logits: torch.Tensor, counts: torch.Tensor, n_tokens: torch.Tensor, k: int, *,
                              scale: float = 1.0, mask: Optional[torch.Tensor] = None,
                              dlogits: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of moe_balance_loss, times scale.  Returns dlogits [T, E]."""
    lib = load_library()
    T, E = logits.shape
    f32, i32 = torch.float32, torch.int32
    at_logits, at_counts = _arg(logits, "logits", f32, T, E), _arg(counts, "counts", i32, E)
    at_n, at_out = _arg(n_tokens, "n_tokens", i32, 1), _arg(dlogits, "dlogits", f32, T, E)
    if dlogits is None:
        dlogits = (torch.empty_like if stream is None else _of(stream, torch.empty_like))(logits)
        at_out = dlogits.data_ptr()
    st = lib.moe_balance_loss_backward(at_logits, _mask(mask, T), at_counts, at_n, T, E, k, scale, at_out,
                                       _stream(stream))
    _check("moe_balance_loss_backward", st)
    return dlogits


def _outputs_apart(reads: Sequence[int], writes: Sequence[int], nbytes: Sequence[int]) -> bool:
    """Whether entries that read nbytes[i] at reads[i] and write as many at writes[i], all at once, keep
    apart: a write meets no other entry's write or read, and its own read only as the same place."""
    spans = [(w, w + n, True) for w, n in zip(writes, nbytes) if n]
    spans += [(r, r + n, False) for r, w, n in zip(reads, writes, nbytes) if n and r != w]
    end = end_written = 0                            # of the spans before, of the written ones
    for at, to, written in sorted(spans):
        if at < (end if written else end_written):
            return False
        end = max(end, to)
        if written:
            end_written = max(end_written, to)
    return True


class GradTable:
    """Host arrays of a step's gradients (float32 or bfloat16, any shapes), as moe_grad_norm and
    moe_clip_grads take them; out (None: in place): where the clipped ones go."""

    def __init__(self, grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        if len(self.out) != len(self.grads):
            raise ValueError("need one output per gradient")
        n = len(self.grads)
        for g, o in zip(self.grads, self.out):
            _dtype_code(g)
            if o.dtype != g.dtype or o.shape != g.shape:
                raise ValueError("outputs must be of the gradients' types and shapes")
        self.pointers = (ctypes.c_void_p * n)(*[_arg(g, "grads", g.dtype, *g.shape) for g in self.grads])
        self.outputs = (ctypes.c_void_p * n)(*[_arg(o, "out", o.dtype, *o.shape) for o in self.out])
        self.sizes = (ctypes.c_int64 * n)(*[g.numel() for g in self.grads])
        self.dtypes = (ctypes.c_int * n)(*[_dtype_code(g) for g in self.grads])
        self._apart = _outputs_apart([g.data_ptr() for g in self.grads], [o.data_ptr() for o in self.out],
                                     [g.numel() * g.element_size() for g in self.grads])

    def __len__(self):
        return len(self.grads)


def moe_grad_norm_ws_bytes(table: GradTable) -> int:
    return int(load_library().moe_grad_norm_ws_bytes(table.sizes, len(table)))


def moe_grad_norm(table: GradTable, *, norm: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The norm over all gradients of a table.  Returns norm [1] float32, on the device."""
    lib = load_library()
    if norm is None:
        if not len(table):
            raise ValueError("a table without gradients needs norm")
        norm = _empty((1,), torch.float32, table.grads[0].device, stream)
    if ws is None:
        ws = workspace(moe_grad_norm_ws_bytes(table), norm.device, stream)
    st = lib.moe_grad_norm(table.pointers, table.sizes, table.dtypes, len(table),
                           _arg(norm, "norm", torch.float32, 1),
                           _dev(ws, "ws"), ws.numel(), _stream(stream))
    _check("moe_grad_norm", st)
    return norm


def moe_clip_grads(table: GradTable, norm: torch.Tensor, max_norm: float, *, stream=None):
    """Scale a table's gradients by max_norm / norm where that is below 1.  Returns its outputs, of which
    none may overlap another, or any gradient but its own in place."""
    lib = load_library()
    if not table._apart:
        raise ValueError("an output is in the table twice, or outputs and gradients overlap")
    st = lib.moe_clip_grads(table.pointers, table.sizes, table.dtypes, len(table),
                            _arg(norm, "norm", torch.float32, 1), max_norm, table.outputs, _stream(stream))
    _check("moe_clip_grads", st)
    return table.out
