"""Thin Python binding of libmoe.so (include/moe.h): argument marshalling only.

Every step of the MoE FFN runs in the HIP library; these wrappers turn torch
tensors into device pointers and the current torch stream into a hipStream_t,
and raise ``MoEError`` on a non-zero status.  The library must be built
(``python -m paper_2410_12247_amd.build``); if it is missing, loading fails
loudly: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmoe.so")

BF16, FP32 = 0, 1
GEMM_AUTO, GEMM_GROUP, GEMM_DENSE = 0, 1, 2
CHUNK_EXPERTS, CHUNK_TOKENS = 0, 1
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
GROUP_MAX, GROUP_TOP_TWO = 0, 1
FLAG_TIMING, FLAG_TIMING_GEMM, FLAG_EXACT_ORDER, FLAG_SERIAL = 1, 2, 4, 8

# the entry points include/moe.h declares
EXPORTS = ("moe_workspace_bytes", "moe_workspace_guards", "moe_route", "moe_permute", "moe_gather", "moe_ffn_group",
           "moe_ffn_dense", "moe_combine", "moe_ffn_forward", "moe_ffn_forward_noalloc",
           "moe_last_timing",
           "moe_gemm_plan", "moe_pipeline_plan", "moe_choose_pipeline_n", "moe_status_string",
           "moe_last_error", "moe_scale_pitch", "moe_quant_rows", "moe_quant_weights",
           "moe_norm_quant", "moe_gemm_scaled", "moe_gemm_group_scaled",
           "moe_scaled_workspace_bytes", "moe_ffn_group_scaled", "moe_combine_rows",
           "moe_forward_scaled", "moe_forward_scaled_bytes",
           "moe_route_logits", "moe_route_scores", "moe_route_scores_backward",
           "moe_adapter_workspace_bytes", "moe_adapter_rows", "moe_adapter_backward_bytes",
           "moe_adapter_backward")


class MoEError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(msg)
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("hidden", ctypes.c_int32),
                ("inter", ctypes.c_int32), ("experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("local_begin", ctypes.c_int32),
                ("local_count", ctypes.c_int32), ("renormalize", ctypes.c_int32),
                ("shared_inter", ctypes.c_int32)]


class Opts(ctypes.Structure):
    _fields_ = [("gemm_mode", ctypes.c_int32), ("dense_min_rows", ctypes.c_int32),
                ("pipeline_n", ctypes.c_int32), ("gemm_cu_budget", ctypes.c_int32),
                ("flags", ctypes.c_int32), ("chunk_mode", ctypes.c_int32),
                ("dense_tile_rows", ctypes.c_int32), ("side_cus", ctypes.c_int32),
                ("group_tile_rows", ctypes.c_int32)]


class Timing(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("route_ms", "permute_ms", "gather_ms", "gateup_ms",
                                             "down_ms", "shared_ms", "combine_ms", "total_ms")] + \
               [(n, ctypes.c_int32) for n in ("gateup_launches", "down_launches",
                                             "dense_stages", "group_stages", "pipeline_n",
                                             "calls")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class ScaledWeights(ctypes.Structure):
    """A layer's quantised weights (moe_scaled_weights); scaled_weights() fills it."""
    _fields_ = [(n + s, ctypes.c_void_p)
                for n in ("gate", "up", "down", "shared_gate", "shared_up", "shared_down")
                for s in ("", "_scales")]


class Routing(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("score", "groups", "top_groups", "group_score")] + \
               [("scale", ctypes.c_float)]


class Adapters(ctypes.Structure):
    """The low-rank adapters of a projection (moe_adapters); adapters() fills it."""
    _fields_ = [(n, ctypes.c_int32) for n in ("count", "rank", "n", "k")] + \
               [(n, ctypes.c_void_p) for n in ("a", "b", "scale")]


class PipelineEval(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("t_comm_us", "t_comp_us", "t_comm_n_us",
                                              "t_comp_n_us", "eps0", "eps1", "overlap_frac",
                                              "gain_us")] + \
               [("enabled", ctypes.c_int32), ("pipeline_n", ctypes.c_int32)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


_lib = None


def lib():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run python -m paper_2410_12247_amd.build")
    L = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    D, O = ctypes.POINTER(Dims), ctypes.POINTER(Opts)
    L.moe_workspace_bytes.argtypes = [D, O]
    L.moe_workspace_bytes.restype = SZ
    L.moe_workspace_guards.argtypes = [D, O, ctypes.POINTER(ctypes.c_int64), ctypes.c_int32]
    L.moe_workspace_guards.restype = ctypes.c_int32
    L.moe_route.argtypes = [D, P, P, P, P, P, P]
    L.moe_permute.argtypes = [D, P, P, P, P, P, P, P, P, SZ, P]
    L.moe_gather.argtypes = [D, I32, I32, P, P, P, P, P]
    L.moe_ffn_group.argtypes = [D, I32, I32, P, P, P, P, P, P, P, I32, P]
    L.moe_ffn_dense.argtypes = [I64, I32, I32, P, P, P, P, P, P, P]
    L.moe_combine.argtypes = [D, I32, I32, P, P, P, P, P, I32, P]
    L.moe_ffn_forward.argtypes = [D, O, P, P, P, P, P, P, P, P, P, P, P, P, P, P, SZ, P]
    L.moe_ffn_forward_noalloc.argtypes = [D, O, P, P, P, P, P, P, P, P, P, P, P, P, P, P]
    L.moe_last_timing.argtypes = [ctypes.POINTER(Timing)]
    L.moe_pipeline_plan.argtypes = [D, O, P, I32, ctypes.POINTER(PipelineEval)]
    L.moe_gemm_plan.argtypes = [D, O, I32, P, ctypes.POINTER(I32), P,
                                ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    L.moe_choose_pipeline_n.argtypes = [ctypes.c_double, ctypes.c_double, ctypes.c_double, I32,
                                        ctypes.POINTER(I32), ctypes.POINTER(ctypes.c_double)]
    L.moe_scale_pitch.argtypes = [I32]
    L.moe_scale_pitch.restype = SZ
    L.moe_quant_rows.argtypes = [I64, I32, P, I32, P, P, P]
    L.moe_quant_weights.argtypes = [I32, I32, I32, P, P, P, P]
    L.moe_norm_quant.argtypes = [I64, I32, P, I32, P, P, ctypes.c_float, P, P, P, P, P]
    L.moe_gemm_scaled.argtypes = [I64, I32, I32, P, P, P, P, P, I32, P]
    L.moe_gemm_group_scaled.argtypes = [D, I32, I32, P, P, I32, I32, P, P, P, P, P, I32, P]
    L.moe_scaled_workspace_bytes.argtypes = [D]
    L.moe_scaled_workspace_bytes.restype = SZ
    L.moe_ffn_group_scaled.argtypes = [D, I32, I32] + [P] * 11 + [I32, P, SZ, P]
    L.moe_combine_rows.argtypes = [D, I32, I32, P, I32, P, P, P, P, I32, P]
    L.moe_forward_scaled_bytes.argtypes = [D]
    L.moe_forward_scaled_bytes.restype = SZ
    L.moe_forward_scaled.argtypes = [D, P, I32, P, P, ctypes.c_float, P, P, P,
                                     ctypes.POINTER(ScaledWeights), P, P, P, P, P, SZ, P]
    R, A = ctypes.POINTER(Routing), ctypes.POINTER(Adapters)
    L.moe_route_logits.argtypes = [D, P, P, P, P]
    L.moe_route_scores.argtypes = [D, R, P, I32, P, P, P, P]
    L.moe_route_scores_backward.argtypes = [D, R, P, I32, P, P, P, P]
    for name in ("moe_adapter_workspace_bytes", "moe_adapter_backward_bytes"):
        getattr(L, name).argtypes = [I64, A]
        getattr(L, name).restype = SZ
    L.moe_adapter_rows.argtypes = [I64, A] + [P] * 6 + [I32, P, SZ, P]
    L.moe_adapter_backward.argtypes = [I64, A] + [P] * 7 + [I32, P, P, I32, P, SZ, P]
    L.moe_status_string.argtypes = [I32]
    L.moe_status_string.restype = ctypes.c_char_p
    L.moe_last_error.restype = ctypes.c_char_p
    for name in ("moe_route", "moe_permute", "moe_gather", "moe_ffn_group", "moe_ffn_dense",
                 "moe_combine", "moe_ffn_forward", "moe_ffn_forward_noalloc", "moe_last_timing",
                 "moe_choose_pipeline_n", "moe_gemm_plan", "moe_pipeline_plan", "moe_quant_rows",
                 "moe_quant_weights", "moe_norm_quant", "moe_gemm_scaled",
                 "moe_gemm_group_scaled", "moe_ffn_group_scaled", "moe_combine_rows",
                 "moe_forward_scaled", "moe_route_logits", "moe_route_scores",
                 "moe_route_scores_backward", "moe_adapter_rows", "moe_adapter_backward"):
        getattr(L, name).restype = I32
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        L = lib()
        raise MoEError(status, f"{L.moe_status_string(status).decode()}: "
                               f"{L.moe_last_error().decode()}")


def dims(tokens, hidden, inter, experts, top_k, local_begin=0, local_count=None,
         renormalize=True, shared_inter=0) -> Dims:
    return Dims(int(tokens), int(hidden), int(inter), int(experts), int(top_k),
                int(local_begin), int(experts if local_count is None else local_count),
                int(bool(renormalize)), int(shared_inter))


def opts(gemm_mode=GEMM_AUTO, dense_min_rows=0, pipeline_n=1, gemm_cu_budget=0,
         timing=False, chunk_mode=CHUNK_EXPERTS, exact_order=False, serial=False,
         dense_tile_rows=0, side_cus=0, group_tile_rows=0) -> Opts:
    """timing: False, True (every phase) or "gemm" (the GEMM launches only).
    exact_order: no K split of the grouped GEMM's last round (the same bits
    for every pipeline number, stage kind, CU budget and GEMM kind).
    serial: every stage on the caller's stream, nothing overlapped."""
    o = Opts()
    o.gemm_mode, o.dense_min_rows, o.pipeline_n = gemm_mode, dense_min_rows, pipeline_n
    o.gemm_cu_budget = gemm_cu_budget
    o.flags = FLAG_TIMING_GEMM if timing == "gemm" else (FLAG_TIMING if timing else 0)
    if exact_order:
        o.flags |= FLAG_EXACT_ORDER
    if serial:
        o.flags |= FLAG_SERIAL
    o.chunk_mode = chunk_mode
    o.dense_tile_rows = dense_tile_rows
    o.side_cus = side_cus
    o.group_tile_rows = group_tile_rows
    return o


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors passed to libmoe must be contiguous device tensors")
    return ctypes.c_void_p(t.data_ptr())


def _s(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def workspace_bytes(d: Dims, o: Optional[Opts] = None) -> int:
    return lib().moe_workspace_bytes(ctypes.byref(d), ctypes.byref(o) if o is not None else None)


WS_GUARD_BYTES = 256  # MOE_WS_GUARD_BYTES


def workspace_guards(d: Dims, o: Optional[Opts] = None) -> list:
    """Byte offsets of the workspace's guard gaps (WS_GUARD_BYTES each)."""
    ob = ctypes.byref(o) if o is not None else None
    n = lib().moe_workspace_guards(ctypes.byref(d), ob, None, 0)
    if n < 0:
        raise MoEError(1, "moe_workspace_guards: invalid dims or options")
    buf = (ctypes.c_int64 * max(n, 1))()
    lib().moe_workspace_guards(ctypes.byref(d), ob, buf, n)
    return list(buf[:n])


def route(d, x, w_router, bias, topk_ids, topk_w, stream=None):
    _check(lib().moe_route(ctypes.byref(d), _p(x), _p(w_router), _p(bias), _p(topk_ids),
                           _p(topk_w), _s(stream)))


def permute(d, topk_ids, x, counts, offsets, sorted_slot, slot_row, x_perm, ws, stream=None):
    _check(lib().moe_permute(ctypes.byref(d), _p(topk_ids), _p(x), _p(counts), _p(offsets),
                             _p(sorted_slot), _p(slot_row), _p(x_perm), _p(ws),
                             ws.numel() * ws.element_size(), _s(stream)))


def gather(d, e_first, e_count, offsets, sorted_slot, x, x_perm, stream=None):
    _check(lib().moe_gather(ctypes.byref(d), e_first, e_count, _p(offsets), _p(sorted_slot),
                            _p(x), _p(x_perm), _s(stream)))


def ffn_group(d, e_first, e_count, offsets, x_perm, w_gate, w_up, w_down, act, y_perm,
              cu_budget=0, stream=None):
    _check(lib().moe_ffn_group(ctypes.byref(d), e_first, e_count, _p(offsets), _p(x_perm),
                               _p(w_gate), _p(w_up), _p(w_down), _p(act), _p(y_perm),
                               cu_budget, _s(stream)))


def ffn_dense(rows, hidden, inter, x, w_gate, w_up, w_down, act, y, stream=None):
    _check(lib().moe_ffn_dense(int(rows), hidden, inter, _p(x), _p(w_gate), _p(w_up),
                               _p(w_down), _p(act), _p(y), _s(stream)))


def combine(d, e_first, e_count, y_perm, topk_ids, slot_row, topk_w, y, accumulate,
            stream=None):
    _check(lib().moe_combine(ctypes.byref(d), e_first, e_count, _p(y_perm), _p(topk_ids),
                             _p(slot_row), _p(topk_w), _p(y), int(accumulate), _s(stream)))


def forward(d, o, x, w_router, bias, w_gate, w_up, w_down, shared_gate, shared_up, shared_down,
            y, topk_ids, topk_w, counts, ws, stream=None):
    _check(lib().moe_ffn_forward(ctypes.byref(d), ctypes.byref(o) if o is not None else None,
                                 _p(x), _p(w_router), _p(bias), _p(w_gate), _p(w_up),
                                 _p(w_down), _p(shared_gate), _p(shared_up), _p(shared_down),
                                 _p(y), _p(topk_ids), _p(topk_w), _p(counts), _p(ws),
                                 ws.numel() * ws.element_size(), _s(stream)))


def forward_noalloc(d, o, x, w_router, bias, w_gate, w_up, w_down, shared_gate, shared_up,
                    shared_down, y, topk_ids, topk_w, counts, stream=None):
    """moe_ffn_forward_noalloc: the forward with the library's static scratch
    buffer instead of a workspace (no allocation in the call)."""
    _check(lib().moe_ffn_forward_noalloc(
        ctypes.byref(d), ctypes.byref(o) if o is not None else None, _p(x), _p(w_router),
        _p(bias), _p(w_gate), _p(w_up), _p(w_down), _p(shared_gate), _p(shared_up),
        _p(shared_down), _p(y), _p(topk_ids), _p(topk_w), _p(counts), _s(stream)))


def choose_pipeline_n(c_ms: float, k_ms: float, b_ms: float, local_count: int):
    """(PN, gain in ms) from the paper's pipeline overhead model."""
    pn = ctypes.c_int32()
    gain = ctypes.c_double()
    _check(lib().moe_choose_pipeline_n(float(c_ms), float(k_ms), float(b_ms), int(local_count),
                                       ctypes.byref(pn), ctypes.byref(gain)))
    return pn.value, gain.value


def last_timing() -> dict:
    t = Timing()
    _check(lib().moe_last_timing(ctypes.byref(t)))
    return t.as_dict()


def pipeline_plan(d: Dims, o: Optional[Opts], rows, pipeline_n: int) -> dict:
    """The paper's pipeline terms for PN = pipeline_n (0: the library's
    choice) from host row counts per local expert."""
    import numpy as np
    r = np.ascontiguousarray(rows, dtype=np.int32)
    ev = PipelineEval()
    _check(lib().moe_pipeline_plan(ctypes.byref(d), ctypes.byref(o) if o is not None else None,
                                   r.ctypes.data_as(ctypes.c_void_p), int(pipeline_n),
                                   ctypes.byref(ev)))
    return ev.as_dict()


def gemm_plan(d: Dims, o: Optional[Opts], rows):
    """AUTO's plan for one stage with host row counts `rows`: (dense, tile
    rows per expert, predicted group us, predicted dense us)."""
    import numpy as np
    r = np.ascontiguousarray(rows, dtype=np.int32)
    tiles = np.zeros(len(r), np.int32)
    dense = ctypes.c_int32()
    gus, dus = ctypes.c_double(), ctypes.c_double()
    _check(lib().moe_gemm_plan(ctypes.byref(d), ctypes.byref(o) if o is not None else None,
                               len(r), r.ctypes.data_as(ctypes.c_void_p), ctypes.byref(dense),
                               tiles.ctypes.data_as(ctypes.c_void_p), ctypes.byref(gus),
                               ctypes.byref(dus)))
    return bool(dense.value), tiles.tolist(), gus.value, dus.value


# ---- block-scaled 8-bit operators -----------------------------------------
# Quantised values are float8_e4m3fn tensors (or their uint8 bits), scales
# uint8 (or float8_e8m0fnu).

_E4M3 = (torch.float8_e4m3fn, torch.uint8)
_SCALE = (torch.uint8, torch.float8_e8m0fnu)
_REAL = {torch.bfloat16: BF16, torch.float32: FP32}
_I32 = (torch.int32,)
_BF16 = (torch.bfloat16,)
_F32 = (torch.float32,)


# (Small batches take a few microseconds on the GPU: these checks are kept to
# tenths of one per tensor, and the stream is asked for without making a Stream
# object, which takes 3.)

def _real(name, t):
    """The element type's code."""
    code = _REAL.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be bfloat16 or float32, not {t.dtype}")
    return code


def _dev(name, t):
    """The current device, which t has to be on."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a contiguous device tensor, not on {t.device}")
    if dev != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    return dev


def _arg(dev, name, t, dtypes, shape):
    """The address of a contiguous tensor on dev with one of the dtypes and the
    shape, or None for None."""
    if t is None:
        return None
    if t.get_device() != dev or t.dtype not in dtypes or t.shape != shape or \
            not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous device tensor of shape {tuple(shape)} and "
                         f"type {dtypes[0]} on cuda:{dev}, not {tuple(t.shape)} of {t.dtype} on "
                         f"{t.device}")
    return t.data_ptr()


def _stream_on(dev, stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError(f"the stream is on cuda:{stream.device_index}, the tensors on cuda:{dev}")
    return stream.cuda_stream


def _rows(name, t, cols=None):
    if t.dim() != 2 or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name} must be 2-dimensional" +
                         (f" with {cols} columns" if cols is not None else ""))
    return t.shape


def scale_pitch(k: int) -> int:
    """Bytes of a scale row of a width k."""
    n = lib().moe_scale_pitch(k)
    if n == 0:
        raise ValueError(f"width {k} is not a positive multiple of 64 up to 2^20")
    return n


def _pitch(k):
    return 4 * -(-k // 512)


def quant_rows(x, q, scales, stream=None):
    """q, scales = Q(x): one scale per row and 128 columns."""
    shape = R, C = _rows("x", x)
    dev, code = _dev("x", x), _real("x", x)
    _check(lib().moe_quant_rows(R, C, _arg(dev, "x", x, (x.dtype,), shape), code,
                                _arg(dev, "q", q, _E4M3, shape),
                                _arg(dev, "scales", scales, _SCALE, (R, _pitch(C))),
                                _stream_on(dev, stream)))


def quant_weights(w, q, scales, stream=None):
    """q, scales = Q(w) in 128 x 128 blocks; w [n, k] or [experts, n, k] bf16."""
    if w.dim() not in (2, 3):
        raise ValueError("w must be [n, k] or [experts, n, k]")
    lead, (n, k), dev = w.shape[:-2], w.shape[-2:], _dev("w", w)
    _check(lib().moe_quant_weights(lead[0] if lead else 1, n, k,
                                   _arg(dev, "w", w, _BF16, w.shape),
                                   _arg(dev, "q", q, _E4M3, w.shape),
                                   _arg(dev, "scales", scales, _SCALE,
                                        lead + (-(-n // 128), _pitch(k))),
                                   _stream_on(dev, stream)))


def norm_quant(x, residual, weight, eps, total, y, q, scales, stream=None):
    """total = bf16(x + residual), y = bf16(v) and q, scales = Q(v) for the
    RMS-normalised rows v = norm(x + residual) * weight.  residual, weight,
    total, y and the pair q, scales may be None."""
    shape = R, H = _rows("x", x)
    dev, code = _dev("x", x), _real("x", x)
    _check(lib().moe_norm_quant(R, H, _arg(dev, "x", x, (x.dtype,), shape), code,
                                _arg(dev, "residual", residual, _BF16, shape),
                                _arg(dev, "weight", weight, _BF16, (H,)), eps,
                                _arg(dev, "total", total, _BF16, shape),
                                _arg(dev, "y", y, _BF16, shape), _arg(dev, "q", q, _E4M3, shape),
                                _arg(dev, "scales", scales, _SCALE, (R, _pitch(H))),
                                _stream_on(dev, stream)))


def gemm_scaled(x, x_scales, w, w_scales, y, stream=None):
    """y = x w^T over block-scaled x [rows, k] and w [n, k]; y bf16 or fp32."""
    R, K = _rows("x", x)
    N, _ = _rows("w", w, K)
    dev, code, P = _dev("x", x), _real("y", y), _pitch(K)
    _check(lib().moe_gemm_scaled(R, N, K, _arg(dev, "x", x, _E4M3, (R, K)),
                                 _arg(dev, "x_scales", x_scales, _SCALE, (R, P)),
                                 _arg(dev, "w", w, _E4M3, (N, K)),
                                 _arg(dev, "w_scales", w_scales, _SCALE, (-(-N // 128), P)),
                                 _arg(dev, "y", y, (y.dtype,), (R, N)), code,
                                 _stream_on(dev, stream)))


def _row_cap(d):
    return d.tokens * min(d.top_k, d.local_count)


def _group_args(dev, d, offsets, sorted_slot, x, x_scales, k):
    """Addresses of what the grouped calls share; x holds the tokens' rows
    with sorted_slot, else the dispatched rows."""
    cap = _row_cap(d)
    rows = d.tokens if sorted_slot is not None else cap
    return (_arg(dev, "offsets", offsets, _I32, (d.local_count + 1,)),
            _arg(dev, "sorted_slot", sorted_slot, _I32, (cap,)),
            _arg(dev, "x", x, _E4M3, (rows, k)),
            _arg(dev, "x_scales", x_scales, _SCALE, (rows, _pitch(k))))


def _stack(dev, name, d, w, s, n, k):
    return (_arg(dev, name, w, _E4M3, (d.local_count, n, k)),
            _arg(dev, name + " scales", s, _SCALE, (d.local_count, -(-n // 128), _pitch(k))))


def gemm_group_scaled(d, e_first, e_count, offsets, sorted_slot, x, x_scales, w, w_scales, y,
                      stream=None):
    """gemm_scaled per local expert over the rows offsets gives each; with
    sorted_slot the rows are gathered from the tokens' x."""
    if w.dim() != 3:
        raise ValueError("w must be [local_count, n, k]")
    N, K = w.shape[1:]
    dev, code = _dev("x", x), _real("y", y)
    off, slot, xp, xsp = _group_args(dev, d, offsets, sorted_slot, x, x_scales, K)
    wp, wsp = _stack(dev, "w", d, w, w_scales, N, K)
    _check(lib().moe_gemm_group_scaled(ctypes.byref(d), e_first, e_count, off, slot, N, K, xp,
                                       xsp, wp, wsp,
                                       _arg(dev, "y", y, (y.dtype,), (_row_cap(d), N)), code,
                                       _stream_on(dev, stream)))


def scaled_workspace_bytes(d: Dims) -> int:
    return lib().moe_scaled_workspace_bytes(ctypes.byref(d))


def ffn_group_scaled(d, e_first, e_count, offsets, sorted_slot, x, x_scales, w_gate, gate_scales,
                     w_up, up_scales, w_down, down_scales, y_perm, ws, stream=None):
    """The experts' SwiGLU FFN in 8 bits; y_perm bf16 or fp32, ws of
    scaled_workspace_bytes(d) bytes."""
    H, I = d.hidden, d.inter
    dev, code = _dev("x", x), _real("y_perm", y_perm)
    off, slot, xp, xsp = _group_args(dev, d, offsets, sorted_slot, x, x_scales, H)
    _check(lib().moe_ffn_group_scaled(
        ctypes.byref(d), e_first, e_count, off, slot, xp, xsp,
        *_stack(dev, "w_gate", d, w_gate, gate_scales, I, H),
        *_stack(dev, "w_up", d, w_up, up_scales, I, H),
        *_stack(dev, "w_down", d, w_down, down_scales, H, I),
        _arg(dev, "y_perm", y_perm, (y_perm.dtype,), (_row_cap(d), H)), code,
        _arg(dev, "ws", ws, (ws.dtype,), ws.shape), ws.numel() * ws.element_size(),
        _stream_on(dev, stream)))


def combine_rows(d, e_first, e_count, y_perm, topk_ids, slot_row, topk_w, y, accumulate,
                 stream=None):
    """combine for y_perm of bf16 or fp32."""
    dev, code = _dev("y_perm", y_perm), _real("y_perm", y_perm)
    slots = (d.tokens, d.top_k)
    _check(lib().moe_combine_rows(
        ctypes.byref(d), e_first, e_count,
        _arg(dev, "y_perm", y_perm, (y_perm.dtype,), (_row_cap(d), d.hidden)), code,
        _arg(dev, "topk_ids", topk_ids, _I32, slots),
        _arg(dev, "slot_row", slot_row.view(-1), _I32, (d.tokens * d.top_k,)),
        _arg(dev, "topk_w", topk_w, _F32, slots),
        _arg(dev, "y", y, _F32, (d.tokens, d.hidden)), int(accumulate), _stream_on(dev, stream)))


def _layer_shape(d):
    return d.hidden, d.inter, d.shared_inter, d.local_count


def scaled_weights(d, gate, up, down, shared_gate=None, shared_up=None,
                   shared_down=None) -> ScaledWeights:
    """Checks and packs a layer's weights, each a pair (q, scales) of
    quant_weights; made once and kept with the tensors."""
    H, I, Is = d.hidden, d.inter, d.shared_inter
    dev = _dev("gate", gate[0])
    w = ScaledWeights()
    w.keep = (gate, up, down, shared_gate, shared_up, shared_down)
    w.made_for = _layer_shape(d), dev
    for name, (q, s), n, k in (("gate", gate, I, H), ("up", up, I, H), ("down", down, H, I)):
        a, b = _stack(dev, name, d, q, s, n, k)
        setattr(w, name, a)
        setattr(w, name + "_scales", b)
    if Is:
        for name, pair, n, k in (("shared_gate", shared_gate, Is, H),
                                 ("shared_up", shared_up, Is, H),
                                 ("shared_down", shared_down, H, Is)):
            if pair is None:
                raise ValueError(f"dims have shared experts: {name} is missing")
            setattr(w, name, _arg(dev, name, pair[0], _E4M3, (n, k)))
            setattr(w, name + "_scales", _arg(dev, name + " scales", pair[1], _SCALE,
                                              (-(-n // 128), _pitch(k))))
    return w


def forward_scaled_bytes(d: Dims) -> int:
    return lib().moe_forward_scaled_bytes(ctypes.byref(d))


def forward_scaled(d, x, residual, norm_weight, eps, total, w_router, bias, weights, y, topk_ids,
                   topk_w, counts, ws, stream=None):
    """The MoE layer in 8 bits (moe_forward_scaled): norm, route, dispatch,
    experts, combine.  weights: scaled_weights(); norm_weight None: x holds bf16
    rows normalised before."""
    T, H, k = d.tokens, d.hidden, d.top_k
    dev, code = _dev("x", x), _real("x", x)
    if getattr(weights, "made_for", None) != (_layer_shape(d), dev):
        raise ValueError("weights are not scaled_weights() of these dims on this device")
    _check(lib().moe_forward_scaled(
        ctypes.byref(d), _arg(dev, "x", x, (x.dtype,), (T, H)), code,
        _arg(dev, "residual", residual, _BF16, (T, H)),
        _arg(dev, "norm_weight", norm_weight, _BF16, (H,)), eps,
        _arg(dev, "total", total, _BF16, (T, H)),
        _arg(dev, "w_router", w_router, _F32, (d.experts, H)),
        _arg(dev, "bias", bias, _F32, (d.experts,)), ctypes.byref(weights),
        _arg(dev, "y", y, _F32, (T, H)), _arg(dev, "topk_ids", topk_ids, _I32, (T, k)),
        _arg(dev, "topk_w", topk_w, _F32, (T, k)),
        _arg(dev, "counts", counts, _I32, (d.local_count,)), _arg(dev, "ws", ws, (ws.dtype,),
                                                                  ws.shape),
        ws.numel() * ws.element_size(), _stream_on(dev, stream)))


# ---- routing by scores ------------------------------------------------------


def routing(score=SCORE_SOFTMAX, groups=1, top_groups=1, group_score=GROUP_MAX,
            scale=1.0) -> Routing:
    return Routing(int(score), int(groups), int(top_groups), int(group_score), float(scale))


def route_logits(d, x, w_router, logits, stream=None):
    """logits = x w_router^T, as route computes them (no bias)."""
    dev = _dev("x", x)
    _check(lib().moe_route_logits(ctypes.byref(d), _arg(dev, "x", x, _BF16, (d.tokens, d.hidden)),
                                  _arg(dev, "w_router", w_router, _F32, (d.experts, d.hidden)),
                                  _arg(dev, "logits", logits, _F32, (d.tokens, d.experts)),
                                  _stream_on(dev, stream)))


def route_scores(d, r, logits, bias, topk_ids, topk_w, stream=None):
    """Experts and weights of logits fp32 or bf16 by the rules of r (routing()).
    bias may be None; ids are -1 where no expert is left."""
    dev, code = _dev("logits", logits), _real("logits", logits)
    slots = (d.tokens, d.top_k)
    _check(lib().moe_route_scores(
        ctypes.byref(d), ctypes.byref(r),
        _arg(dev, "logits", logits, (logits.dtype,), (d.tokens, d.experts)), code,
        _arg(dev, "bias", bias, _F32, (d.experts,)),
        _arg(dev, "topk_ids", topk_ids, _I32, slots), _arg(dev, "topk_w", topk_w, _F32, slots),
        _stream_on(dev, stream)))


def route_scores_backward(d, r, logits, topk_ids, dtopk_w, dlogits, stream=None):
    """dlogits (of logits' type) from dtopk_w, the gradient of route_scores' topk_w."""
    dev, code = _dev("logits", logits), _real("logits", logits)
    shape, slots = (d.tokens, d.experts), (d.tokens, d.top_k)
    _check(lib().moe_route_scores_backward(
        ctypes.byref(d), ctypes.byref(r), _arg(dev, "logits", logits, (logits.dtype,), shape),
        code, _arg(dev, "topk_ids", topk_ids, _I32, slots),
        _arg(dev, "dtopk_w", dtopk_w, _F32, slots),
        _arg(dev, "dlogits", dlogits, (logits.dtype,), shape), _stream_on(dev, stream)))


# ---- low-rank adapters ------------------------------------------------------


def adapters(a, b, scale=None) -> Adapters:
    """Checks and packs a projection's adapters: a [count, rank, k], b [count, n,
    rank] bf16, scale [count] fp32 or None; made once and kept with the tensors."""
    if a.dim() != 3 or b.dim() != 3:
        raise ValueError("a must be [count, rank, k] and b [count, n, rank]")
    (C, r, K), N, dev = a.shape, b.shape[1], _dev("a", a)
    ad = Adapters(C, r, N, K, _arg(dev, "a", a, _BF16, (C, r, K)),
                  _arg(dev, "b", b, _BF16, (C, N, r)), _arg(dev, "scale", scale, _F32, (C,)))
    ad.keep = (a, b, scale)
    ad.device = dev
    return ad


def adapter_workspace_bytes(rows: int, ad: Adapters) -> int:
    return lib().moe_adapter_workspace_bytes(rows, ctypes.byref(ad))


def adapter_backward_bytes(rows: int, ad: Adapters) -> int:
    """No less than adapter_workspace_bytes: one workspace serves both."""
    return lib().moe_adapter_backward_bytes(rows, ctypes.byref(ad))


def _adapter_args(ad, dev, R, offsets, sorted_slot, slot_row):
    """The handle and addresses of the rows' order (permute's outputs)."""
    if ad.device != dev:
        raise ValueError(f"the adapters are on cuda:{ad.device}, the rows on cuda:{dev}")
    if slot_row is not None and slot_row.dim() != 1:
        slot_row = slot_row.view(-1)
    return (ctypes.byref(ad), _arg(dev, "offsets", offsets, _I32, (ad.count + 1,)),
            _arg(dev, "sorted_slot", sorted_slot, _I32, (R,)),
            _arg(dev, "slot_row", slot_row, _I32, (R,)))


def adapter_rows(ad, offsets, sorted_slot, slot_row, x, base, y, ws, stream=None):
    """y = base + scale (x A^T) B^T, each row by its adapter; base may be y or
    None, ws of adapter_workspace_bytes bytes.  The order is permute's of the
    rows' adapters (top_k 1); slot_row may be None where base is y."""
    R, _ = _rows("x", x, ad.k)
    dev, code = _dev("x", x), _real("y", y)
    shape = (R, ad.n)
    _check(lib().moe_adapter_rows(
        R, *_adapter_args(ad, dev, R, offsets, sorted_slot, slot_row),
        _arg(dev, "x", x, _BF16, (R, ad.k)), _arg(dev, "base", base, (y.dtype,), shape),
        _arg(dev, "y", y, (y.dtype,), shape), code, _arg(dev, "ws", ws, (ws.dtype,), ws.shape),
        ws.numel() * ws.element_size(), _stream_on(dev, stream)))


def adapter_backward(ad, offsets, sorted_slot, slot_row, x, dy, dx_base, dx, da, db, ws,
                     accumulate=False, stream=None):
    """adapter_rows' gradients: dx = dx_base + .., and da, db fp32 (added to what
    they hold with accumulate).  dx, or da and db, may be None; ws of
    adapter_backward_bytes bytes."""
    R, _ = _rows("dy", dy, ad.n)
    dev = _dev("dy", dy)
    wide = (dx.dtype,) if dx is not None else _F32
    _check(lib().moe_adapter_backward(
        R, *_adapter_args(ad, dev, R, offsets, sorted_slot, slot_row),
        _arg(dev, "x", x, _BF16, (R, ad.k)), _arg(dev, "dy", dy, _BF16, (R, ad.n)),
        _arg(dev, "dx_base", dx_base, wide, (R, ad.k)), _arg(dev, "dx", dx, wide, (R, ad.k)),
        _real("dx", dx) if dx is not None else FP32,
        _arg(dev, "da", da, _F32, (ad.count, ad.rank, ad.k)),
        _arg(dev, "db", db, _F32, (ad.count, ad.n, ad.rank)), int(accumulate),
        _arg(dev, "ws", ws, (ws.dtype,), ws.shape), ws.numel() * ws.element_size(),
        _stream_on(dev, stream)))


class MoEBuffers:
    """Device tensors of one workload plus the workspace, for callers that
    want the whole forward with one call (tests, benchmark, smoke)."""

    def __init__(self, d: Dims, o: Optional[Opts], device="cuda"):
        T, k, H = d.tokens, d.top_k, d.hidden
        self.d, self.o = d, o
        self.y = torch.empty((T, H), dtype=torch.float32, device=device)
        self.topk_ids = torch.empty((T, k), dtype=torch.int32, device=device)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, device=device)
        self.counts = torch.empty((d.local_count,), dtype=torch.int32, device=device)
        nbytes = workspace_bytes(d, o if o is not None else opts())
        self.ws = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device=device)

    def run(self, x, w_router, bias, w_gate, w_up, w_down, shared_gate=None, shared_up=None,
            shared_down=None, stream=None):
        forward(self.d, self.o, x, w_router, bias, w_gate, w_up, w_down, shared_gate,
                shared_up, shared_down, self.y, self.topk_ids, self.topk_w, self.counts,
                self.ws, stream)
        return self.y
