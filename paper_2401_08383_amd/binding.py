"""Thin ctypes binding of ``libexflow_moe.so`` (the C ABI declared in ``include/exflow_moe.h``).

Argument marshalling only: every step of the path runs in the library's HIP kernels.  PyTorch
is used for device memory (``torch.empty(..., device="cuda")``, ``.data_ptr()``) and for the
current HIP stream.  There is no CPU fallback: if the library is missing, loading fails.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch
from torch.autograd import forward_ad as _forward_ad

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libexflow_moe.so")

EXF_OK = 0
EXF_ERR_NULL_PTR = -1
EXF_ERR_BAD_SHAPE = -2
EXF_ERR_BAD_DTYPE = -3
EXF_ERR_WORKSPACE_TOO_SMALL = -4
EXF_ERR_HIP = -5
EXF_ERR_NOT_IMPLEMENTED = -6
EXF_ERR_MISALIGNED = -7
EXF_F32 = 0
EXF_BF16 = 1
EXF_ACT_GELU_ERF = 0
EXF_ACT_GELU_TANH = 1
EXF_SCORE_SOFTMAX = 0
EXF_SCORE_SIGMOID = 1
EXF_MAX_TOPK = 2
EXF_MX4_BLOCK = 32
EXF_MX4_INLINE_ROWS = 8

_vp, _i, _i64, _sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t

# name -> (restype, argtypes); mirrors include/exflow_moe.h one to one
SIGNATURES = {
    "exf_version": (_i, []),
    "exf_last_error": (ctypes.c_char_p, []),
    "exf_check_placement": (_i, [_vp, _i, _i, _i]),
    "exf_comm_volume": (_i, [_i, _i64, _i, ctypes.c_double, ctypes.c_double, _vp]),
    "exf_transfer_ratios": (_i, [_vp, _vp, _i, _i64, _vp, _vp]),
    "moe_gate_topk": (_i, [_vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "moe_topk_from_logits": (_i, [_vp, _i64, _i, _i, _i, _vp, _vp, _vp]),
    "moe_dispatch_workspace_bytes": (_sz, [_i64, _i, _i]),
    "moe_dispatch": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "moe_dispatch_static": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "moe_expert_ffn_workspace_bytes": (_sz, [_i64, _i, _i, _i, _i]),
    "moe_expert_ffn": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp, _sz, _vp]),
    "moe_expert_ffn_fused_workspace_bytes": (_sz, [_i64, _i, _i, _i, _i, _i]),
    "moe_expert_ffn_fused": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _i, _vp, _vp, _sz, _vp]),
    "moe_combine": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _vp, _vp]),
    "moe_grouped_product": (_i, [_vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp, _vp]),
    "moe_grouped_product_dx": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp, _vp]),
    "moe_grouped_product_dw_workspace_bytes": (_sz, [_i64, _i, _i, _i, _i]),
    "moe_grouped_product_dw": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "mx4_scale_bytes": (_sz, [_i64, _i]),
    "mx4_quantize": (_i, [_vp, _i64, _i, _i, _vp, _vp, _vp]),
    "mx4_dequantize": (_i, [_vp, _vp, _i64, _i, _i, _vp, _vp]),
    "moe_grouped_product_mx4_workspace_bytes": (_sz, [_i64, _i, _i]),
    "moe_grouped_product_mx4": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp, _vp, _sz, _vp]),
    "moe_route": (_i, [_vp, _vp, _i64, _i, _i, _i, _i, _i, _i, _i, ctypes.c_float, _i, _vp, _vp, _vp, _vp]),
    "moe_route_backward": (_i, [_vp, _vp, _vp, _vp, _i64, _i64, _i, _i, _i, _i, ctypes.c_float, _i, _vp, _vp]),
    "moe_dispatch_topk": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "moe_combine_topk": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _vp, _vp]),
    "moe_combine_backward": (_i, [_vp, _vp, _vp, _vp, _i64, _i, _i, _i, _vp, _vp, _vp]),
    "q4_quantize": (_i, [_vp, _i64, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "q4_dequantize": (_i, [_vp, _vp, _vp, _i64, _i, _i, _i, _vp, _vp]),
    "moe_grouped_product_q4": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _i, _vp, _vp]),
    "moe_layer_forward": (_i, [_vp, _vp]),
    "affinity_histogram_workspace_bytes": (_sz, [_i, _i64, _i]),
    "affinity_histogram": (_i, [_vp, _i, _i64, _i, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "affinity_statistics_workspace_bytes": (_sz, [_i, _i64, _i]),
    "affinity_statistics": (_i, [_vp, _vp, _i, _i64, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "placement_locality_workspace_bytes": (_sz, [_i, _i64]),
    "placement_locality": (_i, [_vp, _vp, _i, _i64, _i, _i, _vp, _vp, _sz, _vp]),
    "affinity_multihop_workspace_bytes": (_sz, [_i, _i64, _i]),
    "affinity_multihop": (_i, [_vp, _i, _i64, _i, _vp, _vp, _vp, _sz, _vp]),
    "routing_transfers_workspace_bytes": (_sz, [_i, _i64]),
    "routing_transfers": (_i, [_vp, _vp, _vp, _i, _i64, _i, _i, _vp, _vp, _vp, _sz, _vp]),
    "placement_locality_from_counts": (_i, [_vp, _vp, _i, _i, _i, _vp, _vp]),
    "exf_placement_search": (_i, [_vp, _i, _i, _i, _i, _i, ctypes.c_uint64, _vp]),
    "exf_probe_copy": (_i, [_vp, _vp, _sz, _vp]),
    "exf_probe_mfma": (_i, [_i, _i, _vp, _vp]),
    "exf_probe_gemm_loop_bytes": (_sz, []),
    "exf_probe_gemm_loop": (_i, [_vp, _sz, _i, _vp, _vp]),
    "exf_probe_ffn_timeline": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i, _i, _i, _i, _vp, _vp, _sz, _vp, _i, _vp]),
}

class MoELayerDesc(ctypes.Structure):
    """exf_moe_layer of include/exflow_moe.h."""
    _fields_ = ([(n, _vp) for n in ("x", "w_gate", "w1", "w2", "forced_idx", "expert_map")] + [("T", _i64)]
                + [(n, _i) for n in ("d", "f", "E", "E_local", "k", "renormalize", "act", "dt", "fused", "reserved")]
                + [(n, _vp) for n in ("topk_idx", "topk_w", "x_sorted", "src_of_sorted", "sorted_of_src", "expert_counts", "expert_offsets",
                                      "y_sorted", "out", "dispatch_workspace")]
                + [("dispatch_workspace_bytes", _sz), ("ffn_workspace", _vp), ("ffn_workspace_bytes", _sz)])


_lib = None


class ExflowError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"exflow_moe error {code}: {message}")
        self.code = code


def lib() -> ctypes.CDLL:
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2401_08383_amd.build` (there is no fallback path)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def last_error() -> str:
    return lib().exf_last_error().decode()


def _check(rc: int) -> None:
    if rc != EXF_OK:
        raise ExflowError(rc, last_error())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream() -> int:
    # (the raw handle; a Stream object costs a microsecond more)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream_on(dev) -> int:
    """The same for tensors on device number `dev`, which has to be the current one: a kernel launched elsewhere would not reach them."""
    current = torch._C._cuda_getDevice()
    if dev != current:
        _bad(f"the arguments are on device {dev}, the current one is {current} (torch.cuda.device chooses it)")
    return torch._C._cuda_getCurrentRawStream(current)


def dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return EXF_F32
    if t.dtype == torch.bfloat16:
        return EXF_BF16
    raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {t.dtype}")


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ----------------------------------------------------------------------------------------------
def moe_gate_topk(x, w_gate, k, renormalize=False, want_logits=False):
    """-> (topk_idx int32 [T,k], topk_w fp32 [T,k], logits fp32 [T,E] or None)."""
    T, d = x.shape
    E = w_gate.shape[0]
    assert w_gate.shape[1] == d and x.is_contiguous() and w_gate.is_contiguous() and x.dtype == w_gate.dtype
    idx = torch.empty((T, k), dtype=torch.int32, device=x.device)
    w = torch.empty((T, k), dtype=torch.float32, device=x.device)
    logits = torch.empty((T, E), dtype=torch.float32, device=x.device) if want_logits else None
    _check(lib().moe_gate_topk(_ptr(x), _ptr(w_gate), T, d, E, k, int(bool(renormalize)), dtype_code(x), _ptr(logits),
                               _ptr(idx), _ptr(w), _stream()))
    return idx, w, logits


def moe_topk_from_logits(logits, k, renormalize=False):
    T, E = logits.shape
    assert logits.dtype == torch.float32 and logits.is_contiguous()
    idx = torch.empty((T, k), dtype=torch.int32, device=logits.device)
    w = torch.empty((T, k), dtype=torch.float32, device=logits.device)
    _check(lib().moe_topk_from_logits(_ptr(logits), T, E, k, int(bool(renormalize)), _ptr(idx), _ptr(w), _stream()))
    return idx, w


class DispatchResult:
    __slots__ = ("x_sorted", "src_of_sorted", "sorted_of_src", "expert_counts", "expert_offsets")

    def __init__(self, x_sorted, src_of_sorted, sorted_of_src, expert_counts, expert_offsets):
        self.x_sorted = x_sorted
        self.src_of_sorted = src_of_sorted
        self.sorted_of_src = sorted_of_src
        self.expert_counts = expert_counts
        self.expert_offsets = expert_offsets


def moe_dispatch(x, topk_idx, E, E_local=None, expert_map=None, out=None, workspace=None, gather=True):
    """Stable dispatch of the assignments (up to 16 a token); returns a DispatchResult of device tensors.

    Entries of ``src_of_sorted`` / rows of ``x_sorted`` at or beyond ``expert_offsets[E_local]``
    are left untouched by the library.  ``out`` may carry a previous DispatchResult to reuse.
    """
    T, k = topk_idx.shape
    d = x.shape[1]
    E_local = E if E_local is None else E_local
    A = T * k
    dev = topk_idx.device
    assert topk_idx.dtype == torch.int32 and topk_idx.is_contiguous() and x.is_contiguous()
    given = out is not None
    if not given:
        out = DispatchResult(
            torch.empty((A, d), dtype=x.dtype, device=dev) if gather else None,
            torch.empty(A, dtype=torch.int32, device=dev),
            torch.empty(A, dtype=torch.int32, device=dev),
            torch.empty(E_local, dtype=torch.int32, device=dev),
            torch.empty(E_local + 1, dtype=torch.int32, device=dev),
        )
    if workspace is None:
        workspace = _workspace(lib().moe_dispatch_workspace_bytes(T, k, E_local), dev)
    stream = _dispatch_fits(x, topk_idx, T, k, expert_map, E, E_local, out, given)
    workspace, size = _bytes_of(workspace, topk_idx.get_device())
    call = lib().moe_dispatch if k <= EXF_MAX_TOPK else lib().moe_dispatch_topk
    rc = call(x.data_ptr(), topk_idx.data_ptr(), _ptr(expert_map), T, d, k, E, E_local, dtype_code(x), _ptr(out.x_sorted), out.src_of_sorted.data_ptr(),
              out.sorted_of_src.data_ptr(), out.expert_counts.data_ptr(), out.expert_offsets.data_ptr(), workspace, size, stream)
    if rc:
        _check(rc)
    return out


def _dispatch_fits(x, topk_idx, T, k, expert_map, E, E_local, out, given):
    """Checks of what the library cannot see of a dispatch (`given`: its results are the caller's); -> the stream."""
    dev = topk_idx.get_device()
    d, rows = x.shape[1], out.x_sorted
    if rows is not None and x.requires_grad:
        _untracked("moe_dispatch", "moe_dispatch_backward")
    if rows is not None and _forward_ad._current_level >= 0:
        _no_tangents("moe_dispatch", x)
    # (one and two assignments a token have always been taken with the buffers of a larger call)
    fits = _expect if k > EXF_MAX_TOPK else _room
    if rows is not None and not (x.numel() == T * d and x.get_device() == dev):
        fits("x", x, (T, d), x.dtype, dev)
    if expert_map is not None:
        fits("expert_map", expert_map, (E,), _INT32, dev)
    if given:
        A, src, at, counts, offsets = T * k, out.src_of_sorted, out.sorted_of_src, out.expert_counts, out.expert_offsets
        if rows is not None and not (rows.numel() == A * d and rows.dtype is x.dtype and rows.is_contiguous() and rows.get_device() == dev):
            fits("out.x_sorted", rows, (A, d), x.dtype, dev)
        if not (src.numel() == at.numel() == A and counts.numel() == E_local and offsets.numel() == E_local + 1 and src.dtype is at.dtype is counts.dtype is offsets.dtype is _INT32
                and src.is_contiguous() and at.is_contiguous() and counts.is_contiguous() and offsets.is_contiguous()
                and src.get_device() == at.get_device() == counts.get_device() == offsets.get_device() == dev):
            fits("out.src_of_sorted", src, (A,), _INT32, dev)
            fits("out.sorted_of_src", at, (A,), _INT32, dev)
            fits("out.expert_counts", counts, (E_local,), _INT32, dev)
            fits("out.expert_offsets", offsets, (E_local + 1,), _INT32, dev)
    if dev < 0:
        _on_host()
    return _stream_on(dev)


def moe_dispatch_backward(dx_sorted, sorted_of_src, k, out=None):
    """Gradient of moe_dispatch's rows: dx[t] = sum of the rows of dx_sorted [T*k,d] that token t's k assignments went to."""
    return _combine_rows("moe_dispatch_backward", dx_sorted, sorted_of_src, None, k, out)


def moe_dispatch_static(x, topk_idx, E, out, E_local=None, expert_map=None):
    """moe_dispatch without a workspace and without any allocation: every output tensor comes from the
    caller (``out``: a DispatchResult; ``x_sorted`` None skips the row gather)."""
    T, k = topk_idx.shape
    d = x.shape[1]
    E_local = E if E_local is None else E_local
    assert topk_idx.dtype == torch.int32 and topk_idx.is_contiguous() and x.is_contiguous()
    _check(lib().moe_dispatch_static(_ptr(x), _ptr(topk_idx), _ptr(expert_map), T, d, k, E, E_local, dtype_code(x),
                                     _ptr(out.x_sorted), _ptr(out.src_of_sorted), _ptr(out.sorted_of_src),
                                     _ptr(out.expert_counts), _ptr(out.expert_offsets), _stream()))
    return out


def moe_expert_ffn(x_sorted, expert_offsets, w1, w2, b1=None, b2=None, act=EXF_ACT_GELU_ERF, out=None, workspace=None):
    A, d = x_sorted.shape
    E_local, f, d2 = w1.shape
    assert d2 == d and tuple(w2.shape) == (E_local, d, f) and expert_offsets.numel() == E_local + 1
    assert x_sorted.is_contiguous() and w1.is_contiguous() and w2.is_contiguous()
    assert expert_offsets.dtype == torch.int32
    dt = dtype_code(x_sorted)
    if out is None:
        out = torch.empty((A, d), dtype=x_sorted.dtype, device=x_sorted.device)
    if workspace is None:
        workspace = _workspace(lib().moe_expert_ffn_workspace_bytes(A, d, f, E_local, dt), x_sorted.device)
    _check(lib().moe_expert_ffn(_ptr(x_sorted), _ptr(expert_offsets), _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2), A, d, f,
                                E_local, act, dt, _ptr(out), _ptr(workspace), workspace.numel(), _stream()))
    return out


def moe_expert_ffn_fused(x, src_of_sorted, sorted_of_src, topk_w, expert_offsets, w1, w2, b1=None, b2=None,
                         act=EXF_ACT_GELU_ERF, out=None, workspace=None):
    """Expert FFN + combine straight from / to the unsorted token rows (bf16)."""
    T, d = x.shape
    k = topk_w.shape[1]
    E_local, f, d2 = w1.shape
    assert d2 == d and tuple(w2.shape) == (E_local, d, f) and expert_offsets.numel() == E_local + 1
    assert x.is_contiguous() and w1.is_contiguous() and w2.is_contiguous() and topk_w.is_contiguous()
    assert tuple(topk_w.shape) == (T, k) and topk_w.dtype == torch.float32
    assert src_of_sorted.numel() == T * k and sorted_of_src.numel() == T * k
    assert src_of_sorted.dtype == torch.int32 and sorted_of_src.dtype == torch.int32 and expert_offsets.dtype == torch.int32
    dt = dtype_code(x)
    if out is None:
        out = torch.empty((T, d), dtype=x.dtype, device=x.device)
    if workspace is None:
        workspace = _workspace(lib().moe_expert_ffn_fused_workspace_bytes(T, k, d, f, E_local, dt), x.device)
    _check(lib().moe_expert_ffn_fused(_ptr(x), _ptr(src_of_sorted), _ptr(sorted_of_src), _ptr(topk_w), _ptr(expert_offsets),
                                      _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2), T, k, d, f, E_local, act, dt, _ptr(out),
                                      _ptr(workspace), workspace.numel(), _stream()))
    return out


def moe_combine(y_sorted, sorted_of_src, topk_w, out=None):
    """out[t] = sum of token t's rows of y_sorted, each by its weight; topk_w [T,k], k up to 16."""
    T, k = topk_w.shape
    if k > EXF_MAX_TOPK:
        return _combine_rows("moe_combine", y_sorted, sorted_of_src, topk_w, k, out)
    if y_sorted.requires_grad or topk_w.requires_grad:
        _untracked("moe_combine", "moe_combine_backward")
    if _forward_ad._current_level >= 0:
        _no_tangents("moe_combine", y_sorted, topk_w)
    if len(y_sorted.shape) != 2:
        _bad(f"sorted rows are [T*k,d], got {tuple(y_sorted.shape)}")
    d, dt, dev = y_sorted.shape[1], y_sorted.dtype, y_sorted.get_device()
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    if sorted_of_src.numel() != T * k:
        _bad(f"positions of {T} x {k} assignments expected, got {tuple(sorted_of_src.shape)}")
    if out is None:
        out = _rows(T, d, dt, y_sorted.device)
    if not (y_sorted.shape[0] == T * k and out.shape == (T, d) and out.dtype is dt and sorted_of_src.dtype is _INT32 and topk_w.dtype is _FLOAT and y_sorted.is_contiguous()
            and out.is_contiguous() and sorted_of_src.is_contiguous() and topk_w.is_contiguous()
            and out.get_device() == sorted_of_src.get_device() == topk_w.get_device() == dev):
        _room("the sorted rows", y_sorted, (T * k, d), dt, dev)
        _room("sorted_of_src", sorted_of_src, (T * k,), _INT32, dev)
        _room("topk_w", topk_w, (T, k), _FLOAT, dev)
        _room("out", out, (T, d), dt, dev)
    if dev < 0:
        _on_host()
    rc = lib().moe_combine(y_sorted.data_ptr(), sorted_of_src.data_ptr(), topk_w.data_ptr(), T, d, k, code, out.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)
    return out


def _rows(T, width, dtype, device):
    """A new dense [T, width] (torch.empty takes a microsecond more)."""
    return torch.empty_strided((T, width), (width, 1), dtype=dtype, device=device)


def _combine_rows(name, y_sorted, sorted_of_src, topk_w, k, out):
    if y_sorted.requires_grad or topk_w is not None and topk_w.requires_grad:
        _untracked(name, "moe_combine_backward" if name == "moe_combine" else "moe_dispatch")
    if _forward_ad._current_level >= 0:
        _no_tangents(name, y_sorted, topk_w)
    T, A, d, dt, code, dev = _assigned(y_sorted, sorted_of_src, k)
    if out is None:
        out = _rows(T, d, dt, y_sorted.device)
    if not (out.shape == (T, d) and out.dtype is dt and out.is_contiguous() and out.get_device() == dev):
        _expect("out", out, (T, d), dt, dev)
    if topk_w is not None:
        topk_w = _expect("topk_w", topk_w, (T, k), _FLOAT, dev).data_ptr()
    if dev < 0:
        _on_host()
    rc = lib().moe_combine_topk(y_sorted.data_ptr(), sorted_of_src.data_ptr(), topk_w, T, d, k, code, out.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)
    return out


def _assigned(rows, sorted_of_src, k):
    """(T, T*k, d, type, its code, device number) of sorted rows and the positions of T tokens' k assignments."""
    shape, at = rows.shape, sorted_of_src.shape
    if len(shape) != 2 or len(at) not in (1, 2):
        _bad(f"sorted rows are [T*k,d] and positions [T*k], got {tuple(shape)} and {tuple(at)}")
    A, dev, dt = sorted_of_src.numel(), rows.get_device(), rows.dtype
    if k < 1 or A % k or len(at) == 2 and at[1] != k:
        _bad(f"positions of k = {k} assignments a token expected, got {tuple(at)}")
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    if not (sorted_of_src.dtype is _INT32 and sorted_of_src.is_contiguous() and sorted_of_src.get_device() == dev):
        _expect("sorted_of_src", sorted_of_src, at, _INT32, dev)
    if not (shape[0] == A and rows.is_contiguous()):
        _expect("the sorted rows", rows, (A, shape[1]), dt, dev)
    return A // k, A, shape[1], dt, code, dev


def moe_combine_backward(dout, y_sorted, sorted_of_src, topk_w, want_rows=True, want_weights=True, out=None, out_weights=None):
    """Gradients of moe_combine: (dy_sorted [T*k,d] or None, dtopk_w [T,k] or None).  Rows of dy_sorted that no assignment has are left as they were
    (``out``), or zero: without ``out`` all rows are cleared first (8192 x 8 of 4 KiB 152 us instead of 110)."""
    if dout.requires_grad or y_sorted.requires_grad or topk_w.requires_grad:
        _untracked("moe_combine_backward", "none: there is no second derivative")
    if _forward_ad._current_level >= 0:
        _no_tangents("moe_combine_backward", dout, y_sorted, topk_w)
    weights = topk_w.shape
    if len(weights) != 2:
        _bad(f"topk_w is [T,k], got {tuple(weights)}")
    k = weights[1]
    T, A, d, dt, code, dev = _assigned(y_sorted, sorted_of_src, k)
    if not (dout.shape == (T, d) and weights[0] == T and dout.dtype is dt and topk_w.dtype is _FLOAT and dout.is_contiguous() and topk_w.is_contiguous()
            and dout.get_device() == topk_w.get_device() == dev):
        _expect("dout", dout, (T, d), dt, dev)
        _expect("topk_w", topk_w, (T, k), _FLOAT, dev)
    if out is not None:
        _expect("out", out, (A, d), dt, dev)
    elif want_rows:
        out = torch.zeros((A, d), dtype=dt, device=dout.device)
    if out_weights is not None:
        _expect("out_weights", out_weights, (T, k), _FLOAT, dev)
    elif want_weights:
        out_weights = torch.empty_like(topk_w)
    if dev < 0:
        _on_host()
    rc = lib().moe_combine_backward(dout.data_ptr(), y_sorted.data_ptr(), sorted_of_src.data_ptr(), topk_w.data_ptr(), T, d, k, code, _ptr(out), _ptr(out_weights),
                                    _stream_on(dev))
    if rc:
        _check(rc)
    return out, out_weights


def moe_route(logits, k, bias=None, score=EXF_SCORE_SOFTMAX, renormalize=False, scale=1.0, groups=1, top_groups=None, group_best=1, want_scores=False, out=None):
    """Experts of every token from the gate's logits [T,E], E up to 512: (topk_idx int32 [T,k], topk_w fp32 [T,k], scores fp32 [T,E] or None).

    The k (up to 16) largest of the scores plus ``bias`` (fp32 [E]) are chosen, of the ``top_groups`` best of ``groups`` groups of experts, a group being as
    good as the sum of its ``group_best`` best; the weights are the scores without the bias, renormalised to a sum of one (k > 1), times ``scale``.
    ``out``: (topk_idx, topk_w) to write to."""
    if logits.requires_grad:
        _untracked("moe_route", "moe_route_backward")
    if _forward_ad._current_level >= 0:
        _no_tangents("moe_route", logits)
    shape, dt, dev = logits.shape, logits.dtype, logits.get_device()
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    if len(shape) != 2 or not logits.is_contiguous():
        _bad(f"logits: contiguous [T,E] expected, got {tuple(shape)}")
    T, E = shape
    if bias is not None:
        bias = _expect("bias", bias, (E,), _FLOAT, dev).data_ptr()
    if dev < 0:
        _on_host()
    if out is None:
        if k < 1:
            _bad(f"k = {k}")
        device = logits.device
        idx, w = _rows(T, k, _INT32, device), _rows(T, k, _FLOAT, device)
    else:
        idx, w = out
        _expect("topk_idx", idx, (T, k), _INT32, dev)
        _expect("topk_w", w, (T, k), _FLOAT, dev)
    scores = _rows(T, E, _FLOAT, logits.device) if want_scores else None
    rc = lib().moe_route(logits.data_ptr(), bias, T, E, k, score, groups, groups if top_groups is None else top_groups, group_best, 1 if renormalize else 0, scale, code,
                         idx.data_ptr(), w.data_ptr(), _ptr(scores), _stream_on(dev))
    if rc:
        _check(rc)
    return idx, w, scores


def moe_route_backward(dtopk_w, logits, topk_idx, score=EXF_SCORE_SOFTMAX, renormalize=False, scale=1.0, dscores=None, out=None):
    """Gradient of moe_route's logits, of their type, from that of the weights, fp32 [T,k], and of the scores, fp32 [T,E] or one row [E] for all tokens."""
    if dtopk_w.requires_grad or logits.requires_grad or dscores is not None and dscores.requires_grad:
        _untracked("moe_route_backward", "none: there is no second derivative")
    if _forward_ad._current_level >= 0:
        _no_tangents("moe_route_backward", dtopk_w, logits, dscores)
    shape, dt, dev = logits.shape, logits.dtype, logits.get_device()
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    slots = topk_idx.shape
    if len(shape) != 2 or len(slots) != 2 or not logits.is_contiguous():
        _bad(f"logits: contiguous [T,E] expected, topk_idx [T,k], got {tuple(shape)} and {tuple(slots)}")
    T, E = shape
    k, stride, at = slots[1], 0, None
    if not (slots[0] == T and dtopk_w.shape == slots and topk_idx.dtype is _INT32 and dtopk_w.dtype is _FLOAT and topk_idx.is_contiguous()
            and dtopk_w.is_contiguous() and topk_idx.get_device() == dtopk_w.get_device() == dev):
        _expect("topk_idx", topk_idx, (T, k), _INT32, dev)
        _expect("dtopk_w", dtopk_w, (T, k), _FLOAT, dev)
    if dscores is not None:
        stride = E if len(dscores.shape) == 2 else 0
        at = _expect("dscores", dscores, (T, E) if stride else (E,), _FLOAT, dev).data_ptr()
    out = torch.empty_like(logits) if out is None else _expect("out", out, shape, dt, dev)
    if dev < 0:
        _on_host()
    rc = lib().moe_route_backward(dtopk_w.data_ptr(), logits.data_ptr(), topk_idx.data_ptr(), at, stride, T, E, k, score, 1 if renormalize else 0, scale, code,
                                  out.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)
    return out


_CODES = {torch.float32: EXF_F32, torch.bfloat16: EXF_BF16}
_FLOAT = torch.float32


def _bad(message: str):
    raise ExflowError(EXF_ERR_BAD_SHAPE, message)


def _expect(name, t, shape, dtype, dev):
    """`t` is a dense tensor of this shape and type on device number `dev` (-1: the host, which the calls refuse by themselves)."""
    if t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.get_device() == dev:
        return t
    if t.shape != shape:
        _bad(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"{name} is {t.dtype}, expected {dtype}")
    _bad(f"{name} must be contiguous and on device {dev}")


def _room(name, t, shape, dtype, dev):
    """As _expect(), of a tensor that may be longer."""
    if t.numel() < math.prod(shape):
        _bad(f"{name} has shape {tuple(t.shape)}, {tuple(shape)} needed")
    return _expect(name, t, t.shape, dtype, dev)


def _on_host():
    """The arguments' device number is -1: no kernel can reach them."""
    _bad("the arguments must be on a GPU, they are on the host")


def _bytes_of(workspace, dev):
    """(address, size) of a workspace, of any type."""
    if not workspace.is_contiguous() or workspace.get_device() != dev:
        _bad(f"workspace must be contiguous and on device {dev}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _untracked(name, backward="moe_grouped_product_dx and moe_grouped_product_dw"):
    """An argument requires a gradient, which a result of these calls does not carry on."""
    if torch.is_grad_enabled():
        raise ExflowError(EXF_ERR_NOT_IMPLEMENTED, f"{name} records no autograd history and an argument requires a gradient: call it under torch.no_grad(), or in the "
                                                   f"forward of a torch.autograd.Function whose backward calls {backward}")


def _no_tangents(name, *tensors):
    """Raises for a dual tensor of forward-mode differentiation, whose tangent a result would not have (in the forward of a torch.autograd.Function there are none)."""
    for t in tensors:
        if t is not None and _forward_ad.unpack_dual(t).tangent is not None:
            raise ExflowError(EXF_ERR_NOT_IMPLEMENTED, f"{name} carries no tangents on and an argument is a dual tensor: call it in the forward of a torch.autograd.Function that has a jvp")


_INT32, _UINT8 = torch.int32, torch.uint8


def _fits(rows, width, offsets, E, w, out, out_shape, dt, dev):
    """The rows [A,width], offsets, weights and result of a product are dense, of these shapes and types and on device number `dev`, a GPU (one
    expression: a call of a few microseconds spends a third of them on its checks)."""
    return (rows.shape[1] == width and offsets.shape == (E + 1,) and out.shape == out_shape and w.dtype is dt and out.dtype is dt and offsets.dtype is _INT32
            and rows.is_contiguous() and w.is_contiguous() and out.is_contiguous() and offsets.is_contiguous()
            and w.get_device() == out.get_device() == offsets.get_device() == dev >= 0)


def _grouped(rows, w_shape):
    """(E_local, n, k, A, type, its code, device number) of a product of `rows` [A,*] with weights of this shape."""
    if len(w_shape) != 3 or len(rows.shape) != 2:
        _bad(f"rows are [A,*] and weights [E_local,n,k], got {tuple(rows.shape)} and {tuple(w_shape)}")
    dt = rows.dtype
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    return (*w_shape, rows.shape[0], dt, code, rows.get_device())


def _misfit(rows, rows_shape, offsets, E, w, out, out_shape, dt, dev):
    """Raises for what _fits() found."""
    _expect("the rows", rows, rows_shape, dt, dev)
    _expect("expert_offsets", offsets, (E + 1,), _INT32, dev)
    _expect("w", w, w.shape, dt, dev)
    _expect("out", out, out_shape, dt, dev)
    _on_host()


def moe_grouped_product(x_sorted, expert_offsets, w, bias=None, out=None):
    """y[s] = x_sorted[s] W_e^T (+ bias[e]) for the rows of every expert; w [E_local,n,k].

    No autograd history is recorded: in grad mode an argument that requires a gradient is refused (here and in the calls below)."""
    if x_sorted.requires_grad or w.requires_grad or bias is not None and bias.requires_grad:
        _untracked("moe_grouped_product")
    E, n, k, A, dt, code, dev = _grouped(x_sorted, w.shape)
    if out is None:
        out = torch.empty((A, n), dtype=dt, device=x_sorted.device)
    if bias is not None:
        bias = _expect("bias", bias, (E, n), dt, dev).data_ptr()
    if not _fits(x_sorted, k, expert_offsets, E, w, out, (A, n), dt, dev):
        _misfit(x_sorted, (A, k), expert_offsets, E, w, out, (A, n), dt, dev)
    rc = lib().moe_grouped_product(x_sorted.data_ptr(), expert_offsets.data_ptr(), w.data_ptr(), bias, A, n, k, E, code, out.data_ptr(), _stream())
    if rc:
        _check(rc)
    return out


def moe_grouped_product_dx(dy_sorted, expert_offsets, w, out=None):
    """Gradient of moe_grouped_product's rows: dx[s] = dy_sorted[s] W_e; w [E_local,n,k]."""
    if dy_sorted.requires_grad or w.requires_grad:
        _untracked("moe_grouped_product_dx")
    E, n, k, A, dt, code, dev = _grouped(dy_sorted, w.shape)
    if out is None:
        out = torch.empty((A, k), dtype=dt, device=dy_sorted.device)
    if not _fits(dy_sorted, n, expert_offsets, E, w, out, (A, k), dt, dev):
        _misfit(dy_sorted, (A, n), expert_offsets, E, w, out, (A, k), dt, dev)
    rc = lib().moe_grouped_product_dx(dy_sorted.data_ptr(), expert_offsets.data_ptr(), w.data_ptr(), A, n, k, E, code, out.data_ptr(), _stream())
    if rc:
        _check(rc)
    return out


def moe_grouped_product_dw(dy_sorted, x_sorted, expert_offsets, want_bias=False, grad_dtype=None, workspace=None, out=None, out_bias=None):
    """Gradients of moe_grouped_product's weights and bias: (dw [E_local,n,k], db [E_local,n] or None), both of `grad_dtype` (that of
    ``out``, or the rows')."""
    if dy_sorted.requires_grad or x_sorted.requires_grad:
        _untracked("moe_grouped_product_dw")
    if len(dy_sorted.shape) != 2 or len(x_sorted.shape) != 2 or len(expert_offsets.shape) != 1 or expert_offsets.shape[0] < 2:
        _bad("rows are [A,n] and [A,k], expert_offsets [E_local+1]")
    E, n, k, A, dt, code, dev = _grouped(x_sorted, (expert_offsets.shape[0] - 1, dy_sorted.shape[1], x_sorted.shape[1]))
    _expect("x_sorted", x_sorted, (A, k), dt, dev)
    _expect("dy_sorted", dy_sorted, (A, n), dt, dev)
    _expect("expert_offsets", expert_offsets, (E + 1,), torch.int32, dev)
    if grad_dtype is None:
        grad_dtype = dt if out is None else out.dtype
    if grad_dtype not in _CODES:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {grad_dtype}")
    out = torch.empty((E, n, k), dtype=grad_dtype, device=x_sorted.device) if out is None else _expect("out", out, (E, n, k), grad_dtype, dev)
    if out_bias is not None:
        _expect("out_bias", out_bias, (E, n), grad_dtype, dev)
    elif want_bias:
        out_bias = torch.empty((E, n), dtype=grad_dtype, device=x_sorted.device)
    if dev < 0:
        _on_host()
    if workspace is None:
        need = lib().moe_grouped_product_dw_workspace_bytes(A, n, k, E, code)
        workspace = _workspace(need, x_sorted.device) if need else None
    workspace, size = (None, 0) if workspace is None else _bytes_of(workspace, dev)
    rc = lib().moe_grouped_product_dw(dy_sorted.data_ptr(), x_sorted.data_ptr(), expert_offsets.data_ptr(), A, n, k, E, code, _CODES[grad_dtype], out.data_ptr(),
                                      _ptr(out_bias), workspace, size, _stream())
    if rc:
        _check(rc)
    return out, out_bias


class Mx4:
    """Rows in microscaled 4-bit floating point: ``q`` uint8 [..., k/2] and ``scale`` uint8 [ceil(k/256), rows, 8] (see mx4_quantize).

    Experts a .. b-1 of weights [E,n,k] are ``Mx4(m.q[a:b], m.scale[:, a * n:b * n].contiguous())``."""
    __slots__ = ("q", "scale")

    def __init__(self, q, scale):
        self.q, self.scale = q, scale

    @property
    def shape(self):
        s = self.q.shape
        return (*s[:-1], *(2 * k for k in s[-1:]))

    @property
    def rows(self):
        return self.scale.shape[1]


def _expect_mx4(name, m, shape, dev):
    """`m` holds this shape on device number `dev`; -> its rows."""
    q, scale = m.q, m.scale
    if not len(shape):
        _bad(f"{name} has no rows")
    rows, k = q.numel() * 2 // max(shape[-1], 1), shape[-1]
    if (q.shape == (*shape[:-1], k // 2) and scale.shape == ((k + 255) // 256, rows, 8) and q.dtype is _UINT8 and scale.dtype is _UINT8 and q.is_contiguous()
            and scale.is_contiguous() and q.get_device() == scale.get_device() == dev):
        return rows
    _expect(f"{name}.q", q, (*shape[:-1], k // 2), _UINT8, dev)
    _expect(f"{name}.scale", scale, ((k + 255) // 256, rows, 8), _UINT8, dev)
    return rows


def mx4_quantize(x, out=None):
    """Rows x [..., k] (k a multiple of 32) -> Mx4."""
    shape, code = x.shape, _CODES.get(x.dtype)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {x.dtype}")
    k, dev = shape[-1] if len(shape) else 0, x.get_device()
    if k < EXF_MX4_BLOCK or k % EXF_MX4_BLOCK or not x.is_contiguous():
        _bad(f"mx4_quantize: contiguous rows of a multiple of {EXF_MX4_BLOCK} elements expected, got {tuple(shape)}")
    if out is None:
        rows = x.numel() // k
        out = Mx4(torch.empty((*shape[:-1], k // 2), dtype=torch.uint8, device=x.device),
                  torch.empty(((k + 255) // 256, rows, 8), dtype=torch.uint8, device=x.device))
    else:
        rows = _expect_mx4("out", out, shape, dev)
    if dev < 0:
        _on_host()
    rc = lib().mx4_quantize(x.data_ptr(), rows, k, code, out.q.data_ptr(), out.scale.data_ptr(), _stream())
    if rc:
        _check(rc)
    return out


def mx4_dequantize(m, dtype=torch.bfloat16, out=None):
    """The values an Mx4 stands for, in `dtype` (that of ``out``)."""
    shape, dev = m.shape, m.q.get_device()
    rows = _expect_mx4("m", m, shape, dev)
    out = torch.empty(shape, dtype=dtype, device=m.q.device) if out is None else _expect("out", out, shape, out.dtype, dev)
    code = _CODES.get(out.dtype)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {out.dtype}")
    if dev < 0:
        _on_host()
    rc = lib().mx4_dequantize(m.q.data_ptr(), m.scale.data_ptr(), rows, shape[-1], code, out.data_ptr(), _stream())
    if rc:
        _check(rc)
    return out


def moe_grouped_product_mx4(x_sorted, expert_offsets, w, bias=None, dtype=None, out=None, workspace=None):
    """moe_grouped_product with weights held in 4 bits: w an Mx4 [E_local,n,k]; x_sorted an Mx4 [A,k], or rows of `dtype` that the call
    quantises.  The result has the type of the rows, or `dtype` (bf16)."""
    held = isinstance(x_sorted, Mx4)
    rows = x_sorted.q if held else x_sorted
    if rows.requires_grad or (bias is not None and bias.requires_grad):
        _untracked("moe_grouped_product_mx4")
    if len(w.q.shape) != 3 or len(rows.shape) != 2:
        _bad(f"rows are [A,k] and weights [E_local,n,k], got {tuple(x_sorted.shape)} and {tuple(w.shape)}")
    E, n, k = w.q.shape
    k *= 2
    A, dev = rows.shape[0], rows.get_device()
    _expect_mx4("w", w, (E, n, k), dev)
    if held:
        _expect_mx4("x_sorted", x_sorted, (A, k), dev)
        x_scale = x_sorted.scale.data_ptr()
        if dtype is None:
            dtype = torch.bfloat16 if out is None else out.dtype
    else:
        dtype = _expect("x_sorted", rows, (A, k), rows.dtype if dtype is None else dtype, dev).dtype
        x_scale = None
    code = _CODES.get(dtype)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dtype}")
    _expect("expert_offsets", expert_offsets, (E + 1,), _INT32, dev)
    if bias is not None:
        bias = _expect("bias", bias, (E, n), dtype, dev).data_ptr()
    out = torch.empty((A, n), dtype=dtype, device=rows.device) if out is None else _expect("out", out, (A, n), dtype, dev)
    if dev < 0:
        _on_host()
    if workspace is None and not held and A > EXF_MX4_INLINE_ROWS:
        need = lib().moe_grouped_product_mx4_workspace_bytes(A, n, k)
        workspace = _workspace(need, rows.device) if need else None
    workspace, size = (None, 0) if workspace is None else _bytes_of(workspace, dev)
    rc = lib().moe_grouped_product_mx4(rows.data_ptr(), x_scale, expert_offsets.data_ptr(), w.q.data_ptr(), w.scale.data_ptr(), bias, A, n, k, E, code,
                                       out.data_ptr(), workspace, size, _stream())
    if rc:
        _check(rc)
    return out


class Q4:
    """Rows in 4-bit integers: ``q`` uint8 [..., k/2], ``scale`` [..., k/group] of the rows' type, ``zero`` uint8 [..., k/group] or None (8 throughout); see
    q4_quantize.  Experts a .. b-1 of weights [E,n,k] are ``Q4(m.q[a:b], m.scale[a:b], m.zero[a:b])``."""
    __slots__ = ("q", "scale", "zero")

    def __init__(self, q, scale, zero=None):
        self.q, self.scale, self.zero = q, scale, zero

    @property
    def shape(self):
        s = self.q.shape
        return (*s[:-1], *(2 * k for k in s[-1:]))

    @property
    def group(self):
        return self.shape[-1] // max(self.scale.shape[-1], 1)


def _expect_q4(name, m, shape, dtype, dev):
    """`m` holds this shape with scales of `dtype` on device number `dev`; -> its group, which the library checks."""
    q, scale, zero = m.q, m.scale, m.zero
    if not len(shape) or not len(scale.shape) or not scale.shape[-1]:
        _bad(f"{name} has no groups")
    k, n = shape[-1], scale.shape[-1]
    if k % n:
        _bad(f"{name}: rows of {k} in {n} groups")
    groups = (*shape[:-1], n)
    if not (q.shape == (*shape[:-1], k // 2) and scale.shape == groups and q.dtype is _UINT8 and scale.dtype is dtype and q.is_contiguous() and scale.is_contiguous()
            and q.get_device() == scale.get_device() == dev
            and (zero is None or zero.shape == groups and zero.dtype is _UINT8 and zero.is_contiguous() and zero.get_device() == dev)):
        _expect(f"{name}.q", q, (*shape[:-1], k // 2), _UINT8, dev)
        _expect(f"{name}.scale", scale, groups, dtype, dev)
        if zero is not None:
            _expect(f"{name}.zero", zero, groups, _UINT8, dev)
    return k // n


def q4_quantize(x, group=128, symmetric=False, out=None):
    """Rows x [..., k] (k a multiple of the group: 32, 64 or 128) -> Q4, with zero points unless ``symmetric`` (``out`` says that by what it holds)."""
    if x.requires_grad:
        _untracked("q4_quantize", "none: codes have no gradient")
    if _forward_ad._current_level >= 0:
        _no_tangents("q4_quantize", x)
    shape, dt = x.shape, x.dtype
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    k, dev = shape[-1] if len(shape) else 0, x.get_device()
    if k < 1 or group < 1 or k % group or not x.is_contiguous():
        _bad(f"q4_quantize: contiguous rows of a multiple of {group} elements expected, got {tuple(shape)}")
    if out is None:
        groups = (*shape[:-1], k // group)
        out = Q4(torch.empty((*shape[:-1], k // 2), dtype=_UINT8, device=x.device), torch.empty(groups, dtype=dt, device=x.device),
                 None if symmetric else torch.empty(groups, dtype=_UINT8, device=x.device))
    elif _expect_q4("out", out, shape, dt, dev) != group or (out.zero is None) != bool(symmetric):
        _bad("q4_quantize: out holds other groups, or zero points where none are asked for")
    if dev < 0:
        _on_host()
    rc = lib().q4_quantize(x.data_ptr(), x.numel() // k, k, group, code, out.q.data_ptr(), out.scale.data_ptr(), _ptr(out.zero), _stream_on(dev))
    if rc:
        _check(rc)
    return out


def q4_dequantize(m, out=None):
    """The values a Q4 stands for, in its scales' type."""
    if m.scale.requires_grad:
        _untracked("q4_dequantize", "none: weights in 4 bits are not trained")
    if _forward_ad._current_level >= 0:
        _no_tangents("q4_dequantize", m.scale)
    shape, dt, dev = m.shape, m.scale.dtype, m.q.get_device()
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    group = _expect_q4("m", m, shape, dt, dev)
    out = torch.empty(shape, dtype=dt, device=m.q.device) if out is None else _expect("out", out, shape, dt, dev)
    if dev < 0:
        _on_host()
    rc = lib().q4_dequantize(m.q.data_ptr(), m.scale.data_ptr(), _ptr(m.zero), m.q.numel() * 2 // max(shape[-1], 1), shape[-1], group, code, out.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)
    return out


def moe_grouped_product_q4(x_sorted, expert_offsets, w, bias=None, out=None):
    """moe_grouped_product with weights in 4-bit integers: w a Q4 [E_local,n,k] with scales of the rows' type."""
    if x_sorted.requires_grad or bias is not None and bias.requires_grad or w.scale.requires_grad:
        _untracked("moe_grouped_product_q4", "none: weights in 4 bits are not trained")
    if _forward_ad._current_level >= 0:
        _no_tangents("moe_grouped_product_q4", x_sorted, bias, w.scale)
    q, scale, zero = w.q, w.scale, w.zero
    shape, groups, rows = q.shape, scale.shape, x_sorted.shape
    if len(shape) != 3 or len(rows) != 2:
        _bad(f"rows are [A,k] and weights [E_local,n,k], got {tuple(rows)} and {w.shape}")
    E, n, k = shape
    k *= 2
    A, dt, dev = rows[0], x_sorted.dtype, x_sorted.get_device()
    code = _CODES.get(dt)
    if code is None:
        raise ExflowError(EXF_ERR_BAD_DTYPE, f"unsupported dtype {dt}")
    # (what _expect_q4 finds of the usual case, number by number: a microsecond less)
    if (len(groups) == 3 and groups[0] == E and groups[1] == n and groups[2] and not k % groups[2] and q.dtype is _UINT8 and scale.dtype is dt and q.is_contiguous()
            and scale.is_contiguous() and q.get_device() == scale.get_device() == dev
            and (zero is None or zero.shape == groups and zero.dtype is _UINT8 and zero.is_contiguous() and zero.get_device() == dev)):
        group = k // groups[2]
    else:
        group = _expect_q4("w", w, (E, n, k), dt, dev)
    if out is None:
        out = _rows(A, n, dt, x_sorted.device)
    if bias is not None:
        bias = _expect("bias", bias, (E, n), dt, dev).data_ptr()
    if not (rows[1] == k and expert_offsets.shape == (E + 1,) and out.shape == (A, n) and out.dtype is dt and expert_offsets.dtype is _INT32
            and x_sorted.is_contiguous() and out.is_contiguous() and expert_offsets.is_contiguous() and out.get_device() == expert_offsets.get_device() == dev >= 0):
        _misfit(x_sorted, (A, k), expert_offsets, E, scale, out, (A, n), dt, dev)
    rc = lib().moe_grouped_product_q4(x_sorted.data_ptr(), expert_offsets.data_ptr(), q.data_ptr(), scale.data_ptr(), None if zero is None else zero.data_ptr(), bias, A, n, k, group, E, code,
                                      out.data_ptr(), _stream_on(dev))
    if rc:
        _check(rc)
    return out


def affinity_histogram(trace, E, want_loads=True, want_prob=True, want_invalid=True, workspace=None, out=None):
    """trace int32 [L,N] on the device -> dict(counts, loads, cond_prob, n_invalid) of device tensors."""
    L, N = trace.shape
    assert trace.dtype == torch.int32 and trace.is_contiguous()
    dev = trace.device
    if out is None:
        out = dict(
            counts=torch.empty((max(L - 1, 0), E, E), dtype=torch.int64, device=dev),
            loads=torch.empty((L, E), dtype=torch.int64, device=dev) if want_loads else None,
            cond_prob=torch.empty((max(L - 1, 0), E, E), dtype=torch.float32, device=dev) if want_prob else None,
            n_invalid=torch.empty(1, dtype=torch.int64, device=dev) if want_invalid else None,
        )
    if workspace is None:
        workspace = _workspace(lib().affinity_histogram_workspace_bytes(L, N, E), dev)
    _check(lib().affinity_histogram(_ptr(trace), L, N, E, _ptr(out["counts"]), _ptr(out["loads"]), _ptr(out["cond_prob"]),
                                    _ptr(out["n_invalid"]), _ptr(workspace), workspace.numel(), _stream()))
    return out


def affinity_statistics(trace, placement, G, want_loads=True, want_prob=True, want_invalid=True, workspace=None, out=None):
    """One pass over the trace -> dict(counts, loads, cond_prob, n_invalid, local_per_pair) of device tensors."""
    L, N = trace.shape
    E = placement.shape[1]
    assert placement.shape[0] == L and placement.dtype == torch.int32 and trace.dtype == torch.int32
    assert trace.is_contiguous() and placement.is_contiguous()
    dev = trace.device
    if out is None:
        out = dict(
            counts=torch.empty((max(L - 1, 0), E, E), dtype=torch.int64, device=dev),
            loads=torch.empty((L, E), dtype=torch.int64, device=dev) if want_loads else None,
            cond_prob=torch.empty((max(L - 1, 0), E, E), dtype=torch.float32, device=dev) if want_prob else None,
            n_invalid=torch.empty(1, dtype=torch.int64, device=dev) if want_invalid else None,
            local_per_pair=torch.empty(max(L - 1, 0), dtype=torch.int64, device=dev),
        )
    if workspace is None:
        workspace = _workspace(lib().affinity_statistics_workspace_bytes(L, N, E), dev)
    _check(lib().affinity_statistics(_ptr(trace), _ptr(placement), L, N, E, G, _ptr(out["counts"]), _ptr(out["loads"]),
                                     _ptr(out["cond_prob"]), _ptr(out["n_invalid"]), _ptr(out["local_per_pair"]), _ptr(workspace),
                                     workspace.numel(), _stream()))
    return out


def placement_locality(trace, placement, G, workspace=None, out=None):
    """-> local_per_pair int64 [L-1] (device); fraction = sum / (N*(L-1))."""
    L, N = trace.shape
    E = placement.shape[1]
    assert placement.shape[0] == L and placement.dtype == torch.int32 and trace.dtype == torch.int32
    assert trace.is_contiguous() and placement.is_contiguous()
    if out is None:
        out = torch.empty(max(L - 1, 0), dtype=torch.int64, device=trace.device)
    if workspace is None:
        workspace = _workspace(lib().placement_locality_workspace_bytes(L, N), trace.device)
    _check(lib().placement_locality(_ptr(trace), _ptr(placement), L, N, E, G, _ptr(out), _ptr(workspace), workspace.numel(),
                                    _stream()))
    return out


def affinity_multihop(trace, E, want_prob=True, workspace=None):
    """-> dict(counts int64 [L(L-1)/2,E,E], cond_prob fp32 or None) on the device, pairs source layer first."""
    L, N = trace.shape
    assert trace.dtype == torch.int32 and trace.is_contiguous()
    P = L * (L - 1) // 2
    counts = torch.empty((P, E, E), dtype=torch.int64, device=trace.device)
    prob = torch.empty((P, E, E), dtype=torch.float32, device=trace.device) if want_prob else None
    if workspace is None:
        workspace = _workspace(lib().affinity_multihop_workspace_bytes(L, N, E), trace.device)
    _check(lib().affinity_multihop(_ptr(trace), L, N, E, _ptr(counts), _ptr(prob), _ptr(workspace), workspace.numel(), _stream()))
    return {"counts": counts, "cond_prob": prob}


def routing_transfers(trace, placement, home, G, workspace=None):
    """-> (local_per_pair int64 [L-1], away_per_layer int64 [L]) on the device."""
    L, N = trace.shape
    rows, E = placement.shape
    assert rows == L and home.shape == (N,)
    assert trace.dtype == placement.dtype == home.dtype == torch.int32
    assert trace.is_contiguous() and placement.is_contiguous() and home.is_contiguous()
    dev = trace.device
    local = torch.empty(max(L - 1, 0), dtype=torch.int64, device=dev)
    away = torch.empty(L, dtype=torch.int64, device=dev)
    if workspace is None:
        workspace = _workspace(lib().routing_transfers_workspace_bytes(L, N), dev)
    rc = lib().routing_transfers(trace.data_ptr(), placement.data_ptr(), home.data_ptr(), L, N, E, G, local.data_ptr(), away.data_ptr(),
                                 workspace.data_ptr(), workspace.numel(), _stream())
    if rc:
        _check(rc)
    return local, away


def placement_locality_from_counts(counts, placements, out=None):
    """counts int64 [L-1,E,E] (device), placements int32 [B,L,E] (device) -> local int64 [B,L-1] (device)."""
    B, L, E = placements.shape
    assert counts.shape == (L - 1, E, E) and counts.dtype == torch.int64 and placements.dtype == torch.int32
    assert counts.is_contiguous() and placements.is_contiguous()
    if out is None:
        out = torch.empty((B, max(L - 1, 0)), dtype=torch.int64, device=counts.device)
    _check(lib().placement_locality_from_counts(_ptr(counts), _ptr(placements), B, L, E, _ptr(out), _stream()))
    return out


def placement_search(counts_host, G, nodes=1, restarts=4, seed=0):
    """counts_host int64 [L-1,E,E] (torch CPU) -> placement int32 [L,E] (torch CPU): the host solver."""
    assert counts_host.device.type == "cpu" and counts_host.dtype == torch.int64 and counts_host.is_contiguous()
    Lm1, E, _ = counts_host.shape
    out = torch.empty((Lm1 + 1, E), dtype=torch.int32)
    _check(lib().exf_placement_search(counts_host.data_ptr(), Lm1 + 1, E, G, nodes, restarts, seed, out.data_ptr()))
    return out


def check_placement(placement_host, G) -> bool:
    """Load-balance and exclusivity constraints of a HOST placement (torch CPU int32 [L,E])."""
    assert placement_host.device.type == "cpu" and placement_host.dtype == torch.int32 and placement_host.is_contiguous()
    L, E = placement_host.shape
    return lib().exf_check_placement(placement_host.data_ptr(), L, E, G) == EXF_OK


def comm_volume(G, N, L, p, p_star):
    """Forward communication of the paper's comparison table, in tokens:
    dict(vanilla_top1, vanilla_top2, coherent_top1, coherent_top2)."""
    out = (ctypes.c_double * 4)()
    _check(lib().exf_comm_volume(int(G), int(N), int(L), float(p), float(p_star), ctypes.addressof(out)))
    return dict(vanilla_top1=out[0], vanilla_top2=out[1], coherent_top1=out[2], coherent_top2=out[3])


def transfer_ratios(away_per_layer_host, local_per_pair_host, tokens):
    """(p, p_star) from HOST copies (torch CPU int64) of the counters routing_transfers returns."""
    assert away_per_layer_host.device.type == "cpu" and away_per_layer_host.dtype == torch.int64 and away_per_layer_host.is_contiguous()
    L = away_per_layer_host.numel()
    if L > 1:
        assert local_per_pair_host.device.type == "cpu" and local_per_pair_host.dtype == torch.int64
        assert local_per_pair_host.is_contiguous() and local_per_pair_host.numel() == L - 1
    p, p_star = ctypes.c_double(), ctypes.c_double()
    _check(lib().exf_transfer_ratios(away_per_layer_host.data_ptr(), local_per_pair_host.data_ptr() if L > 1 else None, L, int(tokens),
                                     ctypes.addressof(p), ctypes.addressof(p_star)))
    return p.value, p_star.value
