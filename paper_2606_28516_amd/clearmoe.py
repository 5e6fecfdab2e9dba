"""Python binding of the CLEAR-MoE C ABI (``include/clearmoe.h``).

Argument marshalling only: every step of the layer runs in the HIP library
``libclearmoe.so``.  PyTorch supplies device memory and the current stream.
There is no fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np
import torch

__all__ = ["ClearMoEError", "Shape", "lib", "version", "workspace_bytes", "alloc_workspace",
           "route", "dispatch", "combine", "ffn_forward", "from_stored", "to_stored",
           "DISPATCH_HIST_IN_WS", "F32", "BF16", "SYMBOLS", "N_STAGES", "stage_names",
           "timing_start", "timing_stop", "make_shape", "dense_ffn_forward",
           "padded_workspace_bytes", "ffn_forward_padded", "ffn_forward_noalloc",
           "StackLayer", "make_stack_layer", "stack_shape", "stack_workspace_bytes",
           "stack_forward", "Router", "make_router", "route_ex",
           "ffn_forward_ex", "FEW_MAX_TOKENS", "few_workspace_bytes", "alloc_few_workspace",
           "ffn_forward_few", "Product", "quantize", "quantized_gemm", "quantized_workspace_bytes",
           "alloc_quantized_workspace", "quantized_ffn_forward", "Norm", "dequantize", "rms_norm"]

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libclearmoe.so")
F32, BF16 = 0, 1
DISPATCH_HIST_IN_WS = 1
SYMBOLS = ("clearmoe_version", "clearmoe_source_digest", "clearmoe_status_string", "clearmoe_workspace_bytes",
           "clearmoe_route", "clearmoe_dispatch", "clearmoe_combine", "clearmoe_ffn_forward",
           "clearmoe_dense_ffn_forward", "clearmoe_stage_name", "clearmoe_timing_start",
           "clearmoe_timing_start_sampled", "clearmoe_timing_stop", "clearmoe_padded_workspace_bytes",
           "clearmoe_ffn_forward_padded", "clearmoe_route_ex", "clearmoe_ffn_forward_ex",
           "clearmoe_ffn_forward_noalloc", "clearmoe_stack_workspace_bytes",
           "clearmoe_stack_forward", "clearmoe_few_workspace_bytes", "clearmoe_ffn_forward_few",
           "clearmoe_quantize", "clearmoe_quantized_gemm", "clearmoe_quantized_workspace_bytes",
           "clearmoe_quantized_ffn_forward", "clearmoe_quantized_ffn_forward_ex", "clearmoe_dequantize",
           "clearmoe_rms_norm")
NOALLOC_SCRATCH_BYTES = 64 << 20
ERR_TOO_LARGE = 5
FEW_MAX_TOKENS = 64
N_STAGES = 20


class ClearMoEError(RuntimeError):
    pass


class Shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "D", "H", "E", "k", "r", "q", "dtype", "renorm")]


class Router(ctypes.Structure):
    """clearmoe_router: scores (linear, or an MLP with `hidden` units) and the
    selection rule (top-k, or adaptive top-1 / top-2 at threshold tau)."""
    _fields_ = [("Wg", ctypes.c_void_p), ("bg", ctypes.c_void_p), ("Wh", ctypes.c_void_p),
                ("bh", ctypes.c_void_p), ("W2", ctypes.c_void_p), ("hidden", ctypes.c_int32),
                ("adaptive", ctypes.c_int32), ("dense_stride", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("tau", ctypes.c_double)]


class Product(ctypes.Structure):
    """clearmoe_product: a product of quantised matrices."""
    _fields_ = [("M", ctypes.c_int64), ("N", ctypes.c_int32), ("K", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("a_format", ctypes.c_int32), ("b_format", ctypes.c_int32), ("out", ctypes.c_int32),
                ("gelu", ctypes.c_int32), ("reserved", ctypes.c_int32), ("lda", ctypes.c_int64),
                ("ldc", ctypes.c_int64)]


class Norm(ctypes.Structure):
    """clearmoe_norm: the root-mean-square norm of rows."""
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("out", ctypes.c_int32), ("eps", ctypes.c_float), ("ldx", ctypes.c_int64), ("ldr", ctypes.c_int64),
                ("lds", ctypes.c_int64), ("ldy", ctypes.c_int64)]


class StackLayer(ctypes.Structure):
    """clearmoe_stack_layer: a dense FFN (moe = 0) or a CLEAR-MoE layer
    (moe = 1, k experts per token, with its router)."""
    _fields_ = [("moe", ctypes.c_int32), ("k", ctypes.c_int32), ("W1", ctypes.c_void_p),
                ("b1", ctypes.c_void_p), ("US", ctypes.c_void_p), ("Vt", ctypes.c_void_p),
                ("b2", ctypes.c_void_p), ("P", ctypes.c_void_p), ("Q", ctypes.c_void_p),
                ("W2", ctypes.c_void_p), ("router", Router)]


_lib = None


def lib():
    """Load the in-tree library.  It is built first when it is missing or was
    built from other sources than the ones in the tree (the library carries
    the digest of its sources)."""
    global _lib
    if _lib is None:
        from . import build as _build
        want = _build.source_digest()
        have = _build.built_digest(LIB_PATH)
        if have != want:
            import sys
            print(f"clearmoe: library {'missing' if not have else 'stale (' + have + ')'}, "
                  f"building for sources {want}", file=sys.stderr)
            _build.build()
            if _build.built_digest(LIB_PATH) != want:
                raise ClearMoEError("the rebuilt library does not carry the source digest")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, u32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint
        sp = ctypes.POINTER(Shape)
        L.clearmoe_version.restype = ctypes.c_int
        L.clearmoe_source_digest.restype = ctypes.c_char_p
        L.clearmoe_status_string.restype = ctypes.c_char_p
        L.clearmoe_status_string.argtypes = [ctypes.c_int]
        L.clearmoe_workspace_bytes.restype = sz
        L.clearmoe_workspace_bytes.argtypes = [sp]
        L.clearmoe_route.restype = ctypes.c_int
        L.clearmoe_route.argtypes = [sp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.clearmoe_dispatch.restype = ctypes.c_int
        L.clearmoe_dispatch.argtypes = [sp, vp, vp, sz, vp, vp, vp, vp, vp, vp, u32, vp]
        L.clearmoe_combine.restype = ctypes.c_int
        L.clearmoe_combine.argtypes = [sp, vp, vp, vp, vp, vp]
        L.clearmoe_ffn_forward.restype = ctypes.c_int
        L.clearmoe_ffn_forward.argtypes = [sp] + [vp] * 13 + [vp, sz, vp]
        rp = ctypes.POINTER(Router)
        L.clearmoe_route_ex.restype = ctypes.c_int
        L.clearmoe_route_ex.argtypes = [sp, rp, vp, vp, vp, vp, sz, vp]
        L.clearmoe_ffn_forward_ex.restype = ctypes.c_int
        L.clearmoe_ffn_forward_ex.argtypes = [sp, rp] + [vp] * 11 + [vp, sz, vp]
        L.clearmoe_padded_workspace_bytes.restype = sz
        L.clearmoe_padded_workspace_bytes.argtypes = [sp]
        L.clearmoe_ffn_forward_padded.restype = ctypes.c_int
        L.clearmoe_ffn_forward_padded.argtypes = [sp] + [vp] * 13 + [vp, sz, vp]
        L.clearmoe_ffn_forward_noalloc.restype = ctypes.c_int
        L.clearmoe_ffn_forward_noalloc.argtypes = [sp] + [vp] * 13 + [vp]
        lp = ctypes.POINTER(StackLayer)
        L.clearmoe_stack_workspace_bytes.restype = sz
        L.clearmoe_stack_workspace_bytes.argtypes = [sp, lp, ctypes.c_int32]
        L.clearmoe_stack_forward.restype = ctypes.c_int
        L.clearmoe_stack_forward.argtypes = [sp, lp, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, sz,
                                             vp]
        L.clearmoe_dense_ffn_forward.restype = ctypes.c_int
        L.clearmoe_dense_ffn_forward.argtypes = [sp] + [vp] * 6 + [vp, sz, vp]
        L.clearmoe_few_workspace_bytes.restype = sz
        L.clearmoe_few_workspace_bytes.argtypes = [sp]
        L.clearmoe_ffn_forward_few.restype = ctypes.c_int
        L.clearmoe_ffn_forward_few.argtypes = [sp, rp] + [vp] * 11 + [vp, sz, vp]
        L.clearmoe_quantize.restype = ctypes.c_int
        L.clearmoe_quantize.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64] * 2 + [ctypes.c_int32, vp,
                                                                                  ctypes.c_int64, vp, vp, vp]
        L.clearmoe_quantized_gemm.restype = ctypes.c_int
        L.clearmoe_quantized_gemm.argtypes = [ctypes.POINTER(Product)] + [vp] * 9
        L.clearmoe_quantized_workspace_bytes.restype = sz
        L.clearmoe_quantized_workspace_bytes.argtypes = [sp]
        L.clearmoe_quantized_ffn_forward.restype = ctypes.c_int
        L.clearmoe_quantized_ffn_forward.argtypes = [sp] + [vp] * 10 + [sz, vp]
        L.clearmoe_quantized_ffn_forward_ex.restype = ctypes.c_int
        L.clearmoe_quantized_ffn_forward_ex.argtypes = [sp, ctypes.c_int, ctypes.c_int] + [vp] * 10 + [sz, vp]
        L.clearmoe_dequantize.restype = ctypes.c_int
        L.clearmoe_dequantize.argtypes = [ctypes.c_int] * 2 + [ctypes.c_int64] * 2 + [
            ctypes.c_int32, vp, vp, ctypes.c_int, vp, ctypes.c_int64, vp]
        L.clearmoe_rms_norm.restype = ctypes.c_int
        L.clearmoe_rms_norm.argtypes = [ctypes.POINTER(Norm)] + [vp] * 7
        L.clearmoe_stage_name.restype = ctypes.c_char_p
        L.clearmoe_stage_name.argtypes = [ctypes.c_int]
        L.clearmoe_timing_start.restype = ctypes.c_int
        L.clearmoe_timing_start.argtypes = [u32, ctypes.c_int]
        L.clearmoe_timing_start_sampled.restype = ctypes.c_int
        L.clearmoe_timing_start_sampled.argtypes = [u32, ctypes.c_int, ctypes.c_int]
        L.clearmoe_timing_stop.restype = ctypes.c_int
        L.clearmoe_timing_stop.argtypes = [ctypes.POINTER(ctypes.c_double),
                                           ctypes.POINTER(ctypes.c_int32)]
        _lib = L
    return _lib


def version() -> int:
    return lib().clearmoe_version()


def _check(rc: int, what: str) -> None:
    if rc != 0:
        msg = lib().clearmoe_status_string(rc).decode()
        raise ClearMoEError(f"{what}: {msg} (status {rc})")


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise ClearMoEError(f"unsupported dtype {t.dtype}")


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ClearMoEError("tensor is not on the GPU")
    if not t.is_contiguous():
        raise ClearMoEError("tensor is not contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t: Optional[torch.Tensor], dev: int) -> Optional[int]:
    """The address of a tensor on device dev (_p with a check of the device;
    ctypes turns it into the pointer argument)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ClearMoEError("the tensors are not on one device" if t.is_cuda else "tensor is not on the GPU")
    if not t.is_contiguous():
        raise ClearMoEError("tensor is not contiguous")
    return t.data_ptr()


def _shaped(t: torch.Tensor, dtype, shape: tuple, what: str, dev: int) -> int:
    """The address of a tensor that has to have this type and shape."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype or t.shape != shape:
        raise ClearMoEError(f"{what} must be {dtype} {shape}, not {t.dtype} {tuple(t.shape)}")
    return _ptr(t, dev)


def _shaped_or_none(t: Optional[torch.Tensor], dtype, shape: tuple, what: str, dev: int) -> Optional[int]:
    return None if t is None else _shaped(t, dtype, shape, what, dev)


def _queue(dev: int, stream) -> int:
    """The stream of a call on tensors of device dev, which has to be the
    current one: the kernels are launched there.  The current stream is asked
    for by its handle (a torch.cuda.Stream object costs 3 us, a quarter of a
    small call)."""
    if dev < 0:
        raise ClearMoEError("tensor is not on the GPU")
    if dev != torch._C._cuda_getDevice():
        raise ClearMoEError("the tensors are not on the current device")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ClearMoEError("the stream is not of the tensors' device")
    return stream.cuda_stream


def _empty(x: torch.Tensor, shape: tuple, dtype, stream, kept: bool = True) -> torch.Tensor:
    """A new tensor on x's device for a call on `stream` (None: the current
    one).  Its memory comes from that stream's own pool, so that nothing still
    queued elsewhere uses it and what is freed on return goes to later work of
    the same stream only.  kept: the caller gets it, and may let go of it while
    the current stream still reads it."""
    if stream is None:
        return x.new_empty(*shape, dtype=dtype)  # (a tuple in one piece costs more)
    with torch.cuda.stream(stream):
        t = x.new_empty(shape, dtype=dtype)
    if kept and t.is_cuda:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _workspace(n: int, x: torch.Tensor, stream, what: str = "shape") -> torch.Tensor:
    """n bytes for the duration of a call on `stream`."""
    if n == 0:
        raise ClearMoEError(f"invalid {what}")
    return _empty(x, (n,), torch.uint8, stream, kept=False)


def make_shape(T, D, E, k, dtype, H=0, r=0, q=0, renorm=1) -> Shape:
    """renorm = 1: the top-k gates renormalised over the selected experts;
    0: their probabilities under the softmax over all E."""
    return Shape(int(T), int(D), int(H), int(E), int(k), int(r), int(q), int(dtype), int(renorm))


def workspace_bytes(shape: Shape) -> int:
    return int(lib().clearmoe_workspace_bytes(ctypes.byref(shape)))


def alloc_workspace(shape: Shape, device="cuda") -> torch.Tensor:
    n = workspace_bytes(shape)
    if n == 0:
        raise ClearMoEError("invalid shape")
    return torch.empty(n, dtype=torch.uint8, device=device)


def route(x, Wg, bg, k: int, ws: Optional[torch.Tensor] = None, stream=None, renorm: int = 1):
    """clearmoe_route: returns (idx [T,k] int32, gate [T,k] float32)."""
    T, D = x.shape
    E = Wg.shape[0]
    s = make_shape(T, D, E, k, _dt(x), renorm=renorm)
    ws = _workspace(workspace_bytes(s), x, stream) if ws is None else ws
    idx = _empty(x, (T, k), torch.int32, stream)
    gate = _empty(x, (T, k), torch.float32, stream)
    rc = lib().clearmoe_route(ctypes.byref(s), _p(x), _p(Wg), _p(bg), _p(idx), _p(gate), _p(ws),
                              ws.numel(), _stream(stream))
    _check(rc, "clearmoe_route")
    return idx, gate


def make_router(Wg, bg=None, Wh=None, bh=None, adaptive: bool = False, tau: float = 0.0,
                dense_stride: int = 0, W2=None):
    """A Router over device tensors (keep the tensors alive while it is used):
    linear when Wh is None, else an MLP with Wh.shape[0] hidden units; with
    dense_stride > 0, token t with t % dense_stride == 0 is a class token
    (dense path, fc2 weight W2)."""
    p = lambda t: None if t is None else _p(t).value  # noqa: E731
    return Router(p(Wg), p(bg), p(Wh), p(bh), p(W2), 0 if Wh is None else int(Wh.shape[0]),
                  1 if adaptive else 0, int(dense_stride), 0, float(tau))


def route_ex(x, router: Router, E: int, k: int, ws: Optional[torch.Tensor] = None, stream=None,
             renorm: int = 1):
    """clearmoe_route_ex: returns (idx [T,k] int32, -1 = empty slot; gate [T,k])."""
    T, D = x.shape
    s = make_shape(T, D, E, k, _dt(x), renorm=renorm)
    ws = _workspace(workspace_bytes(s), x, stream) if ws is None else ws
    idx = _empty(x, (T, k), torch.int32, stream)
    gate = _empty(x, (T, k), torch.float32, stream)
    rc = lib().clearmoe_route_ex(ctypes.byref(s), ctypes.byref(router), _p(x), _p(idx), _p(gate),
                                 _p(ws), ws.numel(), _stream(stream))
    _check(rc, "clearmoe_route_ex")
    return idx, gate


def dispatch(idx, E: int, ws: Optional[torch.Tensor] = None, x=None, D: Optional[int] = None,
             hist_in_ws: bool = False, stream=None):
    """clearmoe_dispatch: returns (counts, offsets, perm, inv, xperm or None)."""
    T, k = idx.shape
    if x is not None:
        D, dtype = x.shape[1], _dt(x)
    else:
        D, dtype = 8, BF16          # no rows to copy: D only has to be valid
    s = make_shape(T, D, E, k, dtype)
    ws = _workspace(workspace_bytes(s), idx, stream) if ws is None else ws
    counts = _empty(idx, (E,), torch.int32, stream)
    offsets = _empty(idx, (E + 1,), torch.int32, stream)
    perm = _empty(idx, (T * k,), torch.int32, stream)
    inv = _empty(idx, (T * k,), torch.int32, stream)
    xperm = None if x is None else _empty(idx, (T * k, D), x.dtype, stream)
    rc = lib().clearmoe_dispatch(ctypes.byref(s), _p(idx), _p(ws), ws.numel(), _p(counts),
                                 _p(offsets), _p(perm), _p(inv), _p(x), _p(xperm),
                                 DISPATCH_HIST_IN_WS if hist_in_ws else 0, _stream(stream))
    _check(rc, "clearmoe_dispatch")
    return counts, offsets, perm, inv, xperm


def combine(ye, inv, gate, out: Optional[torch.Tensor] = None, stream=None):
    """clearmoe_combine: y[t] = sum_j gate[t,j] * ye[inv[t*k+j]]."""
    T, k = gate.shape
    D = ye.shape[1]
    E = max(k, 1)
    s = make_shape(T, D, E, k, _dt(ye))
    y = _empty(ye, (T, D), ye.dtype, stream) if out is None else out
    rc = lib().clearmoe_combine(ctypes.byref(s), _p(ye), _p(inv), _p(gate), _p(y),
                                _stream(stream))
    _check(rc, "clearmoe_combine")
    return y


def padded_workspace_bytes(shape: Shape) -> int:
    return int(lib().clearmoe_padded_workspace_bytes(ctypes.byref(shape)))


def _layer_call(name, ws_bytes, x, W1, b1, US, Vt, b2, P, Q, Wg, bg, k, ws, out, idx_out,
                gate_out, stream, renorm=1):
    T, D = x.shape
    H = W1.shape[0]
    r = US.shape[1]
    E, _, q = P.shape
    s = make_shape(T, D, E, k, _dt(x), H=H, r=r, q=q, renorm=renorm)
    ws = _workspace(ws_bytes(s), x, stream) if ws is None else ws
    y = _empty(x, (T, D), x.dtype, stream) if out is None else out
    rc = getattr(lib(), name)(ctypes.byref(s), _p(x), _p(W1), _p(b1), _p(US), _p(Vt), _p(b2),
                              _p(P), _p(Q), _p(Wg), _p(bg), _p(y), _p(idx_out), _p(gate_out),
                              _p(ws), ws.numel(), _stream(stream))
    _check(rc, name)
    return y


def ffn_forward(x, W1, b1, US, Vt, b2, P, Q, Wg, bg, k: int, ws: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, idx_out=None, gate_out=None, stream=None,
                renorm: int = 1):
    """clearmoe_ffn_forward: the whole layer.  Returns y [T, D]."""
    return _layer_call("clearmoe_ffn_forward", workspace_bytes, x, W1, b1, US, Vt, b2, P, Q, Wg,
                       bg, k, ws, out, idx_out, gate_out, stream, renorm)


def ffn_forward_noalloc(x, W1, b1, US, Vt, b2, P, Q, Wg, bg, k: int,
                        out: Optional[torch.Tensor] = None, idx_out=None, gate_out=None,
                        stream=None, renorm: int = 1):
    """clearmoe_ffn_forward_noalloc: the whole layer with the library's own
    fixed scratch (no workspace).  Returns y [T, D]."""
    T, D = x.shape
    H = W1.shape[0]
    r = US.shape[1]
    E, _, q = P.shape
    s = make_shape(T, D, E, k, _dt(x), H=H, r=r, q=q, renorm=renorm)
    y = _empty(x, (T, D), x.dtype, stream) if out is None else out
    rc = lib().clearmoe_ffn_forward_noalloc(ctypes.byref(s), _p(x), _p(W1), _p(b1), _p(US), _p(Vt),
                                            _p(b2), _p(P), _p(Q), _p(Wg), _p(bg), _p(y),
                                            _p(idx_out), _p(gate_out), _stream(stream))
    _check(rc, "clearmoe_ffn_forward_noalloc")
    return y


def ffn_forward_padded(x, W1, b1, US, Vt, b2, P, Q, Wg, bg, k: int,
                       ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       idx_out=None, gate_out=None, stream=None, renorm: int = 1):
    """clearmoe_ffn_forward_padded: the whole layer through the padded batched
    backend (blocks the host until dispatch is done).  Returns y [T, D]."""
    return _layer_call("clearmoe_ffn_forward_padded", padded_workspace_bytes, x, W1, b1, US, Vt,
                       b2, P, Q, Wg, bg, k, ws, out, idx_out, gate_out, stream, renorm)


def ffn_forward_ex(x, W1, b1, US, Vt, b2, P, Q, router: Router, k: int,
                   ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   idx_out=None, gate_out=None, stream=None, renorm: int = 1):
    """clearmoe_ffn_forward_ex: the whole layer with any router.  Returns y."""
    T, D = x.shape
    H = W1.shape[0]
    r = US.shape[1]
    E, _, q = P.shape
    s = make_shape(T, D, E, k, _dt(x), H=H, r=r, q=q, renorm=renorm)
    ws = _workspace(workspace_bytes(s), x, stream) if ws is None else ws
    y = _empty(x, (T, D), x.dtype, stream) if out is None else out
    rc = lib().clearmoe_ffn_forward_ex(ctypes.byref(s), ctypes.byref(router), _p(x), _p(W1),
                                       _p(b1), _p(US), _p(Vt), _p(b2), _p(P), _p(Q), _p(y),
                                       _p(idx_out), _p(gate_out), _p(ws), ws.numel(),
                                       _stream(stream))
    _check(rc, "clearmoe_ffn_forward_ex")
    return y


def dense_ffn_forward(x, W1, b1, W2, b2, ws: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, stream=None):
    """clearmoe_dense_ffn_forward: y = GELU(x W1^T + b1) W2^T + b2."""
    T, D = x.shape
    H = W1.shape[0]
    s = make_shape(T, D, 1, 1, _dt(x), H=H)
    ws = _workspace(workspace_bytes(s), x, stream) if ws is None else ws
    y = _empty(x, (T, D), x.dtype, stream) if out is None else out
    rc = lib().clearmoe_dense_ffn_forward(ctypes.byref(s), _p(x), _p(W1), _p(b1), _p(W2), _p(b2),
                                          _p(y), _p(ws), ws.numel(), _stream(stream))
    _check(rc, "clearmoe_dense_ffn_forward")
    return y


def make_stack_layer(W1, b1, b2, US=None, Vt=None, P=None, Q=None, router: Optional[Router] = None,
                     k: int = 1, W2=None) -> StackLayer:
    """A stack layer over device tensors (keep them alive while it is used):
    dense when router is None (W1, b1, W2, b2), else a CLEAR-MoE layer."""
    p = lambda t: None if t is None else _p(t).value  # noqa: E731
    if router is None:
        return StackLayer(0, 1, p(W1), p(b1), None, None, p(b2), None, None, p(W2), Router())
    return StackLayer(1, int(k), p(W1), p(b1), p(US), p(Vt), p(b2), p(P), p(Q), p(W2), router)


def stack_shape(x, H: int, E: int, r: int, q: int) -> Shape:
    T, D = x.shape
    return make_shape(T, D, E, 1, _dt(x), H=H, r=r, q=q)


def stack_workspace_bytes(shape: Shape, layers) -> int:
    arr = (StackLayer * len(layers))(*layers)
    return int(lib().clearmoe_stack_workspace_bytes(ctypes.byref(shape), arr, len(layers)))


def stack_forward(x, layers, H: int, E: int, r: int, q: int, residual: bool = True,
                  ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  stream=None):
    """clearmoe_stack_forward: x through the chain of layers (each a
    StackLayer), x_{l+1} = x_l + f_l(x_l) with residual, else f_l(x_l).
    Returns y [T, D]."""
    s = stack_shape(x, H, E, r, q)
    arr = (StackLayer * len(layers))(*layers)
    if ws is None:
        ws = _workspace(int(lib().clearmoe_stack_workspace_bytes(ctypes.byref(s), arr, len(layers))), x, stream, "stack")
    y = _empty(x, tuple(x.shape), x.dtype, stream) if out is None else out
    rc = lib().clearmoe_stack_forward(ctypes.byref(s), arr, len(layers), 1 if residual else 0,
                                      _p(x), _p(y), _p(ws), ws.numel(), _stream(stream))
    _check(rc, "clearmoe_stack_forward")
    return y


def few_workspace_bytes(shape: Shape) -> int:
    return int(lib().clearmoe_few_workspace_bytes(ctypes.byref(shape)))


def _alloc(n: int, device) -> torch.Tensor:
    if n == 0:
        raise ClearMoEError("invalid shape")
    return torch.empty(n, dtype=torch.uint8, device=device)


def alloc_few_workspace(shape: Shape, device="cuda") -> torch.Tensor:
    return _alloc(few_workspace_bytes(shape), device)


def ffn_forward_few(x, W1, b1, US, Vt, b2, P, Q, router: Router, k: int,
                    ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    idx_out=None, gate_out=None, stream=None, renorm: int = 1):
    """clearmoe_ffn_forward_few: the whole layer for at most FEW_MAX_TOKENS
    tokens, with any router without class tokens (its tensors on x's device).
    Returns y."""
    T, D = x.shape
    H, r, (E, _, q), dt = W1.shape[0], US.shape[1], P.shape, x.dtype
    s = Shape(T, D, H, E, k, r, q, _dt(x), renorm)
    f32 = torch.float32
    y = out if out is not None else torch.empty_like(x) if stream is None else _empty(x, (T, D), dt, stream)
    # (one expression: a check a tensor would cost a small call 2 us)
    if not (W1.dtype is US.dtype is Vt.dtype is P.dtype is Q.dtype is y.dtype is dt and W1.shape == (H, D)
            and US.shape == (D, r) and Vt.shape == (r, H) and P.shape == (E, D, q) and Q.shape == (E, q, H)
            and y.numel() == T * D and (b1 is None or (b1.numel() == H and b1.dtype is f32))
            and (b2 is None or (b2.numel() == D and b2.dtype is f32))
            and (idx_out is None or (idx_out.numel() == T * k and idx_out.dtype is torch.int32))
            and (gate_out is None or (gate_out.numel() == T * k and gate_out.dtype is f32))):
        raise ClearMoEError(f"the tensors do not fit x [{T}, {D}] {dt}, W1 [{H}, .], US [., {r}] and P [{E}, ., {q}]")
    dev = x.get_device()
    st = _queue(dev, stream)
    ws = _workspace(few_workspace_bytes(s), x, stream) if ws is None else ws
    rc = lib().clearmoe_ffn_forward_few(ctypes.byref(s), ctypes.byref(router), _ptr(x, dev), _ptr(W1, dev),
                                        _ptr(b1, dev), _ptr(US, dev), _ptr(Vt, dev), _ptr(b2, dev), _ptr(P, dev),
                                        _ptr(Q, dev), _ptr(y, dev), _ptr(idx_out, dev), _ptr(gate_out, dev),
                                        _ptr(ws, dev), ws.numel(), st)
    _check(rc, "clearmoe_ffn_forward_few")
    return y


# 8-bit formats, and the C ABI's numbers of every output type; the 4-bit format
# (two values a byte) and the scales' type, which a torch may lack: what needs
# them is refused then, the rest runs
_FORMATS = {torch.float8_e4m3fn: 2, torch.float8_e5m2: 3}
_E2M1, _E8M0 = (getattr(torch, n, n) for n in ("float4_e2m1fn_x2", "float8_e8m0fnu"))
_OUTS = {torch.float32: F32, torch.bfloat16: BF16, **_FORMATS, _E2M1: 5}


def _format(dtype) -> int:
    if not isinstance(dtype, torch.dtype) or _OUTS.get(dtype, 0) < 2:
        raise ClearMoEError(f"unsupported 8- or 4-bit format {dtype}")
    return _OUTS[dtype]


def _value_cols(cols: int, fmt=None) -> int:
    """Elements of a row of values: bytes."""
    return (cols + 31) // 32 * 16 if fmt is _E2M1 else (cols + 15) // 16 * 16


def _scale_cols(cols: int, fmt=None) -> int:
    return (cols + 127) // 128 * 4 if fmt is _E2M1 else (cols + 511) // 512 * 4


def _row_stride(x, what: str = "rows") -> int:
    """Elements between the rows of x [..., rows, cols], which may be strided."""
    if x.is_contiguous():
        return x.shape[-1]
    rows, cols = x.shape[-2:]
    batch = x.shape[0] if x.dim() == 3 else 1
    ld = x.stride(-2) if rows > 1 else x.stride(0) if batch > 1 else cols
    if x.numel() > 0 and ((cols > 1 and x.stride(-1) != 1) or (batch > 1 and x.stride(0) != rows * ld)):
        raise ClearMoEError(f"{what} must be contiguous and evenly spaced over the batch")
    if ld < cols:
        raise ClearMoEError(f"{what} must not overlap")
    return ld


def quantize(x, fmt=torch.float8_e4m3fn, block_rows: int = 1, stream=None):
    """clearmoe_quantize: x [rows, cols] or [batch, rows, cols] (rows may be
    strided) in 8-bit floating point with a power-of-two scale for each block
    of block_rows (1 or 128) x 128 values.  Returns (values [..., rows, cols up
    to a multiple of 16] in fmt, scales [..., ceil(rows / block_rows), column
    blocks up to a multiple of 4] in float8_e8m0fnu).

    fmt torch.float4_e2m1fn_x2: 4 bits, blocks of 1 x 32 (block_rows 1), values
    [..., rows, 16 ceil(cols / 32)] of two each, the even column in the low
    half; a block with a NaN or infinite value has a NaN scale."""
    shape = x.shape
    if len(shape) == 2:
        (rows, cols), batch, lead = shape, 1, ()
    elif len(shape) == 3:
        batch, rows, cols = shape
        lead = (batch,)
    else:
        raise ClearMoEError("quantize takes [rows, cols] or [batch, rows, cols]")
    ldx = cols if x.is_contiguous() else _row_stride(x)
    st = _queue(x.get_device(), stream)
    dt, code = _dt(x), _format(fmt)
    nr = rows if block_rows == 1 else -(-rows // 128)
    v = _empty(x, (*lead, rows, _value_cols(cols, fmt)), fmt, stream)
    s = _empty(x, (*lead, nr, _scale_cols(cols, fmt)), _E8M0, stream)
    rc = lib().clearmoe_quantize(dt, code, block_rows, batch, rows, cols, x.data_ptr(), ldx, v.data_ptr(),
                                 s.data_ptr(), st)
    _check(rc, "clearmoe_quantize")
    return v, s


def dequantize(values, scale, cols: Optional[int] = None, dtype=torch.bfloat16, block_rows: int = 1,
               out: Optional[torch.Tensor] = None, stream=None):
    """clearmoe_dequantize: what quantize's result stands for, [..., rows, cols]
    in float32 or bfloat16 (cols: as x had; default: the values' padded rows)."""
    shape = values.shape
    if len(shape) not in (2, 3):
        raise ClearMoEError("dequantize takes [rows, .] or [batch, rows, .]")
    batch, rows, lead = (1, shape[0], ()) if len(shape) == 2 else (shape[0], shape[1], (shape[0],))
    fmt, dev = values.dtype, values.get_device()
    code = _format(fmt)
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        raise ClearMoEError(f"unsupported dtype {dtype}")
    if cols is None:
        cols = shape[-1] * (2 if fmt is _E2M1 else 1)
    nr = rows if block_rows == 1 else -(-rows // 128)
    vp = _shaped(values, fmt, (*lead, rows, _value_cols(cols, fmt)), "values", dev)
    sp = _shaped(scale, _E8M0, (*lead, nr, _scale_cols(cols, fmt)), "scale", dev)
    st = _queue(dev, stream)
    ldy = cols
    if out is None:
        y = _empty(values, (*lead, rows, cols), dtype, stream)
    else:
        y = out
        if y.dtype is not dtype or y.shape != (*lead, rows, cols) or y.get_device() != dev:
            raise ClearMoEError(f"out must be {dtype} {(*lead, rows, cols)} on the values' device")
        ldy = _row_stride(y, "rows of out")
    rc = lib().clearmoe_dequantize(code, block_rows, batch, rows, cols, vp, sp, _OUTS[dtype], y.data_ptr(), ldy, st)
    _check(rc, "clearmoe_dequantize")
    return y


def rms_norm(x, weight=None, residual=None, eps: float = 1e-6, out_dtype=None,
             out: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None, stream=None):
    """clearmoe_rms_norm: y = h (mean(h^2) + eps)^(-1/2) weight over the rows of
    h = x + residual, x [rows, cols] (rows of x, residual, out and sum_out may
    be strided), weight [cols] float32 or None.  out_dtype: x's (the default),
    or an 8-bit format: then values and scales as quantize returns them.
    Returns y, or (values, scales); with a residual or sum_out also h, last (a
    new tensor, or sum_out, which may be x or residual itself)."""
    shape, xt = x.shape, x.dtype
    if len(shape) != 2:
        raise ClearMoEError("rms_norm takes x [rows, cols]")
    rows, cols = shape
    dt, dev, ot = _dt(x), x.get_device(), xt if out_dtype is None else out_dtype
    byte = ot is not xt
    if byte and ot not in _FORMATS:
        raise ClearMoEError(f"out_dtype must be {xt} or an 8-bit format, not {ot}")
    st = _queue(dev, stream)
    wp = None if weight is None else _shaped(weight, torch.float32, (cols,), "weight", dev)
    yshape = (rows, _value_cols(cols)) if byte else shape
    for t, what, d, size in ((residual, "residual", xt, shape), (sum_out, "sum_out", xt, shape), (out, "out", ot, yshape)):
        if t is not None and (t.dtype is not d or t.shape != size or t.get_device() != dev):
            raise ClearMoEError(f"{what} must be {d} {tuple(size)} on x's device, not {t.dtype} {tuple(t.shape)}")
    plain = x if stream is None and x.is_contiguous() else None         # (empty_like costs less)
    if sum_out is None and residual is not None:
        sum_out = torch.empty_like(x) if plain is not None else _empty(x, (rows, cols), xt, stream)
    y = (out if out is not None else torch.empty_like(x, dtype=ot) if plain is not None and yshape == shape
         else _empty(x, yshape, ot, stream))
    ys = _empty(x, (rows, _scale_cols(cols)), _E8M0, stream) if byte else None
    ld = [0 if t is None or t.is_contiguous() else _row_stride(t, what)
          for t, what in ((x, "rows of x"), (residual, "rows of residual"), (sum_out, "rows of sum_out"), (y, "rows of out"))]
    p = Norm(rows, cols, dt, _OUTS[ot], eps, *ld)
    rc = lib().clearmoe_rms_norm(ctypes.byref(p), x.data_ptr(), None if residual is None else residual.data_ptr(), wp,
                                 y.data_ptr(), None if ys is None else ys.data_ptr(),
                                 None if sum_out is None else sum_out.data_ptr(), st)
    _check(rc, "clearmoe_rms_norm")
    if sum_out is None:
        return (y, ys) if byte else y
    return (y, ys, sum_out) if byte else (y, sum_out)


def quantized_gemm(a, a_scale, b, b_scale, bias=None, gelu: bool = False, offsets=None,
                   out_dtype=torch.bfloat16, out: Optional[torch.Tensor] = None, stream=None):
    """clearmoe_quantized_gemm: a [M, K] with 1 x 128 scales times b [N, K] with
    128 x 128 scales, as quantize returns them, or, with offsets [E + 1], times
    b [E, N, K] for the rows of each expert (rows outside all groups are left
    as out had them; their scales, of an 8-bit result, are not set).  Returns C
    [M, N] in out_dtype; for an 8-bit out_dtype (values [M, N up to a multiple
    of 16], scales).  With b in 8 bits, sums of a float32 result hold every
    product; those of the others come from the 8-bit matrix instructions, which
    cut eight products at a time 14 bits below the largest.

    b in 4 bits (quantize to torch.float4_e2m1fn_x2: 1 x 32 scales): a in e4m3
    or in 4 bits too, of as many columns before their padding; out_dtype
    float32, bfloat16, e4m3 or 4 bits.  Their sums hold every product."""
    M, K = a.shape
    fa, fb = _OUTS.get(a.dtype, 0), _OUTS.get(b.dtype, 0)
    if fa < 2 or fb < 2:
        raise ClearMoEError(f"unsupported 8- or 4-bit format {a.dtype if fa < 2 else b.dtype}")
    four, out_code, shape = fb == 5, _OUTS.get(out_dtype, -1), b.shape
    if out_code < 0:
        raise ClearMoEError(f"unsupported dtype {out_dtype}")
    if fa == 5:
        K *= 2
    lead = () if offsets is None else (shape[0],)
    E, N, kb = (lead[0] if lead else 0), shape[-2], (_value_cols(K, _E2M1) if four else K)
    if shape != (*lead, N, kb):
        raise ClearMoEError(f"b must be [{'E, ' if lead else ''}N, {kb}], not {tuple(shape)}")
    dev = a.get_device()
    ap, bp = _ptr(a, dev), _ptr(b, dev)
    sap = _shaped(a_scale, _E8M0, (M, _scale_cols(K, a.dtype)), "a_scale", dev)
    sbp = _shaped(b_scale, _E8M0, (*lead, N, _scale_cols(K, _E2M1)) if four else (*lead, -(-N // 128), _scale_cols(K)),
                  "b_scale", dev)
    biasp = None if bias is None else _shaped(bias, torch.float32, (*lead, N), "bias", dev)
    offp = None if offsets is None else _shaped(offsets, torch.int32, (E + 1,), "offsets", dev)
    st = _queue(dev, stream)
    byte = out_code >= 2
    cols = _value_cols(N, out_dtype) if byte else N
    if out is None:
        c = _empty(a, (M, cols), out_dtype, stream)
        cp = c.data_ptr()
    else:
        c, cp = out, _shaped(out, out_dtype, (M, cols), "out", dev)
    cs = _empty(a, (M, _scale_cols(N, out_dtype)), _E8M0, stream) if byte else None
    p = Product(M, N, K, E, fa, fb, out_code, 1 if gelu else 0, 0, 0, 0)
    rc = lib().clearmoe_quantized_gemm(ctypes.byref(p), ap, sap, bp, sbp, biasp, offp, cp,
                                       None if cs is None else cs.data_ptr(), st)
    _check(rc, "clearmoe_quantized_gemm")
    return (c, cs) if byte else c


def quantized_workspace_bytes(shape: Shape) -> int:
    return int(lib().clearmoe_quantized_workspace_bytes(ctypes.byref(shape)))


def alloc_quantized_workspace(shape: Shape, device="cuda") -> torch.Tensor:
    return _alloc(quantized_workspace_bytes(shape), device)


def quantized_ffn_forward(x, W1, W1_scale, b1, W2, W2_scale, b2, offsets=None,
                          ws: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                          stream=None, activations=torch.float8_e4m3fn):
    """clearmoe_quantized_ffn_forward_ex: x [T, D] through an FFN with e4m3
    weights (quantize(W, block_rows=128): W1 [H, .], W2 [D, .]) or 4-bit ones
    (quantize(W, torch.float4_e2m1fn_x2)), or, with offsets [E + 1], rows sorted
    by expert through their expert's ([E, H, .], [E, D, .]; rows outside all
    groups are left as out had them).  activations: what x and the hidden
    values are rounded to, e4m3 or, with 4-bit weights, 4 bits too."""
    T, D = x.shape
    shape, fmt, f32, xt = W1.shape, W1.dtype, torch.float32, x.dtype
    lead = () if offsets is None else (shape[0],)
    E, H = (lead[0] if lead else 1), shape[-2]
    four = fmt is _E2M1
    if not four:
        fmt = torch.float8_e4m3fn
    nh, nd = (H, D) if four else (-(-H // 128), -(-D // 128))           # rows of scales
    s = Shape(T, D, H, E, 1, 0, 0, _dt(x), 1)
    dev = x.get_device()
    args = (_shaped(W1, fmt, (*lead, H, _value_cols(D, fmt)), "weights W1", dev),
            _shaped(W1_scale, _E8M0, (*lead, nh, _scale_cols(D, fmt)), "W1_scale", dev),
            None if b1 is None else _shaped(b1, f32, (*lead, H), "b1", dev),
            _shaped(W2, fmt, (*lead, D, _value_cols(H, fmt)), "weights W2", dev),
            _shaped(W2_scale, _E8M0, (*lead, nd, _scale_cols(H, fmt)), "W2_scale", dev),
            None if b2 is None else _shaped(b2, f32, (*lead, D), "b2", dev),
            None if offsets is None else _shaped(offsets, torch.int32, (E + 1,), "offsets", dev))
    fa = _format(activations)
    xp, st = _ptr(x, dev), _queue(dev, stream)
    ws = _workspace(quantized_workspace_bytes(s), x, stream) if ws is None else ws
    if out is None:
        y = torch.empty_like(x) if stream is None else _empty(x, (T, D), xt, stream)
        yp = y.data_ptr()
    else:
        y, yp = out, _shaped(out, xt, (T, D), "out", dev)
    rc = lib().clearmoe_quantized_ffn_forward_ex(ctypes.byref(s), fa, 5 if four else 2, xp, *args, yp, _ptr(ws, dev),
                                                 ws.numel(), st)
    _check(rc, "clearmoe_quantized_ffn_forward_ex")
    return y


def stage_names():
    return [lib().clearmoe_stage_name(i).decode() for i in range(N_STAGES)]


def timing_start(stages, max_records: int, every: int = 1) -> None:
    """Time every every-th launch of the named stages (at most max_records
    timed launches)."""
    names = stage_names()
    mask = 0
    for s in stages:
        mask |= 1 << names.index(s)
    _check(lib().clearmoe_timing_start_sampled(mask, int(max_records), int(every)),
           "clearmoe_timing_start_sampled")


def timing_stop() -> dict:
    """Stop timing; {stage: (total_ms, launches)} for the stages that ran."""
    ms = (ctypes.c_double * N_STAGES)()
    n = (ctypes.c_int32 * N_STAGES)()
    _check(lib().clearmoe_timing_stop(ms, n), "clearmoe_timing_stop")
    return {name: (ms[i], n[i]) for i, name in enumerate(stage_names()) if n[i] > 0}


def from_stored(a: np.ndarray, device="cuda") -> torch.Tensor:
    """Stored host array -> device tensor: uint16 = bfloat16 bits, float32, int32."""
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16).to(device)
    return torch.from_numpy(a).to(device)


def to_stored(t: torch.Tensor) -> np.ndarray:
    """Device tensor -> host array in the stored convention (bf16 -> uint16 bits)."""
    t = t.detach().cpu().contiguous()
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).numpy().view(np.uint16)
    return t.numpy()
