"""ctypes binding of libjetvit.so: same names as the C ABI, argument marshalling
only.  Tensors are CUDA ``torch`` tensors (device memory and streams come from
PyTorch); every step of every mixer runs in the library's CUDA kernels.  There
is no CPU path: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

JV_OK, JV_ERR_INVALID_ARG, JV_ERR_UNSUPPORTED, JV_ERR_WORKSPACE, JV_ERR_CUDA, JV_ERR_TIMEOUT = range(6)
JV_F32, JV_BF16 = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
# JETVIT_LIB selects another build of the same library (e.g. one compiled with other tuning macros)
LIB_PATH = os.environ.get("JETVIT_LIB") or os.path.join(_HERE, "libjetvit.so")


class JvShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hg", ctypes.c_int32),
                ("Wg", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("P", ctypes.c_int32),
                ("in_layout", ctypes.c_int32), ("in_tok_stride", ctypes.c_int64)]


class JvDwc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int32), ("R", ctypes.c_int32), ("W1", ctypes.c_void_p),
                ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p), ("b2", ctypes.c_void_p),
                ("token_wise", ctypes.c_int32)]


class JvNormShape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("x_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64)]


class JvDiffShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "Hkv", "Nq", "Nk", "D", "dtype", "causal")] + [
        ("q_stride", ctypes.c_int64 * 3), ("kv_stride", ctypes.c_int64 * 3)]


class JvDiff(ctypes.Structure):
    _fields_ = [("lam", ctypes.c_void_p), ("lambda_init", ctypes.c_float), ("norm_w", ctypes.c_void_p),
                ("norm_eps", ctypes.c_float), ("kv_len", ctypes.c_void_p), ("q_pos", ctypes.c_void_p)]


class JvConvShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "C", "K", "dtype", "silu")] + [("x_stride", ctypes.c_int64 * 2)]


class JvScanShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "C", "Ns", "dtype", "softplus")] + [
        (n, ctypes.c_int64 * 2) for n in ("u_stride", "dt_stride", "b_stride", "c_stride", "z_stride")]


_DwcPtrs = ctypes.POINTER(ctypes.POINTER(JvDwc))


class JetVitError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (jv_status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libjetvit.so (built in-tree by ``paper_2605_26636_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2605_26636_b200.build` "
                              "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, i32, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_float
        shp, dwc = ctypes.POINTER(JvShape), ctypes.POINTER(JvDwc)
        L.jv_workspace_bytes.argtypes = [ctypes.c_char, shp, dwc]
        L.jv_workspace_bytes.restype = sz
        L.jv_linear_attn.argtypes = [vp, vp, vp, vp, shp, f32, dwc, vp, sz, vp]
        L.jv_linear_attn_focused.argtypes = [vp, vp, vp, vp, shp, f32, f32, dwc, vp, sz, vp]
        L.jv_linear_attn_focused.restype = ctypes.c_int
        L.jv_linear_attn_static.argtypes = [vp, vp, vp, vp, shp, f32, dwc, vp]
        L.jv_linear_attn_static.restype = ctypes.c_int
        L.jv_window_attn.argtypes = [vp, vp, vp, vp, shp, i32, i32, f32, vp, sz, vp]
        L.jv_full_attn.argtypes = [vp, vp, vp, vp, shp, f32, vp, sz, vp]
        L.jv_hybrid_mixers.argtypes = [i32, ctypes.c_char_p, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                       ctypes.POINTER(vp), ctypes.POINTER(vp), shp, i32, i32, f32, f32,
                                       ctypes.POINTER(dwc), vp, sz, vp]
        L.jv_device_status.argtypes = [vp]
        L.jv_selftest_wait_timeout.argtypes = [ctypes.c_uint32, vp, vp]
        L.jv_selftest_wait_timeout.restype = ctypes.c_int
        L.jv_qkv_proj.argtypes = [vp, vp, vp, vp, vp, vp, shp, vp]
        L.jv_out_proj.argtypes = [vp, vp, vp, vp, shp, vp]
        nshp = ctypes.POINTER(JvNormShape)
        L.jv_layer_norm.argtypes = [vp, vp, vp, vp, vp, vp, nshp, f32, vp]
        L.jv_layer_norm_grad_workspace_bytes.argtypes = [nshp]
        L.jv_layer_norm_grad_workspace_bytes.restype = sz
        L.jv_layer_norm_grad.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, nshp, vp, sz, vp]
        dshp, cshp, sshp = ctypes.POINTER(JvDiffShape), ctypes.POINTER(JvConvShape), ctypes.POINTER(JvScanShape)
        L.jv_diff_attn_workspace_bytes.argtypes = [dshp]
        L.jv_diff_attn_workspace_bytes.restype = sz
        L.jv_diff_attn.argtypes = [vp, vp, vp, vp, dshp, ctypes.POINTER(JvDiff), f32, vp, sz, vp]
        L.jv_causal_conv.argtypes = [vp, vp, vp, vp, vp, vp, vp, cshp, vp]
        L.jv_selective_scan_workspace_bytes.argtypes = [sshp]
        L.jv_selective_scan_workspace_bytes.restype = sz
        L.jv_selective_scan.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sshp, vp, sz, vp]
        for f in (L.jv_linear_attn, L.jv_window_attn, L.jv_full_attn, L.jv_hybrid_mixers, L.jv_device_status,
                  L.jv_qkv_proj, L.jv_out_proj, L.jv_layer_norm, L.jv_layer_norm_grad, L.jv_diff_attn,
                  L.jv_causal_conv, L.jv_selective_scan):
            f.restype = ctypes.c_int
        L.jv_set_force_generic.argtypes = [i32]
        L.jv_set_force_generic.restype = i32
        L.jv_launch_count.restype = ctypes.c_uint64
        L.jv_status_string.argtypes = [ctypes.c_int]
        L.jv_status_string.restype = ctypes.c_char_p
        L.jv_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().jv_status_string(int(status)).decode()


def version() -> str:
    return lib().jv_version().decode()


def launch_count() -> int:
    return int(lib().jv_launch_count())


def set_force_generic(on: bool) -> bool:
    return bool(lib().jv_set_force_generic(1 if on else 0))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return JV_F32
    if t.dtype == torch.bfloat16:
        return JV_BF16
    raise TypeError(f"dtype {t.dtype}: the mixers take float32 or bfloat16")


JV_LAYOUT_BHND, JV_LAYOUT_BNHD = 0, 1


def _in_layout(t: torch.Tensor):
    """(jv_layout, token stride) of an input tensor of logical shape [B, H, N, D]: contiguous, or a
    [B, N, H, D] array seen through ``permute(0, 2, 1, 3)`` whose token rows are ``stride(2)`` elements
    apart, e.g. ``qkv[:, :, i].permute(0, 2, 1, 3)`` of a fused [B, N, 3, H, D] activation."""
    if t.is_contiguous():
        return JV_LAYOUT_BHND, 0
    B, H, N, D = t.shape
    sb, sh, sn, sd = t.stride()
    if sd == 1 and sh == D and sn >= H * D and (sb == N * sn or B == 1):
        return JV_LAYOUT_BNHD, sn
    raise ValueError("inputs must be contiguous [B,H,N,D] tensors or permuted views of [B,N,H,D] token rows")


def make_shape(t: torch.Tensor, Hg: int, Wg: int, prefix: int = 0) -> JvShape:
    """Shape of [B, H, prefix + Hg*Wg, D] tensors: ``prefix`` tokens (class / register tokens) in
    front of the grid tokens.  The layout of the inputs is taken from ``t`` (see ``_in_layout``)."""
    B, H, N, D = t.shape
    if prefix < 0 or N != prefix + Hg * Wg:
        raise ValueError(f"N = {N} is not prefix + Hg*Wg = {prefix} + {Hg}*{Wg}")
    layout, tok_stride = _in_layout(t)
    return JvShape(B, H, Hg, Wg, D, _dtype_code(t), prefix, layout, tok_stride)


def _check_tensors(*ts: torch.Tensor):
    """q, k, v[, o]: one shape, dtype and device; q, k, v in one layout; o (a fourth tensor) contiguous."""
    ref = ts[0]
    shape, dtype, dev, dense, strides = ref.shape, ref.dtype, ref.get_device(), ref.is_contiguous(), ref.stride()
    for i, t in enumerate(ts):
        # these cheap attributes settle nearly every call; what they do not settle goes through the checks below, one by one
        if dev >= 0 and t.shape == shape and t.dtype is dtype and t.get_device() == dev \
                and (t.is_contiguous() if dense or i >= 3 else t.stride() == strides):
            continue
        if not t.is_cuda:
            raise ValueError("tensors must live on a CUDA device (there is no CPU path)")
        if t.shape != shape or t.dtype != dtype or t.device != ref.device:
            raise ValueError("q, k, v, o must be [B,H,N,D] tensors of one shape, dtype and device")
        if i < 3 and _in_layout(t) != _in_layout(ref):
            raise ValueError("q, k and v must share one layout (all contiguous, or all views with the same token stride)")
        if i >= 3 and not t.is_contiguous():
            raise ValueError("o must be a contiguous [B,H,N,D] tensor")


class _current_device:
    """``with torch.cuda.device(d)`` that costs nothing when d is the current device already."""
    __slots__ = ("ctx",)

    def __init__(self, device: torch.device):
        self.ctx = None if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def _empty_out(q: torch.Tensor) -> torch.Tensor:
    return torch.empty(q.shape, dtype=q.dtype, device=q.device)


def make_dwc(d: Optional[dict], device) -> Optional[JvDwc]:
    """dict(k, R, W1, b1, W2, b2) of fp32 CUDA tensors -> jv_dwc.  The dict must stay
    alive until the call has been enqueued."""
    if d is None:
        return None
    static = int(d["R"]) == 0          # static kernels in b2: no generator weights
    for key in (("b2",) if static else ("W1", "W2")):
        t = d.get(key)
        if t is None or not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
            raise ValueError(f"dwc[{key!r}] must be a contiguous fp32 CUDA tensor")
    ptr = lambda t: None if t is None else t.data_ptr()
    return JvDwc(int(d["k"]), int(d["R"]), ptr(d.get("W1")), ptr(d.get("b1")), ptr(d.get("W2")), ptr(d.get("b2")),
                 int(d.get("token_wise", 0)))


# the current stream's handle without building a Stream object, where torch has the call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def workspace_bytes(mixer: str, shape: JvShape, dwc: Optional[JvDwc] = None) -> int:
    return int(lib().jv_workspace_bytes(mixer.encode()[:1], ctypes.byref(shape),
                                        ctypes.byref(dwc) if dwc is not None else None))


def alloc_workspace(mixer: str, shape: JvShape, dwc: Optional[JvDwc], device) -> Optional[torch.Tensor]:
    n = workspace_bytes(mixer, shape, dwc)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device) if n else None


def _ws_args(ws: Optional[torch.Tensor]):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


def _raise(status: int, where: str):
    if status != JV_OK:
        raise JetVitError(status, where)


def linear_attn(q, k, v, Hg: int, Wg: int, eps: float = 1e-6, dwc: Optional[dict] = None, out=None,
                ws: Optional[torch.Tensor] = None, stream=None, prefix: int = 0) -> torch.Tensor:
    """jv_linear_attn.  Allocates ``out`` / ``ws`` with torch when not given."""
    out = _empty_out(q) if out is None else out
    _check_tensors(q, k, v, out)
    shape = make_shape(q, Hg, Wg, prefix)
    d = make_dwc(dwc, q.device)
    with _current_device(q.device):
        if ws is None:
            ws = alloc_workspace("L", shape, d, q.device)
            if ws is not None and stream is not None:
                ws.record_stream(stream)      # freed by torch on the current stream, used on `stream`
        wp, wn = _ws_args(ws)
        st = lib().jv_linear_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ctypes.byref(shape),
                                  float(eps), ctypes.byref(d) if d is not None else None, wp, wn, _stream(stream))
    _raise(st, "jv_linear_attn")
    return out


def linear_attn_focused(q, k, v, Hg: int, Wg: int, focus_p: float, eps: float = 1e-6, dwc: Optional[dict] = None,
                        out=None, ws: Optional[torch.Tensor] = None, stream=None, prefix: int = 0) -> torch.Tensor:
    """jv_linear_attn_focused: the linear block with the focused feature map of Eq. 3 (power focus_p)."""
    out = _empty_out(q) if out is None else out
    _check_tensors(q, k, v, out)
    shape = make_shape(q, Hg, Wg, prefix)
    d = make_dwc(dwc, q.device)
    with _current_device(q.device):
        if ws is None:
            ws = alloc_workspace("f", shape, d, q.device)
            if ws is not None and stream is not None:
                ws.record_stream(stream)
        wp, wn = _ws_args(ws)
        st = lib().jv_linear_attn_focused(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ctypes.byref(shape),
                                          float(eps), float(focus_p), ctypes.byref(d) if d is not None else None, wp, wn,
                                          _stream(stream))
    _raise(st, "jv_linear_attn_focused")
    return out


STATIC_SCRATCH_BYTES = 16 << 20


def linear_attn_static(q, k, v, Hg: int, Wg: int, eps: float = 1e-6, dwc: Optional[dict] = None, *, out,
                       stream=None, prefix: int = 0) -> torch.Tensor:
    """jv_linear_attn_static: the linear block with the library's built-in scratch, for
    callers that must not allocate.  This wrapper allocates nothing either: ``out`` is
    required.  Problems needing more than STATIC_SCRATCH_BYTES raise JV_ERR_WORKSPACE;
    calls that can overlap on the GPU must be ordered by the caller (they share the scratch)."""
    _check_tensors(q, k, v, out)
    shape = make_shape(q, Hg, Wg, prefix)
    d = make_dwc(dwc, q.device)
    with _current_device(q.device):
        st = lib().jv_linear_attn_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                         ctypes.byref(shape), float(eps),
                                         ctypes.byref(d) if d is not None else None, _stream(stream))
    _raise(st, "jv_linear_attn_static")
    return out


def window_attn(q, k, v, Hg: int, Wg: int, win_h: int, win_w: int, scale: float = 0.0, out=None,
                stream=None, prefix: int = 0) -> torch.Tensor:
    """jv_window_attn (scale <= 0: 1/sqrt(D))."""
    out = _empty_out(q) if out is None else out
    _check_tensors(q, k, v, out)
    shape = make_shape(q, Hg, Wg, prefix)
    with _current_device(q.device):
        st = lib().jv_window_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ctypes.byref(shape),
                                  int(win_h), int(win_w), float(scale), None, 0, _stream(stream))
    _raise(st, "jv_window_attn")
    return out


def full_attn(q, k, v, Hg: Optional[int] = None, Wg: Optional[int] = None, scale: float = 0.0, out=None,
              stream=None) -> torch.Tensor:
    """jv_full_attn (scale <= 0: 1/sqrt(D)).  The grid split of N is irrelevant to F."""
    out = _empty_out(q) if out is None else out
    _check_tensors(q, k, v, out)
    if Hg is None or Wg is None:
        Hg, Wg = 1, q.shape[2]
    shape = make_shape(q, Hg, Wg)
    with _current_device(q.device):
        st = lib().jv_full_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ctypes.byref(shape),
                                float(scale), None, 0, _stream(stream))
    _raise(st, "jv_full_attn")
    return out


def hybrid_mixers(schedule: str, q: Sequence[torch.Tensor], k, v, Hg: int, Wg: int, win_h: int, win_w: int,
                  scale: float = 0.0, eps: float = 1e-6, dwc: Optional[Sequence[Optional[dict]]] = None,
                  out: Optional[Sequence[torch.Tensor]] = None, ws: Optional[torch.Tensor] = None, stream=None,
                  prefix: int = 0):
    """jv_hybrid_mixers: one mixer per layer, schedule[l] in 'L', 'W', 'F'."""
    n = len(schedule)
    if not (len(q) == len(k) == len(v) == n):
        raise ValueError("need one q, k, v per schedule entry")
    out = [_empty_out(t) for t in q] if out is None else list(out)
    q0 = q[0] if n else None
    for l in range(n):
        _check_tensors(q[l], k[l], v[l], out[l])
        if l and (q[l].shape != q0.shape or q[l].dtype != q0.dtype
                  or q[l].stride() != q0.stride() and _in_layout(q[l]) != _in_layout(q0)):
            raise ValueError("all layers share one shape, dtype and input layout")
    shape = make_shape(q[0], Hg, Wg, prefix)
    vps = ctypes.c_void_p * n
    arr = lambda ts: vps(*[t.data_ptr() for t in ts])
    dstructs = [make_dwc(d, q[0].device) for d in dwc] if dwc is not None else None
    dptr = None
    if dstructs is not None:
        dptr = ctypes.cast(vps(*[None if d is None else ctypes.addressof(d) for d in dstructs]), _DwcPtrs)
    with _current_device(q[0].device):
        if ws is None:
            need = 0
            for l, m in enumerate(schedule):
                if m == "L":
                    need = max(need, workspace_bytes("L", shape, dstructs[l] if dstructs else None))
            ws = torch.empty(max(need, 256), dtype=torch.uint8, device=q[0].device) if need else None
            if ws is not None and stream is not None:
                ws.record_stream(stream)      # freed by torch on the current stream, used on `stream`
        wp, wn = _ws_args(ws)
        st = lib().jv_hybrid_mixers(n, schedule.encode(), arr(q), arr(k), arr(v), arr(out), ctypes.byref(shape),
                                    int(win_h), int(win_w), float(scale), float(eps), dptr, wp, wn, _stream(stream))
    _raise(st, "jv_hybrid_mixers")
    return out


def _check_proj(x, w, bias, H: int, rows: int):
    C = 64 * H
    for t in (x, w):
        if not (t.is_cuda and t.dtype == torch.bfloat16 and t.is_contiguous()):
            raise ValueError("projection operands must be contiguous bf16 CUDA tensors")
    if tuple(w.shape) != (rows, C):
        raise ValueError(f"w must be [{rows}, {C}]")
    if bias is not None and not (bias.is_cuda and bias.dtype == torch.float32 and bias.is_contiguous()
                                 and tuple(bias.shape) == (rows,)):
        raise ValueError(f"bias must be a contiguous fp32 CUDA tensor of [{rows}]")


def qkv_proj(x, w, bias, H: int, Hg: int, Wg: int, out=None, stream=None, prefix: int = 0):
    """jv_qkv_proj: x [B, N, C] bf16, w [3C, C] bf16, bias fp32 [3C] or None -> (q, k, v), each
    [B, H, N, 64] in the mixers' layout.  ``out`` is an optional (q, k, v) triple to write into."""
    B, N, C = x.shape
    if C != 64 * H or N != prefix + Hg * Wg:
        raise ValueError("x must be [B, prefix + Hg*Wg, 64*H]")
    _check_proj(x, w, bias, H, 3 * C)
    q, k, v = out if out is not None else (torch.empty((B, H, N, 64), dtype=x.dtype, device=x.device) for _ in range(3))
    for t in (q, k, v):            # outputs: written contiguously, whatever layout the mixers take as inputs
        if not (t.is_cuda and t.is_contiguous() and tuple(t.shape) == (B, H, N, 64) and t.dtype == x.dtype and t.device == x.device):
            raise ValueError("q, k, v must be contiguous [B, H, N, 64] bf16 tensors on x's device")
    shape = JvShape(B, H, Hg, Wg, 64, JV_BF16, prefix)
    with _current_device(x.device):
        st = lib().jv_qkv_proj(x.data_ptr(), w.data_ptr(), None if bias is None else bias.data_ptr(), q.data_ptr(),
                               k.data_ptr(), v.data_ptr(), ctypes.byref(shape), _stream(stream))
    _raise(st, "jv_qkv_proj")
    return q, k, v


def out_proj(o, w, bias, Hg: int, Wg: int, out=None, stream=None, prefix: int = 0) -> torch.Tensor:
    """jv_out_proj: o [B, H, N, 64] bf16 (a mixer's output), w [C, C] bf16, bias fp32 [C] or None
    -> y [B, N, C]."""
    B, H, N, D = o.shape
    if D != 64 or N != prefix + Hg * Wg:
        raise ValueError("o must be [B, H, prefix + Hg*Wg, 64]")
    C = 64 * H
    _check_proj(o, w, bias, H, C)
    y = torch.empty((B, N, C), dtype=o.dtype, device=o.device) if out is None else out
    if not (y.is_cuda and y.is_contiguous() and tuple(y.shape) == (B, N, C) and y.dtype == o.dtype):
        raise ValueError("y must be a contiguous [B, N, C] bf16 CUDA tensor")
    shape = JvShape(B, H, Hg, Wg, 64, JV_BF16, prefix)
    with _current_device(o.device):
        st = lib().jv_out_proj(o.data_ptr(), w.data_ptr(), None if bias is None else bias.data_ptr(), y.data_ptr(),
                               ctypes.byref(shape), _stream(stream))
    _raise(st, "jv_out_proj")
    return y


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The calls from here on are used token by token, where the checks of their arguments would take longer than their kernels: they
# look at each attribute once, and at the device by its index (-1: not a CUDA tensor).
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32


def _index(t: torch.Tensor) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError("tensors must live on a CUDA device (there is no CPU path)")
    return dev


def _like(t: Optional[torch.Tensor], shape, dtype, dev: int, what: str):
    """``t`` (or None) has to be a contiguous tensor of that shape and type on the call's device."""
    if t is not None and not (t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} CUDA tensor of {list(shape)} on the call's device")


def _per_row(t: Optional[torch.Tensor], n: int, dtype, dev: int, what: str):
    if t is None or not (t.dtype is dtype and t.numel() == n and t.get_device() == dev and t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} CUDA tensor of {n} elements on the call's device")


def _enqueue(dev: int, stream, call):
    """call(stream handle) with the tensors' device current."""
    if dev == _get_device():
        return call(stream.cuda_stream if stream is not None else _raw_stream(dev) if _raw_stream is not None else _stream(None))
    with torch.cuda.device(dev):
        return call(_stream(stream))


def _new(shape, dtype, device, stream) -> torch.Tensor:
    """A tensor that the call writes, from the memory of the stream that it runs on: what is free there, no earlier work of
    another stream still uses."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _scratch(n: int, device, stream) -> Optional[torch.Tensor]:
    return _new(n, torch.uint8, device, stream) if n else None


def _rows(t: torch.Tensor, what: str):
    """(rows, C, elements between rows) of a [..., C] tensor whose rows lie evenly spaced."""
    n = t.numel()
    if n == 0 or t.dim() < 1:
        raise ValueError(f"{what} must be a [..., C] tensor that is not empty")
    C = t.shape[-1]
    if t.is_contiguous():
        return n // C, C, 0
    try:
        flat = t.view(-1, C)
    except RuntimeError:
        flat = None
    if flat is None or (C > 1 and flat.stride(1) != 1) or (flat.shape[0] > 1 and flat.stride(0) < C):
        raise ValueError(f"the rows of {what} must be contiguous, evenly spaced and apart from each other")
    return flat.shape[0], C, flat.stride(0) if flat.shape[0] > 1 else 0


def layer_norm(x, weight=None, bias=None, eps: float = 1e-6, out=None, stats=None, stream=None) -> torch.Tensor:
    """jv_layer_norm over the last axis of ``x`` (f32 or bf16, [..., C]; rows evenly spaced); ``weight`` and ``bias`` fp32 [C] or
    None.  ``stats``: an optional pair of fp32 tensors of one element per row that receive mean and 1 / standard
    deviation, which layer_norm_grad takes."""
    dev = _index(x)
    rows, C, stride = _rows(x, "x")
    vec = (C,)
    _like(weight, vec, _F32, dev, "weight")
    _like(bias, vec, _F32, dev, "bias")
    mean = rstd = None
    if stats is not None:
        mean, rstd = stats
        _per_row(mean, rows, _F32, dev, "stats")
        _per_row(rstd, rows, _F32, dev, "stats")
    if out is None:
        out = _new(x.shape, x.dtype, x.device, stream)
    else:
        _like(out, x.shape, x.dtype, dev, "out")
    shape = JvNormShape(rows, C, _dtype_code(x), stride)
    st = _enqueue(dev, stream, lambda s: lib().jv_layer_norm(
        x.data_ptr(), _ptr(weight), _ptr(bias), out.data_ptr(), _ptr(mean), _ptr(rstd), ctypes.byref(shape), eps, s))
    _raise(st, "jv_layer_norm")
    return out


def layer_norm_grad(dy, x, weight, mean, rstd, weight_grad: bool = True, bias_grad: bool = True, out=None,
                    ws: Optional[torch.Tensor] = None, stream=None):
    """jv_layer_norm_grad: (dx, dw, db) of layer_norm from ``dy`` and what the forward pass left in ``stats``.  dw and db are fp32
    [C], None where not wanted.  ``out``: an optional (dx, dw, db) to write into."""
    dev = _index(x)
    rows, C, stride = _rows(x, "x")
    if dy.shape != x.shape or dy.dtype is not x.dtype or dy.get_device() != dev:
        raise ValueError("dy must have x's shape, dtype and device")
    vec = (C,)
    _like(weight, vec, _F32, dev, "weight")
    _per_row(mean, rows, _F32, dev, "mean")
    _per_row(rstd, rows, _F32, dev, "rstd")
    if out is None:
        new = lambda want: _new(C, _F32, x.device, stream) if want else None
        dx, dw, db = out = (_new(x.shape, x.dtype, x.device, stream), new(weight_grad), new(bias_grad))
    else:
        dx, dw, db = out
        _like(dx, x.shape, x.dtype, dev, "dx")
        _like(dw, vec, _F32, dev, "dw")
        _like(db, vec, _F32, dev, "db")
    shape = JvNormShape(rows, C, _dtype_code(x), stride, _rows(dy, "dy")[2])

    def call(s):
        scratch = ws
        if scratch is None and (dw is not None or db is not None):
            scratch = _scratch(int(lib().jv_layer_norm_grad_workspace_bytes(ctypes.byref(shape))), x.device, stream)
        wp, wn = _ws_args(scratch)
        return lib().jv_layer_norm_grad(dy.data_ptr(), x.data_ptr(), _ptr(weight), mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(),
                                        _ptr(dw), _ptr(db), ctypes.byref(shape), wp, wn, s)

    _raise(_enqueue(dev, stream, call), "jv_layer_norm_grad")
    return dx, dw, db


def _head_strides(t: torch.Tensor, what: str):
    """Elements between {tokens, heads, batch elements} of a [B, H, N, D] tensor; None where it is contiguous."""
    if t.is_contiguous():
        return None
    B, H, N, D = t.shape
    sb, sh, sn, sd = t.stride()
    if sd != 1 and D > 1:
        raise ValueError(f"the channels of {what} must be contiguous")
    e = max(D, 16 // t.element_size())                 # where there is one of something, any step does
    sn, sh, sb = sn if N > 1 else e, sh if H > 1 else e, sb if B > 1 else e
    if sn <= 0 or sh <= 0 or sb <= 0:
        raise ValueError(f"{what} must not repeat its rows")
    return sn, sh, sb


def diff_attn(q, k, v, lam, lambda_init: float, norm_weight=None, norm_eps: float = 1e-5, causal: bool = False, kv_len=None,
              q_pos=None, scale: float = 0.0, out=None, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """jv_diff_attn: q [B, H, Nq, D], k and v [B, Hkv, Nk, D], heads in pairs; any strides with contiguous channels, k and v
    alike.  ``lam``: the four learned vectors, fp32 [4, D]; ``norm_weight``: fp32 [2 D] or None; ``kv_len``, ``q_pos``: int32 [B] or None."""
    dev, dtype, qs, kvs = _index(q), q.dtype, q.shape, k.shape
    if len(qs) != 4 or len(kvs) != 4 or v.shape != kvs or qs[0] != kvs[0] or qs[3] != kvs[3]:
        raise ValueError("q must be [B, H, Nq, D], k and v [B, Hkv, Nk, D]")
    if k.dtype is not dtype or v.dtype is not dtype or k.get_device() != dev or v.get_device() != dev:
        raise ValueError("q, k and v must have one dtype and device")
    B, H, Nq, D = qs
    shape = JvDiffShape(B, H, kvs[1], Nq, kvs[2], D, _dtype_code(q), 1 if causal else 0)
    strides = _head_strides(k, "k")
    if _head_strides(v, "v") != strides:
        raise ValueError("k and v must have the same strides")
    if strides is not None:
        shape.kv_stride = strides
    strides = _head_strides(q, "q")
    if strides is not None:
        shape.q_stride = strides
    _like(lam, (4, D), _F32, dev, "lam")
    _like(norm_weight, (2 * D,), _F32, dev, "norm_weight")
    if kv_len is not None:
        _per_row(kv_len, B, _I32, dev, "kv_len")
    if q_pos is not None:
        _per_row(q_pos, B, _I32, dev, "q_pos")
    d = JvDiff(lam.data_ptr(), lambda_init, _ptr(norm_weight), norm_eps, _ptr(kv_len), _ptr(q_pos))
    if out is None:
        out = _new(qs, dtype, q.device, stream)
    else:
        _like(out, qs, dtype, dev, "out")

    def call(s):
        L = lib()
        scratch = _scratch(L.jv_diff_attn_workspace_bytes(ctypes.byref(shape)), q.device, stream) if ws is None else ws
        wp, wn = _ws_args(scratch)
        return L.jv_diff_attn(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ctypes.byref(shape), ctypes.byref(d),
                              scale, wp, wn, s)

    _raise(_enqueue(dev, stream, call), "jv_diff_attn")
    return out


def _token_rows(t: torch.Tensor, shape, dtype, dev: int, what: str):
    """Elements between {token rows, batch elements} of a [B, L, C] tensor; None where it is contiguous."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{what} must be {list(shape)}, of one dtype and device with the others")
    if t.is_contiguous():
        return None
    B, L, C = shape
    sb, sl, sc = t.stride()
    row = sl if L > 1 else C
    batch = sb if B > 1 else L * row
    if (sc != 1 and C > 1) or row < C or batch <= 0:
        raise ValueError(f"the token rows of {what} must be contiguous, evenly spaced and apart from each other")
    return row, batch


def causal_conv(x, weight, bias=None, state=None, state_out=None, lens=None, silu: bool = True, out=None, stream=None) -> torch.Tensor:
    """jv_causal_conv: x [B, L, C] (token rows evenly spaced), ``weight`` fp32 [C, K], ``bias`` fp32 [C] or None; ``state`` (in) and
    ``state_out`` (may be the same tensor) [B, K - 1, C] of x's dtype; ``lens`` int32 [B].  Rows of ``out`` behind a sequence stay as
    they are (so pass one where that matters)."""
    dev, dtype, xs = _index(x), x.dtype, x.shape
    if len(xs) != 3 or weight.dim() != 2:
        raise ValueError("x must be [B, L, C] and weight [C, K]")
    B, L, C = xs
    K = weight.shape[1]
    shape = JvConvShape(B, L, C, K, _dtype_code(x), 1 if silu else 0)
    strides = _token_rows(x, xs, dtype, dev, "x")
    if strides is not None:
        shape.x_stride = strides
    _like(weight, (C, K), _F32, dev, "weight")
    _like(bias, (C,), _F32, dev, "bias")
    _like(state, (B, K - 1, C), dtype, dev, "state")
    if state_out is not state:
        _like(state_out, (B, K - 1, C), dtype, dev, "state_out")
    if lens is not None:
        _per_row(lens, B, _I32, dev, "lens")
    if out is None:
        out = _new(xs, dtype, x.device, stream)
    else:
        _like(out, xs, dtype, dev, "out")
    st = _enqueue(dev, stream, lambda s: lib().jv_causal_conv(
        x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(state), out.data_ptr(), _ptr(state_out), _ptr(lens), ctypes.byref(shape), s))
    _raise(st, "jv_causal_conv")
    return out


def selective_scan(u, dt, A, Bm, Cm, D=None, z=None, dt_bias=None, state=None, state_out=None, lens=None, softplus: bool = True,
                   out=None, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """jv_selective_scan: u, dt, z [B, L, C], Bm, Cm [B, L, Ns] (token rows evenly spaced), A fp32 [C, Ns], D and dt_bias fp32 [C] or None;
    ``state`` (in) and ``state_out`` (may be the same tensor) fp32 [B, C, Ns]; ``lens`` int32 [B].  Rows of ``out`` behind a sequence
    stay as they are."""
    dev, dtype, us = _index(u), u.dtype, u.shape
    if len(us) != 3 or A.dim() != 2:
        raise ValueError("u must be [B, L, C] and A [C, Ns]")
    B, L, C = us
    Ns = A.shape[1]
    bs, vec, hs = (B, L, Ns), (C,), (B, C, Ns)
    shape = JvScanShape(B, L, C, Ns, _dtype_code(u), 1 if softplus else 0)
    for field, t, want in (("u_stride", u, us), ("dt_stride", dt, us), ("b_stride", Bm, bs), ("c_stride", Cm, bs), ("z_stride", z, us)):
        if t is not None or field != "z_stride":
            strides = _token_rows(t, want, dtype, dev, field[:-7])
            if strides is not None:
                setattr(shape, field, strides)
    _like(A, (C, Ns), _F32, dev, "A")
    _like(D, vec, _F32, dev, "D")
    _like(dt_bias, vec, _F32, dev, "dt_bias")
    _like(state, hs, _F32, dev, "state")
    if state_out is not state:
        _like(state_out, hs, _F32, dev, "state_out")
    if lens is not None:
        _per_row(lens, B, _I32, dev, "lens")
    if out is None:
        out = _new(us, dtype, u.device, stream)
    else:
        _like(out, us, dtype, dev, "out")

    def call(s):
        lb = lib()
        scratch = ws
        if scratch is None and L > 1:                  # (single tokens need none)
            scratch = _scratch(lb.jv_selective_scan_workspace_bytes(ctypes.byref(shape)), u.device, stream)
        wp, wn = _ws_args(scratch)
        return lb.jv_selective_scan(u.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _ptr(D), _ptr(z),
                                    _ptr(dt_bias), _ptr(state), out.data_ptr(), _ptr(state_out), _ptr(lens), ctypes.byref(shape),
                                    wp, wn, s)

    _raise(_enqueue(dev, stream, call), "jv_selective_scan")
    return out


def selftest_wait_timeout(limit_us: int, gave_up: Optional[torch.Tensor] = None, stream=None) -> None:
    """jv_selftest_wait_timeout: enqueues a kernel whose bounded wait runs out after ``limit_us``
    microseconds and sets the sticky status word.  ``gave_up``: optional int32 CUDA tensor (1 element)."""
    st = lib().jv_selftest_wait_timeout(int(limit_us), None if gave_up is None else gave_up.data_ptr(),
                                        _stream(stream))
    _raise(st, "jv_selftest_wait_timeout")


def device_status(stream=None) -> int:
    """jv_device_status: synchronises the stream and returns the sticky status."""
    return int(lib().jv_device_status(_stream(stream)))
