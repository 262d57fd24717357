"""ctypes binding of liballegro_latent.so -- argument marshalling only.

The operators of the scalar (latent) track, declared in include/allegro_latent.h: rows grouped by
type, products per type, the root-mean-square norm with the residual's addition, and 8-bit products.
Functions have the names of the C entry points; like those of the tensor product they check shapes,
dtypes and devices, allocate with PyTorch what the caller does not pass, and hand raw pointers and
the current HIP stream to the library.  Tensors of rows may be views with a row stride.  There is no
fallback: without the compiled library importing this module raises.
"""

from __future__ import annotations

import ctypes
import os

import torch

from .binding import ALLEGRO_OK, AllegroError, _need, _ptr, _stream

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liballegro_latent.so")

ALLEGRO_F32 = 0
ALLEGRO_BF16 = 1
ALLEGRO_ACT_NONE = 0
ALLEGRO_ACT_SILU = 1
SCALE_BLOCK = 128  # columns (and rows of W) that share a scale

EXPORTED = (
    "allegro_latent_last_error", "allegro_group_rows_workspace", "allegro_group_rows", "allegro_grouped_matmul",
    "allegro_grouped_matmul_workspace", "allegro_grouped_matmul_backward", "allegro_rms_norm_forward",
    "allegro_rms_norm_fp8", "allegro_rms_norm_workspace", "allegro_rms_norm_backward", "allegro_grouped_matmul_fp8",
)


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run paper_2504_16068_amd.build_latent.build() or "
                          "__graft_entry__.build() first (there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    szp = ctypes.POINTER(sz)
    lib.allegro_latent_last_error.argtypes = []
    lib.allegro_latent_last_error.restype = ctypes.c_char_p
    lib.allegro_group_rows_workspace.argtypes = [i64, i32, szp]
    lib.allegro_group_rows.argtypes = [i64, i32, vp, vp, vp, vp, sz, vp]
    lib.allegro_grouped_matmul.argtypes = [i32, i32, i64, i32, i32, i32, vp, vp, vp, i64, vp, vp, i64, vp]
    lib.allegro_grouped_matmul_workspace.argtypes = [i64, i32, i32, i32, szp]
    lib.allegro_grouped_matmul_backward.argtypes = [i32, i32, i64, i32, i32, i32, vp, vp, vp, i64, vp, vp, i64, vp, i64,
                                                    vp, vp, sz, vp]
    lib.allegro_rms_norm_forward.argtypes = [i32, i64, i32, f32, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp]
    lib.allegro_rms_norm_fp8.argtypes = [i32, i64, i32, f32, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp]
    lib.allegro_rms_norm_workspace.argtypes = [i64, i32, szp]
    lib.allegro_rms_norm_backward.argtypes = [i32, i64, i32, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
    lib.allegro_grouped_matmul_fp8.argtypes = [i64, i32, i32, i32, vp, vp, vp, i64, vp, vp, vp, vp, i64, vp]
    for name in EXPORTED:
        if name != "allegro_latent_last_error":
            getattr(lib, name).restype = i32
    return lib


_lib = _load()


def library() -> ctypes.CDLL:
    return _lib


def allegro_latent_last_error() -> str:
    return _lib.allegro_latent_last_error().decode()


def _check(rc: int):
    if rc != ALLEGRO_OK:
        raise AllegroError(rc, allegro_latent_last_error())


_DTYPES = {torch.float32: ALLEGRO_F32, torch.bfloat16: ALLEGRO_BF16}


def _dtype(t, name):
    code = _DTYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None:
        raise TypeError(f"{name} must be a float32 or bfloat16 torch.Tensor")
    return code


def _rows(t, name, shape, dtype, device):
    """Checks a tensor of rows and returns its row stride in elements."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device or not t.is_cuda:
        raise ValueError(f"{name} must live on {device}, a GPU")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    m, c = shape
    if m == 0 or c == 0:
        return c
    s0, s1 = t.stride()
    if (s1 != 1 and c > 1) or (s0 < c and m > 1):
        raise ValueError(f"{name} must have unit column stride and rows that do not overlap, got strides {(s0, s1)}")
    return s0 if m > 1 else max(s0, c)


def _matrix(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, got shape {tuple(t.shape)}")
    return t.shape


def _groups(w, dims, offsets, rows, M, dev):
    """Checks weights [G, ., .] and the grouping of M rows; returns w's shape."""
    if not isinstance(w, torch.Tensor):
        raise TypeError("w must be a torch.Tensor")
    if w.dim() != 3:
        raise ValueError(f"w must be [G, {dims}], got shape {tuple(w.shape)}")
    if offsets is not None:
        _need(offsets, "offsets", (w.shape[0] + 1,), torch.int64, dev)
    if rows is not None:
        _need(rows, "rows", (M,), torch.int32, dev)
    return w.shape


def _scratch(t, need, device):
    if need == 0:
        return 0, 0
    if t is None:
        t = torch.empty(need, dtype=torch.uint8, device=device)
    elif not isinstance(t, torch.Tensor) or t.device != device or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return t.data_ptr(), t.numel() * t.element_size()


# ---------------------------------------------------------------- grouping

def allegro_group_rows_workspace(n_rows: int, n_groups: int) -> int:
    """Bytes of workspace allegro_group_rows needs."""
    out = ctypes.c_size_t()
    _check(_lib.allegro_group_rows_workspace(int(n_rows), int(n_groups), ctypes.byref(out)))
    return out.value


def allegro_group_rows(types, n_groups: int, offsets=None, rows=None, workspace=None, stream=None):
    """Returns (offsets [G+1] int64, rows [M] int32): the rows of each type 0 .. G-1 in order, from types [M]
    int32; rows of any other type come last."""
    if not isinstance(types, torch.Tensor):
        raise TypeError("types must be a torch.Tensor")
    dev, m, g = types.device, types.numel(), int(n_groups)
    _need(types, "types", (m,), torch.int32, dev)
    need = allegro_group_rows_workspace(m, g)
    if offsets is None:
        offsets = torch.empty(g + 1, dtype=torch.int64, device=dev)
    if rows is None:
        rows = torch.empty(m, dtype=torch.int32, device=dev)
    _need(offsets, "offsets", (g + 1,), torch.int64, dev)
    _need(rows, "rows", (m,), torch.int32, dev)
    ws, ws_bytes = _scratch(workspace, need, dev)
    _check(_lib.allegro_group_rows(m, g, _ptr(types), _ptr(offsets), _ptr(rows), ws, ws_bytes, _stream(stream, dev)))
    return offsets, rows


# ---------------------------------------------------------------- products

def allegro_grouped_matmul(x, w, offsets, rows=None, act: int = ALLEGRO_ACT_NONE, out=None, stream=None):
    """Returns y [M, N]: act(x[r]) @ w[type of r] for x [M, K] and w [G, K, N]; zeros for rows without a type."""
    code = _dtype(x, "x")
    m, k = _matrix(x, "x")
    dev = x.device
    g, wk, n = _groups(w, "K, N", offsets, rows, m, dev)
    _need(w, "w", (g, k, n), x.dtype, dev)
    if out is None:
        out = torch.empty((m, n), dtype=x.dtype, device=dev)
    ldx, ldy = _rows(x, "x", (m, k), x.dtype, dev), _rows(out, "out", (m, n), x.dtype, dev)
    _check(_lib.allegro_grouped_matmul(code, int(act), m, k, n, g, _ptr(offsets), _ptr(rows), _ptr(x), ldx, _ptr(w),
                                       _ptr(out), ldy, _stream(stream, dev)))
    return out


def allegro_grouped_matmul_workspace(n_rows: int, k: int, n: int, n_groups: int) -> int:
    """Bytes of workspace allegro_grouped_matmul_backward needs for dw."""
    out = ctypes.c_size_t()
    _check(_lib.allegro_grouped_matmul_workspace(int(n_rows), int(k), int(n), int(n_groups), ctypes.byref(out)))
    return out.value


def allegro_grouped_matmul_backward(x, w, dy, offsets, rows=None, act: int = ALLEGRO_ACT_NONE, dx=None, dw=None,
                                    need_dx: bool = True, need_dw: bool = True, workspace=None, stream=None):
    """Returns (dx [M, K], dw [G, K, N]) of allegro_grouped_matmul; None for one that is not needed."""
    code = _dtype(x, "x")
    m, k = _matrix(x, "x")
    dev = x.device
    g, wk, n = _groups(w, "K, N", offsets, rows, m, dev)
    _need(w, "w", (g, k, n), x.dtype, dev)
    ldx, lddy, lddx = _rows(x, "x", (m, k), x.dtype, dev), _rows(dy, "dy", (m, n), x.dtype, dev), k
    ws = ws_bytes = 0
    if need_dx:
        if dx is None:
            dx = torch.empty((m, k), dtype=x.dtype, device=dev)
        lddx = _rows(dx, "dx", (m, k), x.dtype, dev)
    if need_dw:
        if dw is None:
            dw = torch.empty((g, k, n), dtype=x.dtype, device=dev)
        _need(dw, "dw", (g, k, n), x.dtype, dev)
        ws, ws_bytes = _scratch(workspace, allegro_grouped_matmul_workspace(m, k, n, g), dev)
    dx, dw = dx if need_dx else None, dw if need_dw else None
    _check(_lib.allegro_grouped_matmul_backward(code, int(act), m, k, n, g, _ptr(offsets), _ptr(rows), _ptr(x), ldx,
                                                _ptr(w), _ptr(dy), lddy, _ptr(dx), lddx, _ptr(dw), ws, ws_bytes,
                                                _stream(stream, dev)))
    return dx, dw


def allegro_grouped_matmul_fp8(x, x_scale, w, w_scale, offsets=None, rows=None, out=None, stream=None):
    """Returns y [M, N] bfloat16 from float8_e4m3fn x [M, K] with x_scale [M, ceil(K/128)] and float8_e4m3fn w [G, N, K] with
    w_scale [G, ceil(N/128), ceil(K/128)].  Without offsets w has one group, of all rows."""
    f8 = torch.float8_e4m3fn
    m, k = _matrix(x, "x")
    dev = x.device
    g, n, wk = _groups(w, "N, K", offsets, rows, m, dev)
    _need(w, "w", (g, n, k), f8, dev)
    kb, nb = -(-k // SCALE_BLOCK), -(-n // SCALE_BLOCK)
    _need(x_scale, "x_scale", (m, kb), torch.float32, dev)
    _need(w_scale, "w_scale", (g, nb, kb), torch.float32, dev)
    if out is None:
        out = torch.empty((m, n), dtype=torch.bfloat16, device=dev)
    ldx, ldy = _rows(x, "x", (m, k), f8, dev), _rows(out, "out", (m, n), torch.bfloat16, dev)
    _check(_lib.allegro_grouped_matmul_fp8(m, k, n, g, _ptr(offsets), _ptr(rows), _ptr(x), ldx, _ptr(x_scale),
                                           _ptr(w), _ptr(w_scale), _ptr(out), ldy, _stream(stream, dev)))
    return out


# -------------------------------------------------------------------- norm

def _norm_inputs(x, w, residual, total):
    code = _dtype(x, "x")
    m, c = _matrix(x, "x")
    dev = x.device
    _need(w, "w", (c,), torch.float32, dev)
    ldx, ldr, ldt = _rows(x, "x", (m, c), x.dtype, dev), 0, 0
    if residual is not None:
        ldr = _rows(residual, "residual", (m, c), x.dtype, dev)
        if total is None:
            total = torch.empty((m, c), dtype=x.dtype, device=dev)
    if total is not None:
        ldt = _rows(total, "total", (m, c), x.dtype, dev)
    return code, m, c, dev, ldx, ldr, total, ldt


def allegro_rms_norm_forward(x, w, residual=None, eps: float = 1e-6, total=None, out=None, rstd=None, stream=None):
    """Returns (y [M, C], total [M, C], rstd [M]): total = x + residual (x itself without a residual), y = total *
    rstd * w with rstd = 1 / sqrt(mean(total^2) + eps).  total and rstd are what the backward takes."""
    code, m, c, dev, ldx, ldr, total, ldt = _norm_inputs(x, w, residual, total)
    if out is None:
        out = torch.empty((m, c), dtype=x.dtype, device=dev)
    if rstd is None:
        rstd = torch.empty(m, dtype=torch.float32, device=dev)
    _need(rstd, "rstd", (m,), torch.float32, dev)
    ldy = _rows(out, "out", (m, c), x.dtype, dev)
    _check(_lib.allegro_rms_norm_forward(code, m, c, float(eps), _ptr(x), ldx, _ptr(residual), ldr, _ptr(w),
                                         _ptr(total), ldt, _ptr(out), ldy, _ptr(rstd), _stream(stream, dev)))
    return out, x if total is None else total, rstd


def allegro_rms_norm_fp8(x, w, residual=None, eps: float = 1e-6, total=None, q=None, scale=None, stream=None):
    """Returns (q [M, C] float8_e4m3fn, scale [M, ceil(C/128)], total [M, C]): the norm as q * scale."""
    code, m, c, dev, ldx, ldr, total, ldt = _norm_inputs(x, w, residual, total)
    blocks = -(-c // SCALE_BLOCK)
    if q is None:
        q = torch.empty((m, c), dtype=torch.float8_e4m3fn, device=dev)
    if scale is None:
        scale = torch.empty((m, blocks), dtype=torch.float32, device=dev)
    _need(scale, "scale", (m, blocks), torch.float32, dev)
    ldq = _rows(q, "q", (m, c), torch.float8_e4m3fn, dev)
    _check(_lib.allegro_rms_norm_fp8(code, m, c, float(eps), _ptr(x), ldx, _ptr(residual), ldr, _ptr(w), _ptr(total),
                                     ldt, _ptr(q), ldq, _ptr(scale), _stream(stream, dev)))
    return q, scale, x if total is None else total


def allegro_rms_norm_workspace(n_rows: int, c: int) -> int:
    """Bytes of workspace allegro_rms_norm_backward needs."""
    out = ctypes.c_size_t()
    _check(_lib.allegro_rms_norm_workspace(int(n_rows), int(c), ctypes.byref(out)))
    return out.value


def allegro_rms_norm_backward(total, w, rstd, dy, dtotal=None, dx=None, dw=None, workspace=None, stream=None):
    """Returns (dx [M, C], dw [C]): dx is the gradient of x and of the residual alike, with dtotal, the gradient
    that reaches total along the residual, added."""
    code = _dtype(total, "total")
    m, c = _matrix(total, "total")
    dev, dt = total.device, total.dtype
    _need(w, "w", (c,), torch.float32, dev)
    _need(rstd, "rstd", (m,), torch.float32, dev)
    ldt, lddy = _rows(total, "total", (m, c), dt, dev), _rows(dy, "dy", (m, c), dt, dev)
    lddt = 0 if dtotal is None else _rows(dtotal, "dtotal", (m, c), dt, dev)
    if dx is None:
        dx = torch.empty((m, c), dtype=dt, device=dev)
    if dw is None:
        dw = torch.empty(c, dtype=torch.float32, device=dev)
    _need(dw, "dw", (c,), torch.float32, dev)
    lddx = _rows(dx, "dx", (m, c), dt, dev)
    ws, ws_bytes = _scratch(workspace, allegro_rms_norm_workspace(m, c), dev)
    _check(_lib.allegro_rms_norm_backward(code, m, c, _ptr(total), ldt, _ptr(w), _ptr(rstd), _ptr(dy), lddy,
                                          _ptr(dtotal), lddt, _ptr(dx), lddx, _ptr(dw), ws, ws_bytes,
                                          _stream(stream, dev)))
    return dx, dw
