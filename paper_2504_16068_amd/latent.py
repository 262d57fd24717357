"""ctypes binding of liballegro_latent.so -- argument marshalling only.

The operators of the scalar (latent) track, declared in include/allegro_latent.h: rows grouped by
type, products per type, the root-mean-square norm with the residual's addition, and 8-bit products.
Functions have the names of the C entry points; like those of the tensor product they check shapes,
dtypes and devices, allocate with PyTorch what the caller does not pass, and hand raw pointers and
the current HIP stream to the library.  Tensors of rows may be views with a row stride.  There is no
fallback: without the compiled library importing this module raises.

A call with `stream` (a torch.cuda.Stream) is one under `with torch.cuda.stream(stream)`: results and
workspaces that it allocates belong to that stream.  Tensors of other streams are the caller's to order
(wait_stream) and to keep until the call has run (record_stream).
"""

from __future__ import annotations

import ctypes
import os

import torch

from .binding import ALLEGRO_E_INVALID, ALLEGRO_OK, AllegroError, _current_device, _empty, _stream, _there

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


_INT_MAX, _INT64_MAX = 2 ** 31 - 1, 2 ** 63 - 1
_Tensor = torch.Tensor
_F32, _BF16, _F8, _I32, _I64 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.int32, torch.int64

# As in binding.py, an argument that is right takes one pass of cheap comparisons
# (device indices instead of device objects, contiguity before strides): a call with
# six tensors costs 5 us before its launch that way, 6 with objects and strides.


def _matrix(t, name):
    """(dtype code, device index) of a float32 or bfloat16 matrix on a GPU."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    dt = t.dtype
    if dt is not _F32 and dt is not _BF16:
        raise TypeError(f"{name} must be float32 or bfloat16, got {dt}")
    return 0 if dt is _F32 else 1, _index(t, name)


def _index(t, name):
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, got shape {tuple(t.shape)}")
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must live on a GPU, not on {t.device}")
    return index


def _refuse(t, name, shape, dtype, index):
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} must live on cuda:{index}, not on {t.device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _rows(t, name, shape, dtype, index):
    """Checks a tensor of rows and returns its row stride in elements."""
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == index):
        _refuse(t, name, shape, dtype, index)
    if t.is_contiguous():
        return shape[1]
    s0, s1 = t.stride()
    m, c = shape
    if (s1 != 1 and c > 1) or (s0 < c and m > 1):
        raise ValueError(f"{name} must have unit column stride and rows that do not overlap, got strides {(s0, s1)}")
    return s0 if m > 1 else c


def _whole(t, name, shape, dtype, index):
    """Checks a contiguous tensor and returns its address."""
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == index):
        _refuse(t, name, shape, dtype, index)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _weights(w, dims):
    if not isinstance(w, _Tensor):
        raise TypeError("w must be a torch.Tensor")
    if w.dim() != 3:
        raise ValueError(f"w must be [G, {dims}], got shape {tuple(w.shape)}")
    shape = w.shape
    if shape[0] > _INT_MAX:  # widths are seen by the library as row strides too, which are of 64 bits
        raise AllegroError(ALLEGRO_E_INVALID, f"w has {shape[0]} groups")
    return shape


def _groups(offsets, rows, g, m, index):
    """Addresses of the grouping of m rows."""
    return (0 if offsets is None else _whole(offsets, "offsets", (g + 1,), _I64, index),
            0 if rows is None else _whole(rows, "rows", (m,), _I32, index))


def _scratch(t, need, index, stream):
    """(tensor that keeps it, address, bytes) of a workspace."""
    if need == 0:
        return None, 0, 0
    if t is None:
        t = _empty((need,), torch.uint8, index, stream)
        return t, t.data_ptr(), need
    if not isinstance(t, _Tensor) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{index}")
    return t, t.data_ptr(), t.numel() * t.element_size()


def _bytes(fn, rows, *sizes):
    out = ctypes.c_size_t()
    rows, sizes = int(rows), [int(v) for v in sizes]
    # rows is an int64_t in C, the others an int; what does not fit is refused there all the same
    if max(sizes) > _INT_MAX or min(sizes) < -_INT_MAX or abs(rows) > _INT64_MAX:
        rows = max(-_INT64_MAX, min(rows, _INT64_MAX))
        sizes = [max(-_INT_MAX, min(v, _INT_MAX)) for v in sizes]
    _check(fn(rows, *sizes, ctypes.byref(out)))
    return out.value


# ---------------------------------------------------------------- grouping

def allegro_group_rows_workspace(n_rows: int, n_groups: int) -> int:
    """Bytes of workspace allegro_group_rows needs."""
    return _bytes(_lib.allegro_group_rows_workspace, n_rows, n_groups)


def allegro_group_rows(types, n_groups: int, offsets=None, rows=None, workspace=None, stream=None):
    """Returns (offsets [G+1] int64, rows [M] int32): the rows of each type 0 .. G-1 in order, from types [M]
    int32; rows of any other type come last."""
    if not isinstance(types, _Tensor):
        raise TypeError("types must be a torch.Tensor")
    m, g, index = types.numel(), int(n_groups), types.get_device()
    if index < 0:
        raise ValueError(f"types must live on a GPU, not on {types.device}")
    if _current_device() != index:
        return _there(index, allegro_group_rows, types, n_groups, offsets, rows, workspace, stream)
    need = allegro_group_rows_workspace(m, g)
    if offsets is None:
        offsets = _empty((g + 1,), _I64, index, stream)
    if rows is None:
        rows = _empty((m,), _I32, index, stream)
    t_p = _whole(types, "types", (m,), _I32, index)
    o_p, r_p = _groups(offsets, rows, g, m, index)
    keep, ws, ws_bytes = _scratch(workspace, need, index, stream)
    _check(_lib.allegro_group_rows(m, g, t_p, o_p, r_p, ws, ws_bytes, _stream(stream, index)))
    return offsets, rows


# ---------------------------------------------------------------- products

def allegro_grouped_matmul(x, w, offsets, rows=None, act: int = ALLEGRO_ACT_NONE, out=None, stream=None):
    """Returns y [M, N]: act(x[r]) @ w[type of r] for x [M, K] and w [G, K, N]; zeros for rows without a type."""
    g, _, n = _weights(w, "K, N")
    code, index = _matrix(x, "x")
    if _current_device() != index:
        return _there(index, allegro_grouped_matmul, x, w, offsets, rows, act, out, stream)
    dt, shape = x.dtype, x.shape
    m, k = shape
    if out is None:
        out = _empty((m, n), dt, index, stream)
    w_p = _whole(w, "w", (g, k, n), dt, index)
    o_p, r_p = _groups(offsets, rows, g, m, index)
    ldx, ldy = _rows(x, "x", shape, dt, index), _rows(out, "out", (m, n), dt, index)
    _check(_lib.allegro_grouped_matmul(code, act, m, k, n, g, o_p, r_p, x.data_ptr(), ldx, w_p, out.data_ptr(), ldy,
                                       _stream(stream, index)))
    return out


def allegro_grouped_matmul_workspace(n_rows: int, k: int, n: int, n_groups: int) -> int:
    """Bytes of workspace allegro_grouped_matmul_backward needs for dw."""
    return _bytes(_lib.allegro_grouped_matmul_workspace, n_rows, k, n, n_groups)


def allegro_grouped_matmul_backward(x, w, dy, offsets, rows=None, act: int = ALLEGRO_ACT_NONE, dx=None, dw=None,
                                    need_dx: bool = True, need_dw: bool = True, workspace=None, stream=None):
    """Returns (dx [M, K], dw [G, K, N]) of allegro_grouped_matmul; None for one that is not needed."""
    g, _, n = _weights(w, "K, N")
    code, index = _matrix(x, "x")
    if _current_device() != index:
        return _there(index, allegro_grouped_matmul_backward, x, w, dy, offsets, rows, act, dx, dw, need_dx,
                      need_dw, workspace, stream)
    dt, shape = x.dtype, x.shape
    m, k = shape
    w_p = _whole(w, "w", (g, k, n), dt, index)
    o_p, r_p = _groups(offsets, rows, g, m, index)
    ldx, lddy = _rows(x, "x", shape, dt, index), _rows(dy, "dy", (m, n), dt, index)
    dx_p, lddx, dw_p, keep, ws, ws_bytes = 0, k, 0, None, 0, 0
    if need_dx:
        if dx is None:
            dx = _empty((m, k), dt, index, stream)
        dx_p, lddx = dx.data_ptr(), _rows(dx, "dx", shape, dt, index)
    if need_dw:
        if dw is None:
            dw = _empty((g, k, n), dt, index, stream)
        dw_p = _whole(dw, "dw", (g, k, n), dt, index)
        keep, ws, ws_bytes = _scratch(workspace, allegro_grouped_matmul_workspace(m, k, n, g), index, stream)
    _check(_lib.allegro_grouped_matmul_backward(code, act, m, k, n, g, o_p, r_p, x.data_ptr(), ldx, w_p,
                                                dy.data_ptr(), lddy, dx_p, lddx, dw_p, ws, ws_bytes,
                                                _stream(stream, index)))
    return dx if need_dx else None, dw if need_dw else None


def allegro_grouped_matmul_fp8(x, x_scale, w, w_scale, offsets=None, rows=None, out=None, stream=None):
    """Returns y [M, N] bfloat16 from float8_e4m3fn x [M, K] with x_scale [M, ceil(K/128)] and float8_e4m3fn w [G, N, K]
    with w_scale [G, ceil(N/128), ceil(K/128)].  Without offsets w has one group, of all rows."""
    if not isinstance(x, _Tensor):
        raise TypeError("x must be a torch.Tensor")
    index, shape = _index(x, "x"), x.shape
    if _current_device() != index:
        return _there(index, allegro_grouped_matmul_fp8, x, x_scale, w, w_scale, offsets, rows, out, stream)
    m, k = shape
    g, n, _ = _weights(w, "N, K")
    kb, nb = (k + SCALE_BLOCK - 1) // SCALE_BLOCK, (n + SCALE_BLOCK - 1) // SCALE_BLOCK
    if out is None:
        out = _empty((m, n), _BF16, index, stream)
    w_p = _whole(w, "w", (g, n, k), _F8, index)
    xs_p = _whole(x_scale, "x_scale", (m, kb), _F32, index)
    ws_p = _whole(w_scale, "w_scale", (g, nb, kb), _F32, index)
    o_p, r_p = _groups(offsets, rows, g, m, index)
    ldx, ldy = _rows(x, "x", shape, _F8, index), _rows(out, "out", (m, n), _BF16, index)
    _check(_lib.allegro_grouped_matmul_fp8(m, k, n, g, o_p, r_p, x.data_ptr(), ldx, xs_p, w_p, ws_p, out.data_ptr(),
                                           ldy, _stream(stream, index)))
    return out


# -------------------------------------------------------------------- norm

def _norm_inputs(x, w, residual, total, stream):
    """(dtype code, device index, addresses and strides of x, residual, w and total, total)."""
    code, index = _matrix(x, "x")
    dt, shape = x.dtype, x.shape
    w_p = _whole(w, "w", shape[1:], _F32, index)
    ldx, r_p, ldr, t_p, ldt = _rows(x, "x", shape, dt, index), 0, 0, 0, 0
    if residual is not None:
        ldr, r_p = _rows(residual, "residual", shape, dt, index), residual.data_ptr()
        if total is None:
            total = _empty(shape, dt, index, stream)
    if total is not None:
        ldt, t_p = _rows(total, "total", shape, dt, index), total.data_ptr()
    return code, index, (x.data_ptr(), ldx, r_p, ldr, w_p, t_p, ldt), total


def allegro_rms_norm_forward(x, w, residual=None, eps: float = 1e-6, total=None, out=None, rstd=None, stream=None):
    """Returns (y [M, C], total [M, C], rstd [M]): total = x + residual (x itself without a residual), y = total *
    rstd * w with rstd = 1 / sqrt(mean(total^2) + eps).  total and rstd are what the backward takes.  The tensor passed
    for total may be x or residual itself."""
    code, index, args, total = _norm_inputs(x, w, residual, total, stream)
    if _current_device() != index:
        return _there(index, allegro_rms_norm_forward, x, w, residual, eps, total, out, rstd, stream)
    shape, dt = x.shape, x.dtype
    m, c = shape
    if out is None:
        out = _empty(shape, dt, index, stream)
    if rstd is None:
        rstd = _empty((m,), _F32, index, stream)
    rstd_p, ldy = _whole(rstd, "rstd", (m,), _F32, index), _rows(out, "out", shape, dt, index)
    _check(_lib.allegro_rms_norm_forward(code, m, c, eps, *args, out.data_ptr(), ldy, rstd_p, _stream(stream, index)))
    return out, x if total is None else total, rstd


def allegro_rms_norm_fp8(x, w, residual=None, eps: float = 1e-6, total=None, q=None, scale=None, stream=None):
    """Returns (q [M, C] float8_e4m3fn, scale [M, ceil(C/128)], total [M, C]): the norm as q * scale."""
    code, index, args, total = _norm_inputs(x, w, residual, total, stream)
    if _current_device() != index:
        return _there(index, allegro_rms_norm_fp8, x, w, residual, eps, total, q, scale, stream)
    shape = x.shape
    m, c = shape
    blocks = (c + SCALE_BLOCK - 1) // SCALE_BLOCK
    if q is None:
        q = _empty(shape, _F8, index, stream)
    if scale is None:
        scale = _empty((m, blocks), _F32, index, stream)
    scale_p, ldq = _whole(scale, "scale", (m, blocks), _F32, index), _rows(q, "q", shape, _F8, index)
    _check(_lib.allegro_rms_norm_fp8(code, m, c, eps, *args, q.data_ptr(), ldq, scale_p, _stream(stream, index)))
    return q, scale, x if total is None else total


def allegro_rms_norm_workspace(n_rows: int, c: int) -> int:
    """Bytes of workspace allegro_rms_norm_backward needs."""
    return _bytes(_lib.allegro_rms_norm_workspace, n_rows, c)


def allegro_rms_norm_backward(total, w, rstd, dy, dtotal=None, dx=None, dw=None, workspace=None, stream=None):
    """Returns (dx [M, C], dw [C]): dx is the gradient of x and of the residual alike, with dtotal, the gradient
    that reaches total along the residual, added."""
    code, index = _matrix(total, "total")
    if _current_device() != index:
        return _there(index, allegro_rms_norm_backward, total, w, rstd, dy, dtotal, dx, dw, workspace, stream)
    dt, shape = total.dtype, total.shape
    m, c = shape
    w_p, rstd_p = _whole(w, "w", (c,), _F32, index), _whole(rstd, "rstd", (m,), _F32, index)
    ldt, lddy = _rows(total, "total", shape, dt, index), _rows(dy, "dy", shape, dt, index)
    ds_p, ldds = 0, 0
    if dtotal is not None:
        ldds, ds_p = _rows(dtotal, "dtotal", shape, dt, index), dtotal.data_ptr()
    if dx is None:
        dx = _empty(shape, dt, index, stream)
    if dw is None:
        dw = _empty((c,), _F32, index, stream)
    dw_p, lddx = _whole(dw, "dw", (c,), _F32, index), _rows(dx, "dx", shape, dt, index)
    keep, ws, ws_bytes = _scratch(workspace, allegro_rms_norm_workspace(m, c), index, stream)
    _check(_lib.allegro_rms_norm_backward(code, m, c, total.data_ptr(), ldt, w_p, rstd_p, dy.data_ptr(), lddy, ds_p,
                                          ldds, dx.data_ptr(), lddx, dw_p, ws, ws_bytes, _stream(stream, index)))
    return dx, dw
