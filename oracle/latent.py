"""The operators of the latent track in 64 bits (oracle, test infrastructure).

Plain definitions, independent of the HIP path: rows grouped by type, products
per type over ragged groups with their gradients, the root-mean-square norm of
x + residual with its gradients, 8-bit values (4 exponent and 3 mantissa bits,
bias 7, no infinities, largest value 448) with a scale for each block of 128
columns, and the product of such operands.  The paper names the layer's scalar
track and its fp32 arithmetic (Appendix, "Mixed-Precision Architecture") but
none of these operators: parity unpinned, every function is pinned by its
definition, finite differences and special cases.
"""

from __future__ import annotations

import numpy as np

BLOCK = 128
F8_MAX = 448.0


def group_rows(types, n_groups):
    """(offsets [G+1], rows [M]): rows of type 0, then 1, ...; those of no type last, each in order."""
    groups = [[] for _ in range(n_groups + 1)]
    for r, t in enumerate(types):
        groups[t if 0 <= t < n_groups else n_groups].append(r)
    offsets = np.cumsum([0] + [len(g) for g in groups[:n_groups]])
    return offsets.astype(np.int64), np.array([r for g in groups for r in g], dtype=np.int32)


def silu(a):
    return a / (1.0 + np.exp(-a))


def silu_grad(a):
    s = 1.0 / (1.0 + np.exp(-a))
    return s * (1.0 + a * (1.0 - s))


def grouped_matmul(types, x, w, act):
    """y [M, N]; zeros where the type is none of w's."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    y = np.zeros((x.shape[0], w.shape[2]))
    z = silu(x) if act else x
    for g in range(w.shape[0]):
        y[types == g] = z[types == g] @ w[g]
    return y


def grouped_matmul_backward(types, x, w, dy, act):
    """(dx, dw)."""
    x, w, dy = (np.asarray(a, np.float64) for a in (x, w, dy))
    dx, dw = np.zeros_like(x), np.zeros_like(w)
    z = silu(x) if act else x
    for g in range(w.shape[0]):
        m = types == g
        dx[m] = dy[m] @ w[g].T
        dw[g] = z[m].T @ dy[m]
    return (dx * silu_grad(x) if act else dx), dw


def rms_norm(total, w, eps):
    """(y, rstd) of the sum that is normalised."""
    total = np.asarray(total, np.float64)
    rstd = 1.0 / np.sqrt(np.mean(total * total, axis=1) + eps)
    return total * rstd[:, None] * np.asarray(w, np.float64), rstd


def rms_norm_backward(total, w, rstd, dy, dtotal=None):
    """(dx, dw): gradients of <dy, y> + <dtotal, total>, with rstd that of total."""
    total, w, rstd, dy = (np.asarray(a, np.float64) for a in (total, w, rstd, dy))
    u, t = total * rstd[:, None], dy * w
    dx = rstd[:, None] * (t - u * np.mean(t * u, axis=1, keepdims=True))
    return (dx if dtotal is None else dx + np.asarray(dtotal, np.float64)), np.sum(dy * u, axis=0)


def f8_values():
    """The value of each of the 256 codes: sign, 4 bits of exponent (bias 7), 3 of mantissa."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = np.nan if e == 15 and m == 7 else -mag if c & 128 else mag
    return v


def f8_round(v):
    """The nearest 8-bit value, ties to the even mantissa; magnitudes up to 448 only."""
    v = np.asarray(v, np.float64)
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    return np.rint(v / step) * step


def f8_blocks(y):
    """(v [M, C], scale [M, blocks]): the values v = y / scale before their rounding to 8 bits."""
    M, C = y.shape
    blocks = -(-C // BLOCK)
    scale = np.empty((M, blocks))
    v = np.empty_like(y)
    for b in range(blocks):
        c = slice(b * BLOCK, min(C, (b + 1) * BLOCK))
        scale[:, b] = np.maximum(np.abs(y[:, c]).max(axis=1) / F8_MAX, 2.0 ** -126)
        v[:, c] = y[:, c] / scale[:, b:b + 1]
    return v, scale


def dequantise_rows(q, scale):
    """[..., C] values times their blocks' scales [..., blocks]."""
    return q * np.repeat(scale, BLOCK, axis=-1)[..., :q.shape[-1]]


def grouped_matmul_fp8(types, q, scale, wq, w_scale):
    """y [M, N] from 8-bit values q [M, K], wq [G, N, K] and scales [M, kb], [G, nb, kb]."""
    x = dequantise_rows(np.asarray(q, np.float64), np.asarray(scale, np.float64))
    rows = np.repeat(np.asarray(w_scale, np.float64), BLOCK, axis=1)[:, :wq.shape[1]]
    w = dequantise_rows(np.asarray(wq, np.float64), rows)
    return grouped_matmul(types, x, np.swapaxes(w, 1, 2), False)
