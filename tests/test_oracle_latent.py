"""Pins of the latent operators' oracle: differences, special cases, and the 8-bit format."""

import numpy as np
import pytest

from oracle import latent as ol


def test_group_rows_is_a_stable_sort():
    rng = np.random.default_rng(1)
    t = rng.integers(-2, 7, 200)
    offsets, rows = ol.group_rows(t, 5)
    key = np.where((t >= 0) & (t < 5), t, 5)
    assert np.array_equal(rows, np.argsort(key, kind="stable"))
    assert np.array_equal(np.diff(offsets), [np.sum(t == g) for g in range(5)])


@pytest.mark.parametrize("act", [False, True])
def test_product_gradients_against_differences(act):
    rng = np.random.default_rng(2)
    t = rng.integers(-1, 3, 11)
    x, w, dy = rng.normal(size=(11, 5)), rng.normal(size=(3, 5, 4)), rng.normal(size=(11, 4))
    loss = lambda x, w: float(np.sum(dy * ol.grouped_matmul(t, x, w, act)))  # noqa: E731
    dx, dw = ol.grouped_matmul_backward(t, x, w, dy, act)
    h = 1e-6
    for got, arg in ((dx, x), (dw, w)):
        num = np.empty_like(arg)
        for i in np.ndindex(arg.shape):
            keep = arg[i]
            arg[i] = keep + h
            up = loss(x, w)
            arg[i] = keep - h
            num[i] = (up - loss(x, w)) / (2 * h)
            arg[i] = keep
        assert np.max(np.abs(got - num)) < 1e-8
    assert np.all(dx[t < 0] == 0)


def test_norm_and_its_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, r, w = rng.normal(size=(4, 7)), rng.normal(size=(4, 7)), rng.normal(size=7)
    dy, ds, eps = rng.normal(size=(4, 7)), rng.normal(size=(4, 7)), 0.01
    loss = lambda x, w: float(np.sum(dy * ol.rms_norm(x + r, w, eps)[0]) + np.sum(ds * (x + r)))  # noqa: E731
    y, rstd = ol.rms_norm(x + r, w, eps)
    assert np.allclose(np.mean((y / w) ** 2, axis=1), 1 - eps * rstd ** 2)
    dx, dw = ol.rms_norm_backward(x + r, w, rstd, dy, ds)
    h = 1e-6
    for got, arg in ((dx, x), (dw, w)):
        num = np.empty_like(arg)
        for i in np.ndindex(arg.shape):
            keep = arg[i]
            arg[i] = keep + h
            up = loss(x, w)
            arg[i] = keep - h
            num[i] = (up - loss(x, w)) / (2 * h)
            arg[i] = keep
        assert np.max(np.abs(got - num)) < 1e-8


def test_eight_bit_format():
    torch = pytest.importorskip("torch")
    v = ol.f8_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(v, t, equal_nan=True) and np.nanmax(v) == ol.F8_MAX
    rng = np.random.default_rng(4)
    x = np.concatenate([rng.uniform(-448, 448, 2000), rng.normal(size=2000) * 0.02, v[np.isfinite(v)],
                        (v[:126] + v[1:127]) / 2])  # the last: every tie
    got = ol.f8_round(x)
    near = v[np.isfinite(v)]
    assert np.all(np.abs(got - x) == np.min(np.abs(near[None, :] - x[:, None]), axis=1))
    assert np.array_equal(got, torch.from_numpy(x).float().to(torch.float8_e4m3fn).to(torch.float64).numpy())


def test_block_scales():
    rng = np.random.default_rng(5)
    y = rng.normal(size=(3, 300))
    y[1] = 0
    v, scale = ol.f8_blocks(y)
    assert scale.shape == (3, 3) and np.all(scale[1] == 2.0 ** -126) and np.all(v[1] == 0)
    assert np.allclose(np.abs(v[0, :128]).max(), 448) and np.allclose(np.abs(v[0, 256:]).max(), 448)
    assert np.allclose(ol.dequantise_rows(v, scale), y)
    # one group and unit scales: the plain product
    q = ol.f8_round(rng.normal(size=(4, 130)))
    w = ol.f8_round(rng.normal(size=(1, 6, 130)))
    got = ol.grouped_matmul_fp8(np.zeros(4, int), q, np.ones((4, 2)), w, np.ones((1, 1, 2)))
    assert np.allclose(got, q @ w[0].T)
