"""Parity of the latent operators at sizes that reach the launches which the shapes of test_gpu_latent.py leave out.

Those are: tiles of 128 columns in bf16, weight gradients of narrow bf16 products over many rows, norms whose
persistent workgroups take several rounds of rows, and widths between.  With them a kernel trace of these files shows
every kernel of liballegro_latent.so.  Bounds as in test_gpu_latent.py.
"""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_latent import BF16, DEV, F32, U, _f64, _gen, _norm_case, _normal, _note, _product_case, at  # noqa: E402, F401


@pytest.mark.parametrize("m,k,n,g,act", [
    (45000, 200, 127, 3, False), (66003, 192, 128, 3, False), (45011, 64, 400, 5, False), (20003, 520, 300, 7, False),
    (45000, 200, 127, 3, True), (70000, 128, 64, 100, True), (70000, 128, 61, 100, False), (90001, 40, 33, 4, True),
    (90001, 64, 64, 4, False), (60000, 33, 250, 2, True), (60000, 250, 33, 2, False)])
def test_bf16_products_of_many_rows(at, m, k, n, g, act):
    _note(f"[gpu] product M={m} K={k} N={n} G={g} bf16 act={act}")
    _product_case(at, m, k, n, g, BF16, act)


@pytest.mark.parametrize("m,k,n,g,act", [(9000, 300, 500, 4, False), (30000, 400, 256, 200, False), (66000, 513, 390, 3, False),
                                         (90001, 40, 33, 4, False), (70000, 600, 40, 3, True)])
def test_fp32_products_of_many_tiles(at, m, k, n, g, act):
    _note(f"[gpu] product M={m} K={k} N={n} G={g} f32 act={act}")
    _product_case(at, m, k, n, g, F32, act)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,c", [(30000, 300), (9000, 1031), (5000, 4097)])
def test_norm_in_several_rounds(at, dtype, m, c):
    """Workgroups that go through their loop over rows more than once, forward, in 8 bits and backward."""
    _note(f"[gpu] norm M={m} C={c} {dtype}")
    _norm_case(at, m, c, dtype, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("residual", [True, False], ids=["residual", "alone"])
@pytest.mark.parametrize("m,c", [(60, 700), (37, 2000), (33, 1800)])
def test_norm_of_the_other_widths(at, dtype, residual, m, c):
    """Three, and seven or eight, vectors to a lane (four in bf16)."""
    _note(f"[gpu] norm M={m} C={c} {dtype} residual={residual}")
    _norm_case(at, m, c, dtype, residual)


def test_streamed_products_mean_error(at):
    """As test_products_mean_error, of the kernel that streams rows past stationary weights: the mean error of 9e6
    values stays below a fiftieth of their spread."""
    gen = _gen(78)
    m, k, n = 70000, 64, 128
    x, w = _normal(gen, m, k).abs(), _normal(gen, 1, k, n).abs()
    y = _f64(at.allegro_grouped_matmul(x.to(DEV), w.to(DEV), torch.tensor([0, m], device=DEV)))
    rel = y / (_f64(x) @ _f64(w)[0]) - 1
    _note(f"  mean {np.mean(rel):.2e}, spread {np.std(rel):.2e}")
    assert abs(np.mean(rel)) <= 0.02 * np.std(rel) and np.std(rel) <= 4 * U
