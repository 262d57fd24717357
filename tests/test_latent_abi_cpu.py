"""Host-side tests of the latent operators' C ABI (no GPU): exports, workspace sizes, refusals."""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "allegro_latent.h")

latent = pytest.importorskip("paper_2504_16068_amd.latent",
                             reason="libraries not built (run __graft_entry__.build())")
from paper_2504_16068_amd.binding import ALLEGRO_E_INVALID, ALLEGRO_E_UNSUPPORTED, ALLEGRO_OK  # noqa: E402

OK, ODD, OFF8 = 0x10000, 0x10001, 0x10004
vp = ctypes.c_void_p


def _declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    out = {}
    for name, params in re.findall(r"\b(allegro_\w+)\s*\(([^;{]*?)\)\s*;", text, flags=re.S):
        params = params.strip()
        out[name] = 0 if params in ("", "void") else params.count(",") + 1
    return out


def test_exports_and_argument_counts_match_the_header():
    lib, declared = latent.library(), _declared()
    assert set(declared) == set(latent.EXPORTED)
    for name, n in declared.items():
        assert len(getattr(lib, name).argtypes) == n, name


def _refused(fn, args, code, *words):
    rc = fn(*args)
    message = latent.allegro_latent_last_error()
    assert rc == code, (rc, message)
    for w in words:
        assert w in message, message


def _swap(args, i, v):
    return [*args[:i], v, *args[i + 1:]]


def test_workspace_sizes():
    assert latent.allegro_group_rows_workspace(4096, 1024) == 0  # one workgroup
    assert latent.allegro_group_rows_workspace(4097, 4) == (3 + 1) * 5 * 4
    assert latent.allegro_rms_norm_workspace(0, 64) == 0
    assert latent.allegro_rms_norm_workspace(10 ** 6, 64) == 1024 * 64 * 4
    assert latent.allegro_grouped_matmul_workspace(256, 64, 64, 3) == 0  # one range per group
    assert latent.allegro_grouped_matmul_workspace(257, 5, 7, 3) == 3 * 36 * 4
    # no overflow at the largest sizes
    assert latent.allegro_group_rows_workspace(2 ** 31 - 1, 1024) < 2 ** 23
    for fn, args in ((latent.allegro_group_rows_workspace, (-1, 4)), (latent.allegro_group_rows_workspace, (4, 0)),
                     (latent.allegro_group_rows_workspace, (4, 1025)), (latent.allegro_rms_norm_workspace, (4, 65537)),
                     (latent.allegro_grouped_matmul_workspace, (2 ** 31, 4, 4, 4))):
        with pytest.raises(latent.AllegroError) as ex:
            fn(*args)
        assert ex.value.code == ALLEGRO_E_INVALID


@pytest.mark.parametrize("m,k,n,g", [(10 ** 7, 1024, 1024, 1), (10 ** 7, 1024, 1024, 16), (10 ** 6, 128, 64, 225),
                                     (2 ** 31 - 1, 64, 64, 4), (2 ** 25, 65536, 256, 1)])
def test_product_workspace_is_bounded(m, k, n, g):
    """Partial sums of dw: a few for each tile on the chip, whatever the number of rows."""
    tiles = -(-k // 128) * -(-n // 128)
    assert latent.allegro_grouped_matmul_workspace(m, k, n, g) <= 4 * (2 * 1024 + tiles) * 128 * 128 * 4


def test_group_rows_refuses():
    fn = latent.library().allegro_group_rows
    good = [5000, 4, OK, OK, OK, OK, 1 << 20, None]
    for i, v, *words in ((0, -1, "negative"), (0, 2 ** 31, "2^31"), (1, 0, "G=0"), (1, 1025, "G=1025"), (2, None, "type is NULL"),
                         (2, ODD, "type", "aligned"), (3, OFF8, "offsets", "aligned"), (4, None, "rows is NULL"),
                         (5, None, "workspace is NULL"), (5, OFF8, "workspace", "aligned"), (6, 10, "smaller")):
        _refused(fn, _swap(good, i, v), ALLEGRO_E_INVALID, *words)


def test_products_refuse():
    fn = latent.library().allegro_grouped_matmul
    # dtype, act, M, K, N, G, offsets, rows, X, ldx, W, Y, ldy, stream
    good = [0, 0, 100, 64, 32, 4, OK, OK, OK, 64, OK, OK, 32, None]
    for i, v, *words in ((0, 2, "dtype"), (1, 2, "act"), (2, -1, "negative"), (3, 0, "K=0"), (4, 65537, "N=65537"), (5, 0, "G=0"),
                         (6, None, "offsets is NULL"), (7, ODD, "rows", "aligned"), (8, None, "X is NULL"),
                         (8, ODD, "X", "aligned"), (9, 63, "row stride 63"), (10, None, "W is NULL"),
                         (11, None, "Y is NULL"), (12, 31, "row stride 31")):
        _refused(fn, _swap(good, i, v), ALLEGRO_E_INVALID, *words)
    _refused(fn, [0, 0, 2 ** 31 - 1, 64, 65536, 4, OK, OK, OK, 64, OK, OK, 65536, None], ALLEGRO_E_UNSUPPORTED, "tiles")
    assert fn(*_swap(_swap(good, 2, 0), 8, None)) == ALLEGRO_OK  # no rows: nothing to do

    fn = latent.library().allegro_grouped_matmul_backward
    # dtype, act, M, K, N, G, offsets, rows, X, ldx, W, dY, lddy, dX, lddx, dW, workspace, bytes, stream
    good = [1, 1, 1000, 64, 32, 4, OK, OK, OK, 64, OK, OK, 32, OK, 64, OK, OK, 1 << 30, None]
    for i, v, *words in ((0, -1, "dtype"), (6, None, "offsets is NULL"), (8, None, "X is NULL"), (10, None, "W is NULL"),
                         (11, None, "dY is NULL"), (12, 31, "row stride 31"), (13, ODD, "dX", "aligned"),
                         (14, 63, "row stride 63"), (15, ODD, "dW", "aligned"), (16, None, "workspace is NULL"),
                         (17, 100, "smaller")):
        _refused(fn, _swap(good, i, v), ALLEGRO_E_INVALID, *words)


def test_norm_refuses():
    lib = latent.library()
    # dtype, M, C, eps, x, ldx, residual, ldr, w, total, ldt, y, ldy, rstd, stream
    good = [0, 10, 64, 1e-6, OK, 64, OK, 64, OK, OK, 64, OK, 64, OK, None]
    for i, v, *words in ((0, 7, "dtype"), (1, -3, "negative"), (2, 0, "C=0"), (3, -1.0, "eps"), (3, float("nan"), "eps"),
                         (4, None, "x is NULL"), (5, 63, "row stride"), (6, ODD, "residual", "aligned"), (7, 1, "residual"),
                         (8, None, "w is NULL"), (9, ODD, "total", "aligned"), (11, None, "y is NULL"), (12, 3, "y has row stride"),
                         (13, ODD, "rstd", "aligned")):
        _refused(lib.allegro_rms_norm_forward, _swap(good, i, v), ALLEGRO_E_INVALID, *words)
    for i, v, *words in ((11, None, "q is NULL"), (12, 63, "q has row stride"), (13, None, "scale is NULL"),
                         (13, ODD, "scale", "aligned")):
        _refused(lib.allegro_rms_norm_fp8, _swap(good, i, v), ALLEGRO_E_INVALID, *words)
    # dtype, M, C, total, ldt, w, rstd, dy, lddy, dtotal, lddt, dx, lddx, dw, workspace, bytes, stream
    good = [1, 10, 64, OK, 64, OK, OK, OK, 64, OK, 64, OK, 64, OK, OK, 1 << 20, None]
    for i, v, *words in ((3, None, "total is NULL"), (5, None, "w is NULL"), (6, None, "rstd is NULL"), (7, None, "dy is NULL"),
                         (9, ODD, "dtotal", "aligned"), (10, 2, "dtotal has row stride"), (11, None, "dx is NULL"),
                         (13, None, "dw is NULL"), (14, None, "workspace is NULL"), (15, 100, "smaller")):
        _refused(lib.allegro_rms_norm_backward, _swap(good, i, v), ALLEGRO_E_INVALID, *words)


def test_f8_products_refuse():
    fn = latent.library().allegro_grouped_matmul_fp8
    # M, K, N, G, offsets, rows, X, ldx, xs, W, ws, Y, ldy, stream
    good = [10, 128, 64, 4, OK, OK, OK, 128, OK, OK, OK, OK, 64, None]
    for i, v, *words in ((0, -1, "negative"), (1, 0, "K=0"), (4, None, "offsets is NULL with G=4"), (5, ODD, "rows", "aligned"),
                         (6, None, "X is NULL"), (7, 127, "row stride"), (8, None, "xs is NULL"), (9, None, "W is NULL"),
                         (10, ODD, "ws", "aligned"), (11, ODD, "Y", "aligned"), (12, 63, "Y has row stride")):
        _refused(fn, _swap(good, i, v), ALLEGRO_E_INVALID, *words)


def test_binding_refuses_wrong_tensors():
    """On the CPU every tensor is on the wrong device; types and shapes are refused before that is looked at."""
    torch = pytest.importorskip("torch")
    x, w, off = torch.zeros(4, 8), torch.zeros(2, 8, 3), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="must live on"):
        latent.allegro_grouped_matmul(x, w, off)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        latent.allegro_grouped_matmul(x.double(), w, off)
    with pytest.raises(ValueError, match="two dimensions"):
        latent.allegro_rms_norm_forward(x[0], torch.ones(8))
    with pytest.raises(ValueError, match="K, N"):
        latent.allegro_grouped_matmul(x, w[0], off)
    with pytest.raises(TypeError, match="types"):
        latent.allegro_group_rows([0, 1], 2)
