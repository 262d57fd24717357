"""Calls of the latent operators that are refused on the host (no GPU), beyond those of test_latent_abi_cpu.py."""

import pytest

torch = pytest.importorskip("torch")
latent = pytest.importorskip("paper_2504_16068_amd.latent",
                             reason="libraries not built (run __graft_entry__.build())")
from paper_2504_16068_amd.binding import ALLEGRO_E_INVALID  # noqa: E402

X, W, Y, DY, DX, DW, WS, OFF, XS, WSC = (0x10000 * i for i in range(1, 11))


def _refused(fn, args, *words):
    rc = fn(*args)
    message = latent.allegro_latent_last_error()
    assert rc == ALLEGRO_E_INVALID, (rc, message)
    for w in words:
        assert w in message, message


def test_products_refuse_an_output_over_an_input():
    """A workgroup reads rows of its inputs that another has written by then."""
    lib = latent.library()
    for out in (X, W):
        _refused(lib.allegro_grouped_matmul, [0, 0, 100, 64, 64, 4, OFF, None, X, 64, W, out, 64, None], "Y is also an input")
    # dtype, act, M, K, N, G, offsets, rows, X, ldx, W, dY, lddy, dX, lddx, dW, workspace, bytes, stream
    for dx, dw, word in ((DY, None, "dX"), (DY, DW, "dX"), (X, DW, "dX"), (W, None, "dX"), (DX, X, "dW"), (None, DY, "dW")):
        _refused(lib.allegro_grouped_matmul_backward,
                 [1, 1, 100, 64, 64, 4, OFF, None, X, 64, W, DY, 64, dx, 64, dw, WS, 1 << 30, None], word + " is also an input")
    for out in (X, XS, W, WSC):
        _refused(lib.allegro_grouped_matmul_fp8, [10, 128, 64, 4, OFF, None, X, 128, XS, W, WSC, out, 64, None],
                 "Y is also an input")


def test_sizes_beyond_a_c_int_are_refused():
    """ctypes takes a number's low 32 bits: 2^32 + 4 groups or columns must not pass for 4."""
    big = 2 ** 32 + 4
    for fn, args, word in ((latent.allegro_group_rows_workspace, (10, big), "G="),
                           (latent.allegro_group_rows_workspace, (10, 4 - 2 ** 32), "G="),
                           (latent.allegro_group_rows_workspace, (2 ** 64 + 10, 4), "M="),
                           (latent.allegro_grouped_matmul_workspace, (10, big, 4, 4), "K="),
                           (latent.allegro_grouped_matmul_workspace, (10, 4, big, 4), "N="),
                           (latent.allegro_rms_norm_workspace, (10, big), "C=")):
        with pytest.raises(latent.AllegroError, match=word) as ex:
            fn(*args)
        assert ex.value.code == ALLEGRO_E_INVALID
    with pytest.raises(latent.AllegroError, match="groups"):
        latent._weights(torch.empty(1, 1, 1).expand(big, 1, 1), "K, N")
    # a tensor's width is its row stride too, which C takes in 64 bits
    _refused(latent.library().allegro_rms_norm_forward, [0, 1, 4, 1e-6, X, big, None, 0, W, None, 0, Y, big, None, None],
             "row stride")
