"""How the latent operators are called, on the GPU: optional arguments, streams, aliases, the largest sizes.

Parity with the oracle over sizes and types is in test_gpu_latent.py.
"""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_latent import BF16, DEV, F8, _gen, _normal, _note, at  # noqa: E402, F401


# --------------------------------------------------------- optional arguments

@pytest.mark.parametrize("m,k,n", [(300, 256, 96), (131072, 256, 128)], ids=["tiles", "streamed"])
def test_f8_products_without_offsets_ignore_rows(at, m, k, n):
    """Without offsets every row is in the one group, whatever a row list says."""
    _note(f"[gpu] 8-bit product without offsets but with a row list M={m}")
    gen = _gen(m)
    q, w = _normal(gen, m, k).to(F8).to(DEV), _normal(gen, 1, n, k).to(F8).to(DEV)
    xs, ws = torch.rand(m, 2, generator=gen).to(DEV), torch.rand(1, 1, 2, generator=gen).to(DEV)
    want = at.allegro_grouped_matmul_fp8(q, xs, w, ws)
    for rows in (torch.full((m,), -1), torch.zeros(m), torch.arange(m).flip(0)):
        out = torch.full((m, n), 3.0, dtype=BF16, device=DEV)
        got = at.allegro_grouped_matmul_fp8(q, xs, w, ws, rows=rows.to(torch.int32).to(DEV), out=out)
        assert torch.equal(got, want)
