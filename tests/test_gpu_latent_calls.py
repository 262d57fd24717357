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


# ------------------------------------------------------------------- streams

def test_calls_on_a_stream_own_what_they_allocate(at):
    """Every call with stream= and nothing passed in: the results of the current stream's calls, from memory of the
    given stream's own pool."""
    _note("[gpu] latent operators with stream=")
    m, k, n, g = 70000, 128, 64, 5
    gen = _gen(2)
    t = torch.randint(-1, g, (m,), generator=gen, dtype=torch.int32).to(DEV)
    x, dy, w = _normal(gen, m, k).to(DEV), _normal(gen, m, n).to(DEV), _normal(gen, g, k, n).to(DEV)
    norm_w = torch.ones(k, device=DEV)
    w8, ws = _normal(gen, g, n, k).to(F8).to(DEV), torch.ones(g, 1, 1, device=DEV)

    def update(**kw):
        offsets, rows = at.allegro_group_rows(t, g, **kw)
        y, total, rstd = at.allegro_rms_norm_forward(x, norm_w, x, **kw)
        a = at.allegro_grouped_matmul(y, w, offsets, rows, act=at.ALLEGRO_ACT_SILU, **kw)
        da, dw = at.allegro_grouped_matmul_backward(y, w, dy, offsets, rows, act=at.ALLEGRO_ACT_SILU, **kw)
        dx, dnorm = at.allegro_rms_norm_backward(total, norm_w, rstd, da, da, **kw)
        q, scale, _ = at.allegro_rms_norm_fp8(x, norm_w, x, **kw)
        return [offsets, rows, y, total, rstd, a, da, dw, dx, dnorm, q.view(torch.uint8), scale,
                at.allegro_grouped_matmul_fp8(q, scale, w8, ws, offsets, rows, **kw)]

    def pool(handle):
        return sum(s["allocated_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == handle)

    want = update()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    here, there = pool(torch.cuda.current_stream().cuda_stream), pool(side.cuda_stream)
    got = update(stream=side)
    assert pool(torch.cuda.current_stream().cuda_stream) == here
    assert pool(side.cuda_stream) - there >= sum(v.numel() * v.element_size() for v in got)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
