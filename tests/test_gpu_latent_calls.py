"""How the latent operators are called, on the GPU: optional arguments, streams, aliases, the largest sizes.

Parity with the oracle over sizes and types is in test_gpu_latent.py.
"""

import numpy as np
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


# ---------------------------------------------------------------------- SiLU

@pytest.mark.parametrize("m", [1000, 70000], ids=["tiles", "streamed"])
def test_silu_over_its_range(at, m):
    """fp32 SiLU and its derivative on arguments from -87 to 40, through products with the identity.

    Bounds in units of 2^-24: SiLU 7 + |a| / 21 of its value, the derivative 16 + |a| / 21 of the magnitudes of its
    terms s and a s (1 - s); a product with the identity adds its operand's three parts, exact but for the
    instruction's rounding down of at most 2 units of the value; values below 2^-119 may be zero.  The gradient of W
    takes one row at a time."""
    _note(f"[gpu] SiLU from -87 to 40, M={m}")
    k = 64
    x = torch.linspace(-87.0, 40.0, m * k).view(k, m).t().contiguous()
    x[0, :4] = torch.tensor([-1.278464555740, 0.0, -0.0, 1e-30])  # the derivative's zero, and about 0
    eye, off = torch.eye(k, device=DEV)[None], torch.tensor([0, m], device=DEV)
    silu, U, tiny = at.ALLEGRO_ACT_SILU, 2.0 ** -24, 2.0 ** -119
    a = x.numpy().astype(np.longdouble)
    s, rest = 1 / (1 + np.exp(-a)), 1 / (1 + np.exp(a))
    value, terms = a * s, s * (1 + np.abs(a) * rest)
    slope = s * (1 + a * rest)
    far = np.abs(a) / 21

    def within(got, ref, tol, tag):
        err = np.abs(got.cpu().numpy() - ref)
        _note(f"  {tag}: largest error {float(np.max(err / tol)):.2g} of its bound")
        assert np.all(err <= tol), tag

    y = at.allegro_grouped_matmul(x.to(DEV), eye, off, act=silu)
    within(y, value, (9 + far) * U * np.abs(value) + tiny, "silu")
    dx, _ = at.allegro_grouped_matmul_backward(x.to(DEV), eye, torch.ones(m, k, device=DEV), off, act=silu, need_dw=False)
    within(dx, slope, (18 + far) * U * terms + tiny, "derivative")
    g = 500  # rows that are groups of their own
    _, dw = at.allegro_grouped_matmul_backward(x[:g].to(DEV), eye.expand(g, k, k).contiguous(),
                                               torch.eye(k)[torch.arange(g) % k].to(DEV),
                                               torch.arange(g + 1, device=DEV), act=silu, need_dx=False)
    want = np.zeros((g, k, k), np.longdouble)
    want[np.arange(g), :, np.arange(g) % k] = value[:g]
    within(dw, want, (9 + 87 / 21) * U * np.abs(want) + tiny, "weight gradient")
    # what the formulas give at the ends
    ends = torch.tensor([[float("inf"), float("-inf"), float("nan"), -1e30, 1e30, -3e38]], device=DEV).t().contiguous()
    one, two = torch.ones(1, 1, 1, device=DEV), torch.tensor([0, 6], device=DEV)
    y = at.allegro_grouped_matmul(ends, one, two, act=silu)[:, 0].cpu()
    assert y[0] == float("inf") and y[1:3].isnan().all() and y[3] == 0 and y[4] == ends[4, 0] and y[5] == 0
    dx, _ = at.allegro_grouped_matmul_backward(ends, one, torch.ones(6, 1, device=DEV), two, act=silu, need_dw=False)
    dx = dx[:, 0].cpu()
    assert dx[:3].isnan().all() and dx[3] == 0 and dx[4] == 1 and dx[5] == 0
