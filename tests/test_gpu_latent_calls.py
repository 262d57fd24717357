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


# -------------------------------------------------------------- largest sizes

MOST = 2 ** 31 - 1  # rows


def _needs(gib):
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0] / 2 ** 30
    if free < gib:
        pytest.skip(f"needs {gib} GiB of GPU memory, {free:.0f} are free")


def _parts(m, part=2 ** 27):
    return [slice(i, min(i + part, m)) for i in range(0, m, part)]


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
def test_products_of_the_most_rows(at, dtype):
    """2^31 - 1 rows of one column are more tiles than a launch has workgroups for.  A product of one term is exact
    in fp32 up to the parts that are left out (2^-24) and the roundings of six sums, and rounded once in bf16."""
    _needs(40 if dtype is torch.float32 else 20)
    _note(f"[gpu] product of 2^31 - 1 rows {dtype}")
    base = torch.randn(2 ** 20, generator=_gen(1)).to(dtype).to(DEV)
    x = torch.empty(MOST, 1, dtype=dtype, device=DEV)
    for s in _parts(MOST, 2 ** 20):
        x[s, 0] = base[:s.stop - s.start]
    w = torch.tensor([1.25, -0.75], device=DEV).to(dtype).view(2, 1, 1)
    cut, end = MOST // 3 + 5, MOST - 1001  # two groups, and rows of none
    off = torch.tensor([0, cut, end], device=DEV)
    y = torch.full((MOST, 1), 7.0, dtype=dtype, device=DEV)
    at.allegro_grouped_matmul(x, w, off, out=y)
    dx = torch.full((MOST, 1), 7.0, dtype=dtype, device=DEV) if dtype is BF16 else None
    if dx is not None:
        at.allegro_grouped_matmul_backward(x, w, x, off, dx=dx, need_dw=False)
    for s in _parts(MOST):
        r = torch.arange(s.start, s.stop, device=DEV)
        factor = torch.where(r < cut, 1.25, torch.where(r < end, -0.75, 0.0))
        want = x[s, 0].float() * factor
        for got in (y,) if dx is None else (y, dx):
            if dtype is BF16:
                assert torch.equal(got[s, 0], want.to(BF16)), s
            else:
                assert bool(((got[s, 0] - want).abs() <= 8 * 2.0 ** -24 * want.abs()).all()), s
    torch.cuda.empty_cache()


def test_f8_products_of_the_most_rows(at):
    """As above with 8-bit operands: one term of values that are powers of two is exact."""
    _needs(40)
    _note("[gpu] 8-bit product of 2^31 - 1 rows")
    base = torch.exp2(torch.randint(-6, 8, (2 ** 20,), generator=_gen(2)).float()).to(F8).to(DEV)
    x = torch.empty(MOST, 1, dtype=F8, device=DEV)
    for s in _parts(MOST, 2 ** 20):
        x[s, 0] = base[:s.stop - s.start]
    xs = torch.full((MOST, 1), 0.5, device=DEV)
    xs[MOST // 2:] = 0.25
    w, ws = torch.full((1, 1, 1), 4.0, device=DEV).to(F8), torch.ones(1, 1, 1, device=DEV)
    y = at.allegro_grouped_matmul_fp8(x, xs, w, ws, out=torch.full((MOST, 1), 7.0, dtype=BF16, device=DEV))
    for s in _parts(MOST):
        assert torch.equal(y[s, 0].float(), x[s, 0].float() * xs[s, 0] * 4.0), s
    torch.cuda.empty_cache()


def test_norm_of_many_long_rows(at):
    """2^27 rows of 257 columns: more row groups than a launch has workgroups for.  Rows that repeat have the
    results of a call on the first of them."""
    _needs(150)
    _note("[gpu] norm of 2^27 rows of 257 columns")
    m, c, n = 2 ** 27, 257, 4096
    base, w = _normal(_gen(3), n, c, dtype=BF16).to(DEV), torch.ones(c, device=DEV)
    x = torch.empty(m, c, dtype=BF16, device=DEV)
    x.view(m // n, n, c).copy_(base)
    want, want_scale, _ = at.allegro_rms_norm_fp8(base, w)
    q = torch.empty(m, c, dtype=F8, device=DEV)
    q.view(torch.uint8).fill_(0x7F)
    scale = torch.zeros(m, 3, device=DEV)
    at.allegro_rms_norm_fp8(x, w, q=q, scale=scale)
    del x
    q = q.view(torch.uint8).view(m // n, n, c)
    for s in _parts(m // n, 1024):
        assert bool((q[s] == want.view(torch.uint8)).all()) and bool((scale.view(m // n, n, 3)[s] == want_scale).all()), s
    del q, scale
    torch.cuda.empty_cache()


# ------------------------------------------------------------------- aliases

@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,c", [(500, 3), (500, 65), (300, 1031), (40, 4096), (40, 4097), (5000, 4100), (9, 65536)])
def test_norm_in_place_of_an_operand(at, dtype, m, c):
    """total written over x or over the residual: the results of the call with a tensor of its own."""
    _note(f"[gpu] norm with total in place M={m} C={c} {dtype}")
    gen = _gen(c)
    x, r = (_normal(gen, m, c, dtype=dtype).to(DEV) for _ in range(2))
    w = (1 + _normal(gen, c, scale=0.3)).to(DEV)
    want = at.allegro_rms_norm_forward(x, w, r)
    want8 = at.allegro_rms_norm_fp8(x, w, r)
    for i in (0, 1):
        args = [x.clone(), r.clone()]
        y, total, rstd = at.allegro_rms_norm_forward(args[0], w, args[1], total=args[i])
        assert total is args[i] and all(torch.equal(a, b) for a, b in zip((y, total, rstd), want))
        args = [x.clone(), r.clone()]
        q, scale, total = at.allegro_rms_norm_fp8(args[0], w, args[1], total=args[i])
        assert torch.equal(q.view(torch.uint8), want8[0].view(torch.uint8)) and torch.equal(scale, want8[1])
        assert torch.equal(total, want8[2])
