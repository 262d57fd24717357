"""GPU parity of the latent track's operators (include/allegro_latent.h) against the fp64 oracle.

Bounds, by element, with S the sum of the magnitudes of a sum's terms:

* fp32 products: six chained sums per step of 32 (each may round down by a unit of
  fp32, and 32 terms enter it), one rounding per step, and 2^-24 for the parts that
  are left out: (48 + K / 16) 2^-24 S.  SiLU from the hardware's exponential and
  reciprocal: 16 2^-24 S for arguments up to 6.  A bfloat16 output adds half a unit
  (8 significant bits: 2^-8), SiLU as a bfloat16 operand 2^-8 S.
* norm: the sum of squares has no cancellation, so its relative error is at most
  its depth, C / 64 + 10 units; everything behind it a few roundings.
* 8 bits: half a unit (2^-4 of the value, 2^-10 below the normal range) of y / scale.
* 8-bit products: each 8 products are added in units of 2^-13 of the largest, so the 7
  others lose at most 7 2^-13 of it: 7 2^-13 S, and the bfloat16 output's 2^-8.  Of
  many independent errors the 2-norm is that of the output's rounding, at most
  2^-8 / sqrt(3), to a tenth.
"""

import sys

import numpy as np
import pytest

from oracle import latent as ol

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


def _note(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def at():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import paper_2504_16068_amd as lib
    return lib


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _normal(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def _dev(t, pad=0, shift=0):
    """The tensor on the GPU; with pad as columns of a wider one, with shift off its alignment."""
    if pad == 0 and shift == 0:
        return t.to(DEV)
    m, c = t.shape
    buf = torch.full((m * (c + pad) + shift + 16,), 7.0, dtype=F32).to(t.dtype).to(DEV)
    view = buf[shift:shift + m * (c + pad)].view(m, c + pad)[:, :c]
    view.copy_(t)
    return view


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _types(gen, m, g, untyped=True):
    t = torch.randint(-1 if untyped else 0, g, (m,), generator=gen, dtype=torch.int32)
    if g > 2:
        t[t == 1] = 0  # a group without rows, and a larger one
    return t


def _within(got, ref, tol, tag):
    got, tol = _f64(got), np.broadcast_to(tol, ref.shape)
    assert got.shape == ref.shape, (tag, got.shape, ref.shape)
    if ref.size == 0:
        return
    assert np.all(np.isfinite(got)), f"{tag}: not finite"
    over = np.abs(got - ref) - tol
    i = np.unravel_index(np.argmax(over), over.shape)
    worst = float(np.max(np.abs(got - ref) / np.maximum(tol, 1e-300)))
    _note(f"  {tag}: largest error {worst:.2g} of its bound")
    assert over[i] <= 0, f"{tag}: {got[i]} against {ref[i]} at {i}, bound {tol[i]}"


# ---------------------------------------------------------------- grouping

@pytest.mark.parametrize("m,g", [(1, 1), (63, 4), (64, 3), (1142, 4), (4096, 1024), (4097, 16), (52180, 225), (8192, 1),
                                 (200003, 100), (2300001, 7)])
def test_group_rows(at, m, g):
    _note(f"[gpu] group_rows M={m} G={g}")
    gen = _gen(m + g)
    t = torch.randint(-3, g + 2, (m,), generator=gen, dtype=torch.int32)
    t[torch.rand(m, generator=gen) < 0.4] = g // 2  # one type with many rows
    key = np.where((t.numpy() >= 0) & (t.numpy() < g), t.numpy(), g)
    offsets, rows = at.allegro_group_rows(t.to(DEV), g)
    assert np.array_equal(rows.cpu().numpy(), np.argsort(key, kind="stable"))
    counts = np.bincount(key, minlength=g + 1)[:g]
    assert np.array_equal(offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(counts)]))


@pytest.mark.parametrize("m,g", [(131072, 255), (131073, 16), (9000, 256), (30000, 1000), (1048820, 225)])
def test_group_rows_by_chunks(at, m, g):
    """Few and many chunks of rows, types by the hundred."""
    test_group_rows(at, m, g)


def test_group_rows_without_rows_or_types(at):
    offsets, rows = at.allegro_group_rows(torch.empty(0, dtype=torch.int32, device=DEV), 5)
    assert offsets.tolist() == [0] * 6 and rows.numel() == 0
    offsets, rows = at.allegro_group_rows(torch.full((5000,), -1, dtype=torch.int32, device=DEV), 3)
    assert offsets.tolist() == [0] * 4 and rows.tolist() == list(range(5000))


# ---------------------------------------------------------------- products

def _product_case(at, m, k, n, g, dtype, act, pad=0, shift=0, listed=True, seed=0):
    gen = _gen(seed + 1000 * m + 10 * k + n)
    t = _types(gen, m, g, untyped=listed)
    x = _normal(gen, m, k, dtype=dtype).clamp_(-6, 6)
    w = _normal(gen, g, k, n, dtype=dtype, scale=k ** -0.5)
    dy = _normal(gen, m, n, dtype=dtype)
    if listed:
        offsets, rows = at.allegro_group_rows(t.to(DEV), g)
    else:
        t = t.sort().values
        offsets, rows = at.allegro_group_rows(t.to(DEV), g)[0], None
    a = at.ALLEGRO_ACT_SILU if act else at.ALLEGRO_ACT_NONE
    xd, wd, dyd = _dev(x, pad, shift), w.to(DEV), _dev(dy, pad, shift)
    y = at.allegro_grouped_matmul(xd, wd, offsets, rows, act=a, out=_dev(torch.full((m, n), 3.0).to(dtype), pad, shift))
    dx, dw = at.allegro_grouped_matmul_backward(xd, wd, dyd, offsets, rows, act=a,
                                                dx=_dev(torch.full((m, k), 3.0).to(dtype), pad, shift))
    torch.cuda.synchronize()
    t, x, w, dy = t.numpy(), _f64(x), _f64(w), _f64(dy)
    half = 2.0 ** -8 if dtype is BF16 else U  # rounding of an output
    extra = ((2.0 ** -8 if dtype is BF16 else 0.0) + 16 * U) if act else 0.0
    z = np.abs(ol.silu(x)) if act else np.abs(x)
    ref = ol.grouped_matmul(t, x, w, act)
    s = ol.grouped_matmul(t, z, np.abs(w), False)
    _within(y, ref, half * np.abs(ref) + ((48 + k / 16) * U + extra) * s, "y")
    rdx, rdw = ol.grouped_matmul_backward(t, x, w, dy, act)
    up, s = (ol.grouped_matmul(t, a, np.swapaxes(b, 1, 2), False) for a, b in ((dy, w), (np.abs(dy), np.abs(w))))
    tol = half * np.abs(rdx) + (48 + n / 16) * U * s * (np.abs(ol.silu_grad(x)) if act else 1.0)
    if act:
        tol = tol + 16 * U * (1 + np.abs(x)) * np.abs(up)
    _within(dx, rdx, tol, "dx")
    _, s = ol.grouped_matmul_backward(t, z, np.abs(w), np.abs(dy), False)
    rows_of = max(1, int(np.bincount(t[t >= 0], minlength=g).max()) if np.any(t >= 0) else 1)
    _within(dw, rdw, half * np.abs(rdw) + ((48 + rows_of / 16) * U + extra) * s, "dw")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("act", [False, True], ids=["plain", "silu"])
@pytest.mark.parametrize("m,k,n,g", [
    (1, 64, 64, 1), (1, 1, 1, 3), (7, 3, 5, 2), (128, 128, 128, 1), (129, 65, 33, 4), (300, 128, 64, 16),
    (1142, 64, 128, 4), (777, 192, 128, 5), (513, 40, 200, 3), (260, 257, 129, 70), (3700, 128, 64, 16),
    (900, 512, 320, 6), (2049, 96, 72, 1000)])
def test_products(at, dtype, act, m, k, n, g):
    _note(f"[gpu] product M={m} K={k} N={n} G={g} {dtype} act={act}")
    _product_case(at, m, k, n, g, dtype, act)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (24, 4)])
def test_products_strides_and_alignment(at, dtype, pad, shift):
    _note(f"[gpu] product strides pad={pad} shift={shift} {dtype}")
    _product_case(at, 333, 72, 136, 3, dtype, True, pad, shift)
    _product_case(at, 333, 64, 64, 3, dtype, False, pad, shift)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_products_without_row_list(at, dtype):
    _note(f"[gpu] product without a row list {dtype}")
    _product_case(at, 1000, 64, 96, 5, dtype, False, listed=False)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,k,n,g", [(30000, 64, 64, 3), (30011, 128, 96, 4), (70001, 33, 65, 2)])
def test_products_over_many_rows(at, dtype, m, k, n, g):
    """Groups of several ranges of rows, whose partial weight gradients are summed."""
    _note(f"[gpu] product M={m} K={k} N={n} G={g} {dtype}")
    _product_case(at, m, k, n, g, dtype, True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,k,n,g", [(9000, 300, 500, 4), (17003, 257, 390, 6), (66000, 513, 390, 3), (30000, 400, 256, 200)])
def test_products_over_many_tiles(at, dtype, m, k, n, g):
    """Grids from a tile to a compute unit up to many, whose tiles are of other widths."""
    _note(f"[gpu] product M={m} K={k} N={n} G={g} {dtype} many tiles")
    _product_case(at, m, k, n, g, dtype, True)


@pytest.mark.parametrize("m,k,n,g,act", [(66003, 192, 128, 3, False), (70000, 128, 64, 100, True), (65600, 20, 130, 16, True),
                                         (65536, 65, 191, 5, False), (90001, 4, 3, 128, False), (65537, 384, 61, 2, True)])
def test_products_of_many_rows(at, m, k, n, g, act):
    """fp32 rows that are streamed past stationary weights, with rows of no type and types of few rows."""
    _note(f"[gpu] product M={m} K={k} N={n} G={g} f32 streamed")
    _product_case(at, m, k, n, g, F32, act)


def test_products_of_many_rows_special_values(at):
    gen = _gen(13)
    m, k, n = 66000, 72, 70
    x, w, dy = _normal(gen, m, k), _normal(gen, 2, k, n), _normal(gen, m, n)
    x[3, 5], x[40000, 69], x[40031, 0], x[65999, 7] = float("inf"), float("nan"), float("-inf"), 3e38
    t = torch.randint(-1, 2, (m,), generator=gen, dtype=torch.int32)
    t[[3, 40000, 40031, 65999]] = 1
    offsets, rows = at.allegro_group_rows(t.to(DEV), 2)
    y = _f64(at.allegro_grouped_matmul(x.to(DEV), w.to(DEV), offsets, rows))
    ref = ol.grouped_matmul(t.numpy(), _f64(x), _f64(w), False)
    over = np.abs(ref) > 3.5e38  # beyond fp32
    assert np.array_equal(np.isnan(y), np.isnan(ref))
    assert np.array_equal(y[np.isinf(ref)], ref[np.isinf(ref)]) and np.all(np.isinf(y[over & np.isfinite(ref)]))
    ordinary = np.ones(m, bool)
    ordinary[[3, 40000, 40031, 65999]] = False
    assert np.max(np.abs(y - ref)[ordinary]) <= 1e-4
    # many rows whose list is out of order or range
    for off in ([0, 50000, 100], [-5, 1 << 40, 20], [m, 0, 0]):
        bad = torch.randint(-1000, 2 * m, (m,), generator=gen, dtype=torch.int32).to(DEV)
        at.allegro_grouped_matmul(x.to(DEV), w.to(DEV), torch.tensor(off, device=DEV), bad)
        at.allegro_grouped_matmul_backward(x.to(DEV), w.to(DEV), dy.to(DEV), torch.tensor(off, device=DEV), bad)
    torch.cuda.synchronize()


def test_products_without_any_row(at):
    for dtype in (F32, BF16):
        x, w = torch.empty(0, 12, dtype=dtype, device=DEV), torch.randn(3, 12, 20, device=DEV).to(dtype)
        offsets = torch.zeros(4, dtype=torch.int64, device=DEV)
        assert at.allegro_grouped_matmul(x, w, offsets).shape == (0, 20)
        dx, dw = at.allegro_grouped_matmul_backward(x, w, torch.empty(0, 20, dtype=dtype, device=DEV), offsets)
        assert dx.shape == (0, 12) and torch.count_nonzero(dw) == 0
        # rows, but none with a type
        x = torch.randn(300, 12, device=DEV).to(dtype)
        offsets, rows = at.allegro_group_rows(torch.full((300,), 9, dtype=torch.int32, device=DEV), 3)
        dy = torch.randn(300, 20, device=DEV).to(dtype)
        y = at.allegro_grouped_matmul(x, w, offsets, rows)
        dx, dw = at.allegro_grouped_matmul_backward(x, w, dy, offsets, rows)
        assert all(torch.count_nonzero(v) == 0 for v in (y, dx, dw))


def test_products_partial_outputs(at):
    """Either gradient alone equals that of the call for both."""
    gen = _gen(9)
    x, w, dy = (_normal(gen, *s).to(DEV) for s in ((700, 64), (4, 64, 80), (700, 80)))
    offsets, rows = at.allegro_group_rows(_types(gen, 700, 4).to(DEV), 4)
    dx, dw = at.allegro_grouped_matmul_backward(x, w, dy, offsets, rows)
    only_dx, none = at.allegro_grouped_matmul_backward(x, w, dy, offsets, rows, need_dw=False)
    assert none is None and torch.equal(only_dx, dx)
    none, only_dw = at.allegro_grouped_matmul_backward(x, w, dy, offsets, rows, need_dx=False)
    assert none is None and torch.equal(only_dw, dw)


def test_products_gradients_against_differences(at):
    """Central differences of the forward in fp32 along random directions.  The step's error is h^2 / 6 of third
    derivatives (about 1 here), the forward's 1e-6 of sums of about 1e2 terms over 2 h."""
    gen = _gen(4)
    x, w, dy = _normal(gen, 500, 48), _normal(gen, 3, 48, 40, scale=0.15), _normal(gen, 500, 40)
    offsets, rows = at.allegro_group_rows(_types(gen, 500, 3).to(DEV), 3)
    xd, wd, dyd = x.to(DEV), w.to(DEV), dy.to(DEV)
    dx, dw = at.allegro_grouped_matmul_backward(xd, wd, dyd, offsets, rows, act=at.ALLEGRO_ACT_SILU)

    def loss(a, b):
        return float((at.allegro_grouped_matmul(a, b, offsets, rows, act=at.ALLEGRO_ACT_SILU).double()
                      * dyd.double()).sum())

    h = 2.0 ** -7
    for got, base, arg in ((dx, xd, 0), (dw, wd, 1)):
        d = _normal(gen, *base.shape).to(DEV)
        args = [xd, wd]
        args[arg] = base + h * d
        up = loss(*args)
        args[arg] = base - h * d
        num = (up - loss(*args)) / (2 * h)
        want = float((got.double() * d.double()).sum())
        scale = float((got.double().norm() * d.double().norm()))
        assert abs(num - want) <= 1e-3 * scale, (num, want, scale)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_products_special_values(at, dtype):
    """Infinities and NaN reach what the formulas say and nothing else; fp32 holds its whole range."""
    gen = _gen(12)
    m, k, n = 260, 70, 68
    x, w = _normal(gen, m, k, dtype=dtype), _normal(gen, 1, k, n, dtype=dtype)
    x[3, 5], x[40, 69], x[41, 0], x[200, 7] = float("inf"), float("nan"), float("-inf"), float("inf")
    w[0, 7, 11] = 0.0  # infinity times zero
    offsets = torch.tensor([0, m], device=DEV)
    y = at.allegro_grouped_matmul(x.to(DEV), w.to(DEV), offsets)
    ref = ol.grouped_matmul(np.zeros(m, int), _f64(x), _f64(w), False)
    got = _f64(y)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]) and not np.any(np.isinf(got[np.isfinite(ref)]))
    fine = np.isfinite(ref)
    assert np.max(np.abs(got - ref)[fine]) <= (1e-4 if dtype is F32 else 0.3)
    if dtype is BF16:
        return
    # near the ends of the range: results that are normal numbers, from operands that no scale holds
    for sx, sw in ((2.0 ** 120, 2.0 ** -115), (2.0 ** -120, 2.0 ** 90), (2.0 ** -140, 2.0 ** 60), (2.0 ** 100, 2.0 ** -20)):
        xs, wsc = (_normal(gen, m, k).double() * sx).float(), (_normal(gen, 1, k, n).double() * sw).float()
        ref = ol.grouped_matmul(np.zeros(m, int), _f64(xs), _f64(wsc), False)
        s = ol.grouped_matmul(np.zeros(m, int), np.abs(_f64(xs)), np.abs(_f64(wsc)), False)
        _within(at.allegro_grouped_matmul(xs.to(DEV), wsc.to(DEV), offsets), ref, (48 + k / 4) * U * s + 2.0 ** -126,
                f"scales {sx:g} {sw:g}")
    # a weight gradient with an infinity in one row of one column
    x, dy = _normal(gen, m, k), _normal(gen, m, n)
    x[100, 9] = float("inf")
    _, dw = at.allegro_grouped_matmul_backward(x.to(DEV), w.to(DEV), dy.to(DEV), offsets)
    _, ref = ol.grouped_matmul_backward(np.zeros(m, int), _f64(x), _f64(w), _f64(dy), False)
    got = _f64(dw)
    assert np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)]) and np.all(np.isfinite(got[np.isfinite(ref)]))


def test_products_mean_error(at):
    """The matrix instructions round down; over rows and steps nothing of it may add up: the mean error of 2e6
    values, relative to their terms' magnitudes, stays below 4 / sqrt(count) times their spread."""
    gen = _gen(77)
    m, k, n = 16384, 64, 128
    x, w = _normal(gen, m, k).abs(), _normal(gen, 1, k, n).abs()
    offsets = torch.tensor([0, m], device=DEV)
    y = _f64(at.allegro_grouped_matmul(x.to(DEV), w.to(DEV), offsets))
    ref = _f64(x) @ _f64(w)[0]
    rel = (y - ref) / ref
    _note(f"  mean {rel.mean():.2e}, spread {rel.std():.2e}")
    assert abs(rel.mean()) <= 0.02 * rel.std() and rel.std() <= 4 * U


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_products_long_offsets(at, dtype):
    """Rows that start beyond 2^32 bytes and 2^31 elements of their tensor."""
    m, ld, k, n = 40000, 65536, 64, 64
    x = torch.empty(m * ld, dtype=dtype, device=DEV).view(m, ld)[:, :k]
    gen = _gen(5)
    xs, w = _normal(gen, m, k, dtype=dtype), _normal(gen, 2, k, n, dtype=dtype, scale=0.125)
    x.copy_(xs)
    t = torch.randint(0, 2, (m,), generator=gen, dtype=torch.int32)
    offsets, rows = at.allegro_group_rows(t.to(DEV), 2)
    y = at.allegro_grouped_matmul(x, w.to(DEV), offsets, rows)
    same = at.allegro_grouped_matmul(xs.to(DEV), w.to(DEV), offsets, rows)
    assert torch.equal(y, same)
    _, dw = at.allegro_grouped_matmul_backward(x, w.to(DEV), y, offsets, rows)
    _, dws = at.allegro_grouped_matmul_backward(xs.to(DEV), w.to(DEV), y, offsets, rows)
    assert torch.equal(dw, dws)
    ref = ol.grouped_matmul(t.numpy()[-500:], _f64(xs)[-500:], _f64(w), False)
    s = ol.grouped_matmul(t.numpy()[-500:], np.abs(_f64(xs))[-500:], np.abs(_f64(w)), False)
    _within(y[-500:], ref, (2.0 ** -8 if dtype is BF16 else U) * np.abs(ref) + 52 * U * s, "last rows")


def test_products_bad_lists_stay_in_bounds(at):
    """Offsets out of order or range and rows out of range: checked indices, no access out of bounds."""
    gen = _gen(6)
    x, w, dy = (_normal(gen, *s).to(DEV) for s in ((500, 32), (3, 32, 48), (500, 48)))
    for off in ([0, 400, 100, 500], [-5, 10, 20, 1 << 40], [500, 500, 0, 0], [7, 7, 7, 7]):
        offsets = torch.tensor(off, device=DEV)
        rows = torch.randint(-1000, 1000, (500,), generator=gen, dtype=torch.int32).to(DEV)
        at.allegro_grouped_matmul(x, w, offsets, rows)
        at.allegro_grouped_matmul_backward(x, w, dy, offsets, rows)
    torch.cuda.synchronize()
    offsets = torch.tensor([0, 200, 300, 500], device=DEV)  # one row out of range among good ones
    rows = torch.arange(500, dtype=torch.int32, device=DEV)
    y = at.allegro_grouped_matmul(x, w, offsets, rows)
    rows[77] = 1 << 30
    other = at.allegro_grouped_matmul(x, w, offsets, rows, out=torch.zeros_like(y))
    keep = torch.arange(500, device=DEV) != 77
    assert torch.equal(y[keep], other[keep]) and torch.count_nonzero(other[77]) == 0


# -------------------------------------------------------------------- norm

def _norm_case(at, m, c, dtype, residual, pad=0, shift=0, eps=1e-6):
    gen = _gen(31 * m + c)
    x, r = _normal(gen, m, c, dtype=dtype), _normal(gen, m, c, dtype=dtype) if residual else None
    w, dy, ds = 1 + _normal(gen, c, scale=0.3), _normal(gen, m, c, dtype=dtype), _normal(gen, m, c, dtype=dtype)
    xd, rd, dyd = _dev(x, pad, shift), None if r is None else _dev(r, pad, shift), _dev(dy, pad, shift)
    dsd = _dev(ds, pad, shift) if residual else None
    wd = w.to(DEV)
    like = lambda: _dev(torch.zeros(m, c, dtype=dtype), pad, shift)  # noqa: E731
    y, total, rstd = at.allegro_rms_norm_forward(xd, wd, rd, eps=eps, out=like(), total=like() if residual else None)
    q, scale, total8 = at.allegro_rms_norm_fp8(xd, wd, rd, eps=eps)
    dx, dw = at.allegro_rms_norm_backward(total, wd, rstd, dyd, dsd, dx=like())
    torch.cuda.synchronize()
    half = 2.0 ** -8 if dtype is BF16 else U
    s = _f64(x) + (_f64(r) if residual else 0.0)
    ry, rr = ol.rms_norm(s, _f64(w), eps)
    depth = (c / 64 + 16) * U
    if residual:
        _within(total, s, half * np.abs(s) + U * np.abs(s), "total")
        assert torch.equal(total, total8)
    _within(rstd, rr, depth * rr, "rstd")
    _within(y, ry, (half + depth) * np.abs(ry) + 2 * U * np.abs(rr[:, None] * _f64(w)) * np.abs(s), "y")
    v, rs = ol.f8_blocks(ry)
    _within(scale, rs, (depth + 4 * U) * rs, "scale")
    q64 = q.cpu().to(F32).double().numpy()
    assert np.all(np.abs(q64 - v) <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10) + 4 * depth * np.abs(v)), "q"
    assert np.mean(q64 != ol.f8_round(v)) <= 16 * depth * 16 + 1.0 / v.size, "q is not the nearest value"
    # the backward starts from the total and rstd that were written
    t64, r64 = _f64(total), _f64(rstd)
    rdx, rdw = ol.rms_norm_backward(t64, _f64(w), r64, _f64(dy), _f64(ds) if residual else None)
    u, t = np.abs(t64 * r64[:, None]), np.abs(_f64(dy) * _f64(w))
    size = r64[:, None] * (t + u * np.mean(t * u, axis=1, keepdims=True))
    _within(dx, rdx, half * np.abs(rdx) + (c / 64 + 24) * U * size, "dx")
    _within(dw, rdw, (64 + m / 256) * U * np.sum(np.abs(_f64(dy)) * u, axis=0), "dw")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("residual", [True, False], ids=["residual", "alone"])
@pytest.mark.parametrize("m,c", [(1, 1), (1, 128), (5, 3), (64, 64), (333, 65), (100, 200), (77, 256), (1000, 16), (41, 1031),
                                 (33, 1024), (20, 2560), (9, 4096), (7, 4097), (6, 9000), (3, 65536)])
def test_norm(at, dtype, residual, m, c):
    _note(f"[gpu] norm M={m} C={c} {dtype} residual={residual}")
    _norm_case(at, m, c, dtype, residual)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (8, 4)])
def test_norm_strides_and_alignment(at, dtype, pad, shift):
    _note(f"[gpu] norm strides pad={pad} shift={shift} {dtype}")
    _norm_case(at, 130, 136, dtype, True, pad, shift)
    _norm_case(at, 19, 4104, dtype, True, pad, shift)


@pytest.mark.parametrize("m,c", [(30000, 128), (20011, 72)])
def test_norm_over_many_rows(at, m, c):
    _note(f"[gpu] norm M={m} C={c}")
    _norm_case(at, m, c, F32, True)


def test_norm_without_rows(at):
    w = torch.ones(40, device=DEV)
    x = torch.empty(0, 40, device=DEV)
    y, total, rstd = at.allegro_rms_norm_forward(x, w)
    dx, dw = at.allegro_rms_norm_backward(total, w, rstd, x)
    assert y.shape == dx.shape == (0, 40) and torch.count_nonzero(dw) == 0
    q, scale, _ = at.allegro_rms_norm_fp8(x, w)
    assert q.shape == (0, 40) and scale.shape == (0, 1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [64, 65, 300, 5000])
def test_norm_special_values(at, dtype, c):
    """Rows of zeros, of tiny and large values, with infinities and NaN: each row by itself."""
    x = torch.randn(6, c, generator=_gen(c)).to(dtype)
    x[1] = 0
    x[2] *= 2.0 ** -60
    x[3] *= 2.0 ** 50
    x[4, c // 2] = float("inf")
    x[5, c - 1] = float("nan")
    w = torch.ones(c, device=DEV)
    y, _, rstd = at.allegro_rms_norm_forward(x.to(DEV), w)
    q, scale, _ = at.allegro_rms_norm_fp8(x.to(DEV), w)
    ry, rr = ol.rms_norm(_f64(x)[:4], np.ones(c), 1e-6)
    assert np.allclose(_f64(y)[:4], ry, rtol=2.0 ** -8, atol=1e-30) and np.allclose(_f64(rstd)[:4], rr, rtol=1e-5)
    q, scale = q.cpu().to(F32).numpy(), scale.cpu().numpy()
    assert np.all(q[1] == 0) and np.all(scale[1] == np.float32(2.0 ** -126))
    back = ol.dequantise_rows(q[:4].astype(np.float64), scale[:4].astype(np.float64))
    assert np.all(np.abs(back - ry) <= 2.0 ** -4 * np.abs(ry) * 1.001 + 2.0 ** -10 * np.repeat(scale[:4], 128, 1)[:, :c])
    # infinity: rstd is zero, the infinite element NaN, the others zero; its block of 128 has no scale
    assert float(rstd[4]) == 0 and np.isnan(_f64(y)[4, c // 2]) and np.count_nonzero(np.nan_to_num(_f64(y)[4])) == 0
    b = c // 2 // 128
    assert np.isnan(scale[4, b]) and np.all(np.isnan(q[4, b * 128:(b + 1) * 128]))
    assert np.all(np.isnan(_f64(y)[5])) and np.all(np.isnan(scale[5])) and np.all(np.isnan(q[5]))


def test_norm_gradient_against_differences(at):
    gen = _gen(8)
    x, w = _normal(gen, 200, 96).to(DEV), (1 + _normal(gen, 96, scale=0.3)).to(DEV)
    dy, ds = _normal(gen, 200, 96).to(DEV), _normal(gen, 200, 96).to(DEV)
    r = _normal(gen, 200, 96).to(DEV)
    y, total, rstd = at.allegro_rms_norm_forward(x, w, r, eps=0.01)
    dx, dw = at.allegro_rms_norm_backward(total, w, rstd, dy, ds)

    def loss(a, b):
        y, total, _ = at.allegro_rms_norm_forward(a, b, r, eps=0.01)
        return float((y.double() * dy.double()).sum() + (total.double() * ds.double()).sum())

    h = 2.0 ** -7
    for got, d, args in ((dx, _normal(gen, 200, 96).to(DEV), 0), (dw, _normal(gen, 96).to(DEV), 1)):
        up = loss(x + h * d, w) if args == 0 else loss(x, w + h * d)
        down = loss(x - h * d, w) if args == 0 else loss(x, w - h * d)
        num, want = (up - down) / (2 * h), float((got.double() * d.double()).sum())
        assert abs(num - want) <= 1e-3 * float(got.double().norm() * d.double().norm()), (num, want)


# ---------------------------------------------------------- 8-bit products

def _f8_case(at, m, k, n, g, pad=0, shift=0, typed=True, rows=True):
    gen = _gen(7 * m + 3 * k + n)
    q = _normal(gen, m, k, scale=60.0).clamp_(-448, 448).to(F8)
    wq = _normal(gen, g, n, k, scale=60.0).clamp_(-448, 448).to(F8)
    kb, nb = -(-k // 128), -(-n // 128)
    xs = torch.exp2(torch.randn(m, kb, generator=gen) * 2)
    ws = torch.exp2(torch.randn(g, nb, kb, generator=gen) * 2)
    t = _types(gen, m, g)
    offsets = listed = None
    if typed:
        offsets, listed = at.allegro_group_rows(t.to(DEV), g)
        if not rows:
            t = torch.where(t < 0, 0, t).sort().values
            offsets, listed = at.allegro_group_rows(t.to(DEV), g)[0], None
    else:
        t = torch.zeros(m, dtype=torch.int32)
    if pad or shift:
        buf = torch.zeros(m * (k + pad) + shift + 16, dtype=torch.uint8, device=DEV)
        qd = buf[shift:shift + m * (k + pad)].view(m, k + pad)[:, :k]
        qd.copy_(q.view(torch.uint8))
        qd = qd.view(F8)
    else:
        qd = q.to(DEV)
    out = _dev(torch.full((m, n), 3.0).to(BF16), pad, shift) if pad or shift else None
    y = at.allegro_grouped_matmul_fp8(qd, xs.to(DEV), wq.to(DEV), ws.to(DEV), offsets, listed, out=out)
    torch.cuda.synchronize()
    q64, w64 = q.to(F32).double().numpy(), wq.to(F32).double().numpy()
    ref = ol.grouped_matmul_fp8(t.numpy(), q64, _f64(xs), w64, _f64(ws))
    s = ol.grouped_matmul_fp8(t.numpy(), np.abs(q64), _f64(xs), np.abs(w64), _f64(ws))
    _within(y, ref, 2.0 ** -8 * np.abs(ref) + 7 * 2.0 ** -13 * s, "y")
    if ref.size >= 1000:  # enough independent errors
        assert np.linalg.norm(_f64(y) - ref) <= 1.1 * 2.0 ** -8 / 3 ** 0.5 * np.linalg.norm(ref)


@pytest.mark.parametrize("m,k,n,g", [(1, 128, 128, 1), (1, 1, 1, 1), (130, 64, 48, 3), (300, 256, 512, 4), (257, 129, 200, 2),
                                     (500, 1024, 96, 16), (1142, 256, 512, 4), (99, 300, 77, 50), (640, 1040, 392, 5)])
def test_f8_products(at, m, k, n, g):
    _note(f"[gpu] 8-bit product M={m} K={k} N={n} G={g}")
    _f8_case(at, m, k, n, g)


@pytest.mark.parametrize("pad,shift", [(16, 0), (3, 0), (0, 1), (16, 16), (8, 8)])
def test_f8_products_strides_and_alignment(at, pad, shift):
    _note(f"[gpu] 8-bit product strides pad={pad} shift={shift}")
    _f8_case(at, 200, 272, 144, 3, pad, shift)
    _f8_case(at, 200, 128, 64, 3, pad, shift, rows=False)


@pytest.mark.parametrize("m,k,n,g,typed,rows", [(70000, 130, 160, 3, True, True), (131075, 16, 66, 100, True, True),
                                                (66001, 1152, 256, 2, True, False), (131072, 40, 128, 1, False, False),
                                                (65600, 257, 391, 64, True, True)])
def test_f8_products_of_many_rows(at, m, k, n, g, typed, rows):
    """Rows that are streamed past stationary weights."""
    _note(f"[gpu] 8-bit product M={m} K={k} N={n} G={g} streamed")
    _f8_case(at, m, k, n, g, typed=typed, rows=rows)
    if k == 130:
        _f8_case(at, m, k, n, g, 3, 1)


def test_f8_products_one_group(at):
    _note("[gpu] 8-bit product without offsets")
    _f8_case(at, 777, 384, 256, 1, typed=False)
    y = at.allegro_grouped_matmul_fp8(torch.empty(0, 128, device=DEV).to(F8), torch.empty(0, 1, device=DEV),
                                      torch.zeros(1, 64, 128, device=DEV).to(F8), torch.ones(1, 1, 1, device=DEV))
    assert y.shape == (0, 64)


def test_f8_products_special_values(at):
    """A NaN code and scales that are infinite or NaN reach their rows, columns and blocks alone."""
    m, k, n = 140, 256, 130
    gen = _gen(3)
    q, w = _normal(gen, m, k).to(F8), _normal(gen, 1, n, k).to(F8)
    q.view(torch.uint8)[5, 200] = 0x7F
    w.view(torch.uint8)[0, 129, 3] = 0xFF
    xs, ws = torch.ones(m, 2), torch.ones(1, 2, 2)
    xs[9, 1] = float("nan")
    xs[10, 0] = float("inf")
    y = _f64(at.allegro_grouped_matmul_fp8(q.to(DEV), xs.to(DEV), w.to(DEV), ws.to(DEV)))
    bad = np.zeros((m, n), bool)
    bad[[5, 9]] = True
    bad[:, 129] = True
    assert np.all(np.isnan(y[bad])) and not np.any(np.isfinite(y[10]))
    bad[10] = True
    assert np.all(np.isfinite(y[~bad]))


# --------------------------------------------------- streams, graphs, order

def _whole_update(at, s):
    """All operators as they follow each other in use."""
    offsets, rows = at.allegro_group_rows(s["t"], s["G"], offsets=s["offsets"], rows=s["rows"], workspace=s["ws0"])
    y, total, rstd = at.allegro_rms_norm_forward(s["h"], s["w"], s["d"], total=s["total"], out=s["y"], rstd=s["rstd"])
    a = at.allegro_grouped_matmul(y, s["B1"], offsets, rows, out=s["a"])
    u = at.allegro_grouped_matmul(a, s["B2"], offsets, rows, act=at.ALLEGRO_ACT_SILU, out=s["u"])
    da, dB2 = at.allegro_grouped_matmul_backward(a, s["B2"], s["du"], offsets, rows, act=at.ALLEGRO_ACT_SILU,
                                                 dx=s["da"], dw=s["dB2"], workspace=s["ws1"])
    dy, dB1 = at.allegro_grouped_matmul_backward(y, s["B1"], da, offsets, rows, dx=s["dy"], dw=s["dB1"],
                                                 workspace=s["ws2"])
    dh, dw = at.allegro_rms_norm_backward(total, s["w"], rstd, dy, s["ds"], dx=s["dh"], dw=s["dw"], workspace=s["ws3"])
    q, scale, _ = at.allegro_rms_norm_fp8(s["h"], s["w"], s["d"], total=s["total"], q=s["q"], scale=s["scale"])
    return [offsets, rows, y, total, rstd, a, u, dB2, dB1, dh, dw, q.view(torch.uint8), scale]


def _whole_state(at, m=9000, L=64, H=128, G=5, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV)  # noqa: E731
    empty = lambda *shape, dtype=F32: torch.empty(shape, device=DEV, dtype=dtype)  # noqa: E731
    scratch = lambda n: empty(max(n, 16), dtype=torch.uint8)  # noqa: E731
    return {"G": G, "t": torch.randint(-1, G, (m,), generator=gen, device=DEV, dtype=torch.int32), "h": normal(m, L),
            "d": normal(m, L), "w": 1 + 0.2 * normal(L), "B1": normal(G, L, H) / L ** 0.5,
            "B2": normal(G, H, L) / H ** 0.5, "du": normal(m, L), "ds": normal(m, L),
            "offsets": empty(G + 1, dtype=torch.int64), "rows": empty(m, dtype=torch.int32), "total": empty(m, L),
            "y": empty(m, L), "rstd": empty(m), "a": empty(m, H), "u": empty(m, L), "da": empty(m, H),
            "dB2": empty(G, H, L), "dy": empty(m, L), "dB1": empty(G, L, H), "dh": empty(m, L), "dw": empty(L),
            "q": empty(m, L, dtype=F8), "scale": empty(m, 1), "ws0": scratch(at.allegro_group_rows_workspace(m, G)),
            "ws1": scratch(at.allegro_grouped_matmul_workspace(m, H, L, G)),
            "ws2": scratch(at.allegro_grouped_matmul_workspace(m, L, H, G)),
            "ws3": scratch(at.allegro_rms_norm_workspace(m, L))}


def test_bit_identical_runs_and_another_stream(at):
    _note("[gpu] latent operators twice and on another stream")
    first = [v.clone() for v in _whole_update(at, _whole_state(at))]
    again = _whole_update(at, _whole_state(at))
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    side = torch.cuda.Stream()
    s = _whole_state(at)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = _whole_update(at, s)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, other))


def test_graph_replays(at):
    """The whole update captured, replayed on changing inputs among eager work."""
    _note("[gpu] latent operators in a captured graph")
    s = _whole_state(at)
    _whole_update(at, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _whole_update(at, s)
    for seed in (1, 2, 3, 4):
        new = _whole_state(at, seed=seed)
        for k in ("t", "h", "d", "w", "B1", "B2", "du", "ds"):
            s[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in outs]
        ref = _whole_update(at, new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), seed
