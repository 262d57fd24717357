"""The typed latent example on the GPU: gradients against a plain fp64 model, training, 8-bit inference.

Bounds: fp32 products are within 64 units of 2^-24 of their terms' magnitudes (see test_gpu_latent.py) and the
norms within 20; three blocks of two products and a norm, forward and backward, are 18 of them: 18 * 64 * 2^-24 =
7e-5 of a gradient's 2-norm, asked for is 1e-4.  In 8 bits each operand of the first products is off by at most
2^-4 of its values, so a by at most 2^-3 of its terms, in a fixed part of independent errors: 2^-3 of the outputs.
"""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

DEV = "cuda:0"


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a ROCm GPU"
    import typed_latent
    return typed_latent


def _plain(params, n_blocks, x, types, n_types):
    """The example's formula, in the parameters' type on the CPU."""
    def norm(s, w):
        return s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-6) * w

    def product(a, b):
        out = torch.zeros(a.shape[0], b.shape[2], dtype=a.dtype)
        for g in range(n_types):
            at = torch.nonzero(types == g)[:, 0]
            out = out.index_add(0, at, a[at] @ b[g])
        return out

    s = x
    for i in range(n_blocks):
        w, b1, b2 = params[3 * i:3 * i + 3]
        s = s + product(torch.nn.functional.silu(product(norm(s, w), b1)), b2)
    return norm(s, params[-2]) @ params[-1]


@pytest.mark.parametrize("m,width,hidden,n_types", [(700, 64, 128, 4), (333, 40, 72, 16), (1, 8, 8, 2)])
def test_gradients(example, m, width, hidden, n_types):
    print(f"[gpu] typed latent gradients M={m} C={width} H={hidden} G={n_types}", flush=True)
    gen = torch.Generator().manual_seed(m)
    types = torch.randint(-1, n_types, (m,), generator=gen, dtype=torch.int32)
    x, grad = torch.randn(m, width, generator=gen), torch.randn(m, generator=gen)
    model = example.TypedLatent(3, width, hidden, n_types, torch.float32, DEV)
    offsets, rows = example.allegro.allegro_group_rows(types.to(DEV), n_types)
    out, state = model.forward(x.to(DEV), offsets, rows)
    grads, dx = model.backward(grad.to(DEV), state, offsets, rows)
    params = [p.cpu().double().requires_grad_() for p in model.parameters()]
    x64 = x.double().requires_grad_()
    ref = _plain(params, 3, x64, types, n_types)
    ref.backward(grad.double())
    for name, got, want in [("out", out, ref.detach()), ("dx", dx, x64.grad)] + [
            (f"parameter {i}", g, p.grad) for i, (g, p) in enumerate(zip(grads, params))]:
        got = got.cpu().double()
        assert got.shape == want.shape and float((got - want).norm()) <= 1e-4 * float(want.norm()), name


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_trains_and_infers(example, dtype):
    print(f"[gpu] typed latent example {dtype}", flush=True)
    losses, error = example.run("tiny", n_species=2, steps=20, dtype=getattr(torch, dtype))
    assert losses[-1] < 0.9 * losses[0]
    assert error <= 2.0 ** -3
