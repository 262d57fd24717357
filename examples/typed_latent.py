"""A residual latent track with weights per edge type: training in fp32 or bf16, inference in 8 bits.

Edges of a synthetic box have the type (species of the center, species of the neighbour).  Blocks of

    s = h + d,  y = rms_norm(s),  a = y B1[type],  d' = SiLU(a) B2[type],  h' = s

update a latent row per edge; a last norm and a readout vector give one number per edge.  Types change
only with the neighbour list, so rows are grouped once per list and every product takes that grouping.

    python examples/typed_latent.py --steps 50

trains on random targets with a hand-written backward pass, then runs the same weights with the first
product of each block in 8 bits and prints how far its output is from the training path's.
"""

from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2504_16068_amd as allegro  # noqa: E402
import workloads  # noqa: E402

SILU = allegro.ALLEGRO_ACT_SILU
BLOCK, F8_MAX = 128, 448.0


def edge_types(graph, n_species: int, device):
    """int32 [E]: center species * n_species + neighbour species, species drawn per atom."""
    centers = torch.repeat_interleave(torch.arange(graph.config.n_atoms), torch.from_numpy(graph.row_ptr).diff())
    species = torch.randint(n_species, (graph.config.n_atoms,), generator=torch.Generator().manual_seed(5))
    neighbours = torch.from_numpy(graph.nbr).long()
    return (species[centers] * n_species + species[neighbours]).to(torch.int32).to(device)


def quantised(b):
    """[G, K, N] weights as float8 [G, N, K] with a scale for each 128 x 128 block."""
    w = b.float().transpose(1, 2)
    g, n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    wide = torch.zeros(g, nb * BLOCK, kb * BLOCK, device=w.device)
    wide[:, :n, :k] = w
    tiles = wide.view(g, nb, BLOCK, kb, BLOCK)
    scale = (tiles.abs().amax((2, 4)) / F8_MAX).clamp_min(2.0 ** -126)
    q = (tiles / scale[:, :, None, :, None]).view(g, nb * BLOCK, kb * BLOCK)[:, :n, :k]
    return q.contiguous().to(torch.float8_e4m3fn), scale


@dataclass
class Block:
    norm: torch.Tensor  # fp32 [C]
    b1: torch.Tensor    # [G, C, H]
    b2: torch.Tensor    # [G, H, C]


class TypedLatent:
    """Weights of the track; rows and products in `dtype`, norm weights and readout in fp32."""

    def __init__(self, n_blocks, width, hidden, n_types, dtype, device, seed=3):
        gen = torch.Generator().manual_seed(seed)

        def draw(*shape, sd):
            return (torch.randn(shape, generator=gen) * sd).to(dtype).to(device)

        self.blocks = [Block(torch.ones(width, device=device), draw(n_types, width, hidden, sd=width ** -0.5),
                             draw(n_types, hidden, width, sd=hidden ** -0.5)) for _ in range(n_blocks)]
        self.norm = torch.ones(width, device=device)
        self.readout = (torch.randn(width, generator=gen) / width ** 0.5).to(device)

    def parameters(self):
        return [t for b in self.blocks for t in (b.norm, b.b1, b.b2)] + [self.norm, self.readout]

    def forward(self, h, offsets, rows):
        """(number per edge [E], what the backward needs)."""
        d, saved = None, []
        for b in self.blocks:
            y, h, rstd = allegro.allegro_rms_norm_forward(h, b.norm, residual=d)
            a = allegro.allegro_grouped_matmul(y, b.b1, offsets, rows)
            d = allegro.allegro_grouped_matmul(a, b.b2, offsets, rows, act=SILU)
            saved.append((y, h, rstd, a))
        y, h, rstd = allegro.allegro_rms_norm_forward(h, self.norm, residual=d)
        return y.float() @ self.readout, (saved, y, h, rstd)

    def backward(self, grad, state, offsets, rows):
        """Gradients of parameters(), in their order, and of the input rows, from that of the numbers per edge."""
        saved, y, h, rstd = state
        d_readout = grad @ y.float()
        dy = (grad[:, None] * self.readout).to(h.dtype)
        # the gradient of a block's output reaches its rows directly and through its update
        ds, d_norm = allegro.allegro_rms_norm_backward(h, self.norm, rstd, dy)
        out = [d_norm, d_readout]
        for b, (y, h, rstd, a) in zip(reversed(self.blocks), reversed(saved)):
            da, d_b2 = allegro.allegro_grouped_matmul_backward(a, b.b2, ds, offsets, rows, act=SILU)
            dy, d_b1 = allegro.allegro_grouped_matmul_backward(y, b.b1, da, offsets, rows)
            ds, d_norm = allegro.allegro_rms_norm_backward(h, b.norm, rstd, dy, dtotal=ds)
            out = [d_norm, d_b1, d_b2] + out
        return out, ds

    def inference_weights(self):
        """What infer() takes, laid out once: B1 in 8 bits, the rest in bf16."""
        return [quantised(b.b1) + (b.b2.to(torch.bfloat16),) for b in self.blocks]

    def infer(self, h, offsets, rows, weights):
        """The number per edge from bf16 rows; the first product of each block in 8 bits."""
        d = None
        for b, (q1, s1, b2) in zip(self.blocks, weights):
            q, scale, h = allegro.allegro_rms_norm_fp8(h, b.norm, residual=d)
            a = allegro.allegro_grouped_matmul_fp8(q, scale, q1, s1, offsets, rows)
            d = allegro.allegro_grouped_matmul(a, b2, offsets, rows, act=SILU)
        y, _, _ = allegro.allegro_rms_norm_forward(h, self.norm, residual=d)
        return y.float() @ self.readout


def run(workload="small", n_species=4, n_blocks=3, width=128, hidden=256, dtype=torch.float32, steps=50, lr=3e-3,
        device="cuda:0", log=print):
    """Trains, then infers in 8 bits: (losses, relative 2-norm of the 8-bit outputs' difference)."""
    graph = workloads.make_graph(workload)
    n_types = n_species ** 2
    offsets, rows = allegro.allegro_group_rows(edge_types(graph, n_species, device), n_types)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(graph.n_edges, width, generator=gen).to(dtype).to(device)
    target = torch.randn(graph.n_edges, generator=gen).to(device)
    model = TypedLatent(n_blocks, width, hidden, n_types, dtype, device)
    optimiser = torch.optim.Adam(model.parameters(), lr=lr)
    losses = []
    for step in range(steps):
        out, state = model.forward(x, offsets, rows)
        diff = out - target
        losses.append(float(diff.square().mean()))
        grads, _ = model.backward(diff * (2.0 / graph.n_edges), state, offsets, rows)
        for p, g in zip(model.parameters(), grads):
            p.grad = g
        optimiser.step()
        if step % 10 == 0 or step == steps - 1:
            log(f"step {step}: loss {losses[-1]:.5f}", flush=True)
    out, _ = model.forward(x, offsets, rows)
    low = model.infer(x.to(torch.bfloat16), offsets, rows, model.inference_weights())
    error = float((low - out).norm() / out.norm())
    log(f"{graph.n_edges} edges of {n_types} types; 8-bit inference differs by {error:.4f} of the outputs' 2-norm",
        flush=True)
    return losses, error


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--workload", default="small", choices=sorted(workloads.CONFIGS))
    parser.add_argument("--steps", type=int, default=50)
    parser.add_argument("--dtype", default="fp32", choices=("fp32", "bf16"))
    args = parser.parse_args()
    run(args.workload, steps=args.steps, dtype=torch.float32 if args.dtype == "fp32" else torch.bfloat16)
