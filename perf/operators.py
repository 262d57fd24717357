"""The operators of the latent track whose speed matters to a user of this library, in their plain form.

Four operators, each through the public entry points of paper_2504_16068_amd where `own` is true, and in
elementary torch operations where it is not:

  group     the rows (edges or atoms) of each type: a stable counting sort of the types into offsets and a row list
  product   one matrix product per type over ragged groups of rows, Y[r] = act(X[r]) W[type(r)], forward alone or
            with both gradients
  norm      the residual's addition and the root-mean-square norm of the sum: forward, forward and backward, or
            with the output in 8 bits and a scale for each row and 128 columns
  fp8       the product per type of 8-bit floating-point operands with a scale for each row and 128 columns of X
            and each 128 x 128 block of W

Rows are edges (or atoms) of structures, their types pairs of species (or species) with the uneven shares that
species have; one type is usually absent, and some rows may have no type (padding).  Latents are N(0, 1),
weights N(0, 1 / sqrt(fan-in)).  Sizes: the edge counts and the latent widths of the layer (64, 128, 192) and
of wider latents.
"""

from __future__ import annotations

from math import exp, log, sqrt

import torch

own = False

BLOCK = 128          # columns (or rows and columns of W) that share a scale
FP8_MAX = 448.0      # largest value of 8 bits with 4 exponent and 3 mantissa bits
FP8_MIN_SCALE = 2.0 ** -126
EPS = 1e-6


def _case(op, M, **opt):
    c = {"op": op, "M": M, "G": 1, "K": 0, "N": 0, "dtype": "float32", "act": "none", "train": False, "residual": True,
         "fp8": False, "pad": 0, "untyped": 0.0}
    c.update(opt)
    return c


def listed():
    def case(name, op, M, **opt):
        return {"name": name, **_case(op, M, **opt)}

    return [
        # the edges of one molecule of two species: nothing but latency
        case("group_small", "group", 1142, G=4),
        # the edges of a large box, pairs of 15 species, 3% of the rows padding
        case("group_large", "group", 1048820, G=225, untyped=0.03),
        # one small structure in inference: the latent's second product
        case("product_small", "product", 3700, G=16, K=128, N=64, act="silu"),
        # energies of a large box: [h, s] B1 of the wide latent with weights per species pair
        case("product_forward", "product", 1048820, G=16, K=192, N=128),
        # training on half of that box: the second product with its SiLU, and both gradients
        case("product_train", "product", 523599, G=16, K=128, N=64, act="silu", train=True),
        # a wide latent in bfloat16, pairs of ten species, an odd number of rows
        case("product_wide", "product", 100003, G=100, K=1024, N=512, dtype="bfloat16", act="silu", train=True),
        # single centers in inference
        case("norm_single", "norm", 64, K=128),
        # training: the latent of every edge of a large box
        case("norm_train", "norm", 1048820, K=128, train=True),
        # wide latents of atoms in bfloat16, odd in both sizes
        case("norm_odd", "norm", 20001, K=1031, dtype="bfloat16", train=True),
        # inference with 8-bit products: the norm writes their operand
        case("norm_fp8", "norm", 523599, K=256, dtype="bfloat16", fp8=True),
        # one molecule through a wide 8-bit product
        case("fp8_small", "fp8", 1142, G=4, K=256, N=512, dtype="bfloat16"),
        # a large box through a wide 8-bit product with weights per species pair
        case("fp8_large", "fp8", 262144, G=16, K=1024, N=1024, dtype="bfloat16"),
    ]


# the largest listed cases: values moved and operations of a pass
MOST_VALUES = {"product": 1048820 * 320, "norm": 1048820 * 128, "fp8": 262144 * 2048}
MOST_FLOPS = {"product": 2.0 * 100003 * 1024 * 512, "fp8": 2.0 * 262144 * 1024 * 1024}


def draw(rng):
    def between(lo, hi):
        return round(exp(rng.uniform(log(lo), log(hi))))

    op = rng.choice(["group", "product", "product", "product", "norm", "norm", "norm", "fp8", "fp8"])
    if op == "group":
        return _case(op, between(200, 1000000), G=between(1, 256), untyped=rng.choice([0.0, 0.03]))

    def width(lo, hi):  # half of them whole vectors, the others as they fall
        w = between(lo, hi)
        return w if rng.random() < 0.5 else max(16, w // 16 * 16)

    dtype = rng.choice(["float32", "bfloat16"])
    pad = rng.choice([0, 0, 0, 8, 3])
    if op == "norm":
        K = width(16, 4096)
        train = rng.random() < 0.6
        M = max(1, min(between(1, 1000000), MOST_VALUES[op] // K))
        return _case(op, M, K=K, dtype=dtype, pad=pad, train=train, residual=rng.random() < 0.75,
                     fp8=not train and rng.random() < 0.6)
    if op == "product":
        K, N = width(24, 1024), width(24, 1024)
        G = between(1, 128)
        M = between(1, 1000000)
        M = max(1, min(M, MOST_VALUES[op] // (K + N), int(MOST_FLOPS[op] / (2.0 * K * N))))
        return _case(op, M, G=G, K=K, N=N, dtype=dtype, pad=pad, act=rng.choice(["none", "silu"]),
                     train=rng.random() < 0.6, untyped=rng.choice([0.0, 0.0, 0.03]))
    # 8-bit operands, results in bfloat16
    K, N, G = width(64, 2048), width(64, 2048), between(1, 64)
    M = max(1, min(between(1, 262144), MOST_VALUES[op] // (K + N), int(MOST_FLOPS[op] / (2.0 * K * N))))
    return _case(op, M, G=G, K=K, N=N, dtype="bfloat16", pad=16 if pad == 8 else pad, untyped=rng.choice([0.0, 0.0, 0.03]))


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return {"float32": torch.float32, "bfloat16": torch.bfloat16}[case["dtype"]]


def _types(case, gen, dev):
    """Types with the uneven shares of species; of more than two the last is absent."""
    M, G = case["M"], case["G"]
    share = torch.arange(1, G + 1, device=dev, dtype=torch.float32) ** -1.2
    if G > 2:
        share[G - 1] = 0
    edges = torch.cumsum(share / share.sum(), 0)[: G - 1]
    u = torch.rand(M, generator=gen, device=dev)
    t = torch.bucketize(u, edges).to(torch.int32).clamp_(max=max(0, G - 2) if G > 2 else G - 1)
    if case["untyped"]:
        t[torch.rand(M, generator=gen, device=dev) < case["untyped"]] = -1
    return t


def prepare(case, seed):
    """Latents, weights, types, the grouping that a program keeps with its neighbour list, and its buffers."""
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 1000003 + 29)
    M, G, K, N, dt = case["M"], case["G"], case["K"], case["N"], _dtype(case)
    f8 = torch.float8_e4m3fn

    def normal(*shape, scale=1.0, dtype=dt):
        t = torch.randn(shape, generator=gen, device=dev)
        return (t if scale == 1.0 else t.mul_(scale)).to(dtype)

    def rows_of(width, dtype=dt):  # a tensor of rows, or the first columns of a wider one
        return normal(M, width + case["pad"], dtype=dtype)[:, :width]

    s = {"case": case}
    if case["op"] == "norm":
        s["x"], s["w"] = rows_of(K), normal(K, scale=0.2, dtype=torch.float32) + 1.0
        s["residual"] = normal(M, K) if case["residual"] else None
        s["total"] = torch.empty(M, K, device=dev, dtype=dt) if case["residual"] else None
        if case["fp8"]:
            s["q"] = torch.empty(M, K, device=dev, dtype=f8)
            s["scale"] = torch.empty(M, -(-K // BLOCK), device=dev)
        else:
            s["y"], s["rstd"] = torch.empty(M, K, device=dev, dtype=dt), torch.empty(M, device=dev)
        if case["train"]:
            s["dy"], s["dtotal"] = normal(M, K), normal(M, K) if case["residual"] else None
            s["dx"], s["dw"] = torch.empty(M, K, device=dev, dtype=dt), torch.empty(K, device=dev)
        return s
    t = s["types"] = _types(case, gen, dev)
    key = torch.where(t < 0, G, t.long())
    if case["op"] == "group":
        s["offsets"] = torch.empty(G + 1, device=dev, dtype=torch.int64)
        s["rows"] = torch.empty(M, device=dev, dtype=torch.int32)
        return s
    s["rows"] = torch.argsort(key, stable=True).to(torch.int32)
    counts = torch.bincount(key, minlength=G + 1)
    s["offsets"] = torch.zeros(G + 1, device=dev, dtype=torch.int64)
    s["offsets"][1:] = torch.cumsum(counts[:G], 0)
    s["sizes"] = counts[:G].tolist()  # host copy, for a program that calls one product per group
    s["y"] = torch.empty(M, N, device=dev, dtype=dt)
    if case["op"] == "product":
        s["x"], s["w"] = rows_of(K), normal(G, K, N, scale=1 / sqrt(K))
        if case["train"]:
            s["dy"] = normal(M, N)
            s["dx"], s["dw"] = torch.empty(M, K, device=dev, dtype=dt), torch.empty_like(s["w"])
        return s
    # 8-bit operands as the norm and a quantised checkpoint hand them over
    kb, nb = -(-K // BLOCK), -(-N // BLOCK)
    x = torch.randn(M, K + case["pad"], generator=gen, device=dev)
    s["xs"] = _blocks_amax(x[:, :K], kb) / FP8_MAX
    s["x"] = torch.zeros(M, K + case["pad"], device=dev, dtype=f8)
    s["x"][:, :K].copy_((x[:, :K] / _spread(s["xs"], K)).to(f8))
    s["x"] = s["x"][:, :K]
    w = torch.randn(G, N, K, generator=gen, device=dev).mul_(1 / sqrt(K))
    s["ws"] = torch.nn.functional.pad(_blocks_amax(w, kb), (0, 0, 0, nb * BLOCK - N)).view(G, nb, BLOCK, kb).amax(2)
    s["ws"] = s["ws"] / FP8_MAX
    s["w"] = (w / _spread(s["ws"].repeat_interleave(BLOCK, 1)[:, :N], K)).to(f8)
    return s


def _blocks_amax(x, blocks):
    """Largest magnitude of each BLOCK columns: [..., C] to [..., blocks]."""
    C = x.shape[-1]
    a = torch.nn.functional.pad(x.abs(), (0, blocks * BLOCK - C))
    return a.view(*x.shape[:-1], blocks, BLOCK).amax(-1)


def _spread(scale, C):
    """Each block's scale over its columns: [..., blocks] to [..., C]."""
    return scale.repeat_interleave(BLOCK, -1)[..., :C]


# -------------------------------------------------------------------- runs

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2504_16068_amd as at

    case = s["case"]
    if case["op"] == "group":
        offsets, rows = at.allegro_group_rows(s["types"], case["G"], offsets=s["offsets"], rows=s["rows"])
        return {"offsets": offsets, "rows": rows}
    if case["op"] == "product":
        act = at.ALLEGRO_ACT_SILU if case["act"] == "silu" else at.ALLEGRO_ACT_NONE
        y = at.allegro_grouped_matmul(s["x"], s["w"], s["offsets"], s["rows"], act=act, out=s["y"])
        if not case["train"]:
            return {"y": y}
        dx, dw = at.allegro_grouped_matmul_backward(s["x"], s["w"], s["dy"], s["offsets"], s["rows"], act=act,
                                                    dx=s["dx"], dw=s["dw"])
        return {"y": y, "dx": dx, "dw": dw}
    if case["op"] == "fp8":
        return {"y": at.allegro_grouped_matmul_fp8(s["x"], s["xs"], s["w"], s["ws"], s["offsets"], s["rows"],
                                                   out=s["y"])}
    if case["fp8"]:
        q, scale, total = at.allegro_rms_norm_fp8(s["x"], s["w"], residual=s["residual"], eps=EPS, total=s["total"],
                                                  q=s["q"], scale=s["scale"])
        return {"q": q, "scale": scale, "total": total}
    y, total, rstd = at.allegro_rms_norm_forward(s["x"], s["w"], residual=s["residual"], eps=EPS, total=s["total"],
                                                 out=s["y"], rstd=s["rstd"])
    if not case["train"]:
        return {"y": y, "total": total, "rstd": rstd}
    dx, dw = at.allegro_rms_norm_backward(total, s["w"], rstd, s["dy"], dtotal=s["dtotal"], dx=s["dx"], dw=s["dw"])
    return {"y": y, "total": total, "rstd": rstd, "dx": dx, "dw": dw}


def _silu(a):
    return a / (1.0 + torch.exp(-a))


def _silu_grad(a):
    sg = 1.0 / (1.0 + torch.exp(-a))
    return sg * (1.0 + a * (1.0 - sg))


def _run_plain(s):
    case = s["case"]
    if case["op"] == "group":
        G, t = case["G"], s["types"].long()
        key = torch.where((t >= 0) & (t < G), t, G)
        counts = torch.zeros(G + 1, device=t.device, dtype=torch.int64).index_add_(0, key, torch.ones_like(key))
        offsets = torch.zeros(G + 1, device=t.device, dtype=torch.int64)
        offsets[1:] = torch.cumsum(counts[:G], 0)
        return {"offsets": offsets, "rows": torch.argsort(key, stable=True).to(torch.int32)}
    dt = _dtype(case)
    if case["op"] == "norm":
        total = s["x"].float()
        if s["residual"] is not None:
            total = total + s["residual"].float()
        rstd = 1.0 / torch.sqrt((total * total).mean(1) + EPS)
        y = total * rstd[:, None] * s["w"]
        stored = total.to(dt)
        if case["fp8"]:
            kb = -(-case["K"] // BLOCK)
            scale = (_blocks_amax(y, kb) / FP8_MAX).clamp_(min=FP8_MIN_SCALE)
            return {"q": (y * _spread(1.0 / scale, case["K"])).to(torch.float8_e4m3fn), "scale": scale, "total": stored}
        out = {"y": y.to(dt), "total": stored, "rstd": rstd}
        if case["train"]:
            unit, dy = stored.float() * rstd[:, None], s["dy"].float()
            t = dy * s["w"]
            dx = rstd[:, None] * (t - unit * (t * unit).mean(1, keepdim=True))
            if s["dtotal"] is not None:
                dx = dx + s["dtotal"].float()
            out.update(dx=dx.to(dt), dw=(dy * unit).sum(0))
        return out
    # rows by group, one product per group that has any, and back to their places
    order = s["rows"].long()
    first = sum(s["sizes"])
    if case["op"] == "fp8":
        x = s["x"].float() * _spread(s["xs"], case["K"])
        w = s["w"].float() * _spread(s["ws"].repeat_interleave(BLOCK, 1)[:, : case["N"]], case["K"])
        w = w.transpose(1, 2)
        act = x
    else:
        x, w = s["x"].float(), s["w"].float()
        act = _silu(x) if case["act"] == "silu" else x
    sizes = [n for n in s["sizes"]] + [case["M"] - first]
    parts = act[order].split(sizes)
    out = [p @ w[g] for g, p in enumerate(parts[:-1])] + [x.new_zeros(sizes[-1], case["N"])]
    y = torch.empty(case["M"], case["N"], device=x.device, dtype=dt)
    y[order] = torch.cat(out).to(dt)
    if not case["train"]:
        return {"y": y}
    gparts = s["dy"].float()[order].split(sizes)
    back = [p @ w[g].t() for g, p in enumerate(gparts[:-1])] + [x.new_zeros(sizes[-1], case["K"])]
    dx = torch.empty_like(x)
    dx[order] = torch.cat(back)
    if case["act"] == "silu":
        dx = dx * _silu_grad(x)
    dw = torch.stack([a.t() @ b for a, b in zip(parts[:-1], gparts[:-1])])
    return {"y": y, "dx": dx.to(dt), "dw": dw.to(dt)}


def work(case):
    """Bytes: every input and output of a pass once.  Operations: the products, or a few per value."""
    M, G, K, N = case["M"], case["G"], case["K"], case["N"]
    b = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "group":
        return {"bytes": 8 * M + 8 * (G + 1), "flops": M}
    if case["op"] == "norm":
        kb = -(-K // BLOCK)
        r = 1 if case["residual"] else 0
        nbytes = M * K * b * (1 + 2 * r) + 4 * K + (M * (K + 4 * kb) if case["fp8"] else M * K * b + 4 * M)
        if case["train"]:
            nbytes += M * K * b * (3 + r) + 4 * M + 8 * K
        return {"bytes": nbytes, "flops": M * K * (14 if case["train"] else 5)}
    flops, index = 2 * M * K * N, 4 * M + 8 * (G + 1)
    if case["op"] == "fp8":
        kb, nb = -(-K // BLOCK), -(-N // BLOCK)
        return {"bytes": M * (K + 4 * kb) + G * (N * K + 4 * nb * kb) + M * N * b + index, "flops": flops}
    forward, weights = M * (K + N) * b + index, G * K * N * b
    if not case["train"]:
        return {"bytes": forward + weights, "flops": flops}
    # the backward reads X and dY and the weights once more and writes dX and dW
    return {"bytes": forward + weights + M * (2 * K + N) * b + index + 2 * weights, "flops": 3 * flops}


# ------------------------------------------------- the same values in 64 bits

def exact(case, seed):
    if case["op"] == "group":
        return None  # whole numbers
    s = prepare(case, seed)
    d = torch.float64
    M, G, K, N = case["M"], case["G"], case["K"], case["N"]
    if case["op"] == "norm":
        v = s["x"].to(d) + (s["residual"].to(d) if case["residual"] else 0)
        inv = (v.pow(2).sum(1, keepdim=True) / K + EPS).rsqrt()
        y = v * inv * s["w"].to(d)
        if case["fp8"]:
            q, scale = torch.empty_like(y), torch.empty(M, -(-K // BLOCK), device=y.device, dtype=d)
            for j, c in enumerate(range(0, K, BLOCK)):
                piece = y[:, c:c + BLOCK]
                scale[:, j] = piece.abs().max(1).values.div(FP8_MAX).clamp(min=FP8_MIN_SCALE)
                q[:, c:c + BLOCK] = piece / scale[:, j:j + 1]
            return {"q": q, "scale": scale, "total": v}
        out = {"y": y, "total": v, "rstd": inv[:, 0]}
        if case["train"]:
            # the gradient of <dy, y> + <dtotal, total> at the total that is kept
            v, g = v.to(_dtype(case)).to(d), s["dy"].to(d) * s["w"].to(d)
            along = (g * v).sum(1, keepdim=True) * inv.pow(3) / K
            dx = g * inv - v * along
            out["dx"] = dx + s["dtotal"].to(d) if case["residual"] else dx
            out["dw"] = (s["dy"].to(d) * v).mul(inv).sum(0)
        return out
    dev, t = s["types"].device, s["types"]
    y = torch.zeros(M, N, device=dev, dtype=d)
    if case["op"] == "fp8":
        col = torch.arange(K, device=dev) // BLOCK
        row = torch.arange(N, device=dev) // BLOCK
        for g in range(G):
            at = (t == g).nonzero()[:, 0]
            w = s["w"][g].to(d) * s["ws"][g].to(d)[row][:, col]
            y[at] = (s["x"].view(torch.uint8)[at].view(torch.float8_e4m3fn).to(d) * s["xs"][at].to(d)[:, col]) @ w.T
        return {"y": y}
    dx = torch.zeros(M, K, device=dev, dtype=d)
    dw = torch.zeros(G, K, N, device=dev, dtype=d)
    for g in range(G):
        at = (t == g).nonzero()[:, 0]
        a, w = s["x"][at].to(d), s["w"][g].to(d)
        sig = torch.sigmoid(a)
        z = a * sig if case["act"] == "silu" else a
        y[at] = z @ w
        if case["train"]:
            e = s["dy"][at].to(d)
            dw[g] = z.T @ e
            up = e @ w.T
            dx[at] = up * (sig + z * (1 - sig)) if case["act"] == "silu" else up
    return {"y": y, "dx": dx, "dw": dw} if case["train"] else {"y": y}
