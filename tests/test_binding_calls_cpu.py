"""How the bindings place their calls (no GPU): streams, allocations, devices.

The libraries' launches are replaced by a record of their arguments, and tensors of the CPU report a GPU.
"""

import contextlib
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")
latent = pytest.importorskip("paper_2504_16068_amd.latent",
                             reason="libraries not built (run __graft_entry__.build())")
from paper_2504_16068_amd import binding  # noqa: E402

SIDE, CURRENT = 0x51DE, 0xC0
_plain_empty = torch.empty


class _OnGpu(torch.Tensor):
    is_cuda = True
    device = torch.device("cuda", 0)

    def get_device(self):
        return 0


class _Lib:
    """A library with recorded launches; its host arithmetic is called."""

    def __init__(self, lib, rec):
        self.lib, self.rec = lib, rec

    def __getattr__(self, name):
        if name.endswith(("_workspace", "_buffers")) or "_plan_" in name:
            return getattr(self.lib, name)

        def launch(*args):
            self.rec.launches.append((name, args[-1]))
            self.rec.devices.append(self.rec.device)
            return 0
        return launch


@pytest.fixture
def calls(monkeypatch):
    """Records: launches (name, stream handle) and the devices current at them, allocations (bytes, stream or None)."""
    rec = SimpleNamespace(launches=[], devices=[], allocated=[], stream=None, device=0)

    def empty(shape, dtype, device=None):
        t = _plain_empty(shape, dtype=dtype)
        rec.allocated.append((t.numel() * t.element_size(), rec.stream))
        return t.as_subclass(_OnGpu)

    def empty_like(t):
        return empty(t.shape, t.dtype)

    @contextlib.contextmanager
    def stream(s):
        before, rec.stream = rec.stream, s
        yield
        rec.stream = before

    @contextlib.contextmanager
    def device(index):
        before, rec.device = rec.device, index
        yield
        rec.device = before

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", empty_like)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(binding, "_raw_stream", lambda index: CURRENT)
    for module in (binding, latent):
        monkeypatch.setattr(module, "_current_device", lambda: rec.device)
        monkeypatch.setattr(module, "_lib", _Lib(module.library(), rec))
    return rec


def _gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


def _latent_entries():
    """(name, call(**kw), allocated bytes) of every entry point, nothing passed in."""
    m, k, n, g, f8 = 5000, 40, 24, 3, torch.float8_e4m3fn
    x, dy, w = _gpu(m, k), _gpu(m, n), _gpu(g, k, n)
    off, norm_w, rstd = _gpu(g + 1, dtype=torch.int64), _gpu(k), _gpu(m)
    return [
        ("allegro_group_rows", lambda **kw: latent.allegro_group_rows(_gpu(m, dtype=torch.int32), g, **kw),
         8 * (g + 1) + 4 * m + latent.allegro_group_rows_workspace(m, g)),
        ("allegro_grouped_matmul", lambda **kw: latent.allegro_grouped_matmul(x, w, off, **kw), 4 * m * n),
        ("allegro_grouped_matmul_backward", lambda **kw: latent.allegro_grouped_matmul_backward(x, w, dy, off, **kw),
         4 * m * k + 4 * g * k * n + latent.allegro_grouped_matmul_workspace(m, k, n, g)),
        ("allegro_grouped_matmul_fp8", lambda **kw: latent.allegro_grouped_matmul_fp8(
            x.to(f8), _gpu(m, 1), _gpu(1, n, k).to(f8), _gpu(1, 1, 1), **kw), 2 * m * n),
        ("allegro_rms_norm_forward", lambda **kw: latent.allegro_rms_norm_forward(x, norm_w, x, **kw),
         2 * 4 * m * k + 4 * m),
        ("allegro_rms_norm_fp8", lambda **kw: latent.allegro_rms_norm_fp8(x, norm_w, x, **kw), m * k + 4 * m + 4 * m * k),
        ("allegro_rms_norm_backward", lambda **kw: latent.allegro_rms_norm_backward(x, norm_w, rstd, x, **kw),
         4 * m * k + 4 * k + latent.allegro_rms_norm_workspace(m, k)),
    ]


def _layer_entries():
    """The same of the tensor product and the layer."""
    plan = binding.allegro_tp_plan_create(2, 64)
    n, e, L, H = 3, 10, 64, 128
    row_ptr = _gpu(n + 1, dtype=torch.int64)
    x, env, path_w = _gpu(e, 64, plan.d1), _gpu(n, 64, plan.d2), _gpu(plan.n_paths, 64)
    w, Y, vec, h = _gpu(e, 64), _gpu(e, plan.d2), _gpu(e, 3, dtype=torch.float64), _gpu(e, L)
    weights = {k: _gpu(*s) for k, s in binding.layer_weight_shapes(plan, L, H).items()}
    saved, scratch = binding.allegro_layer_buffers(plan, L, H, n, e)
    size = lambda *ts: sum(t.numel() * t.element_size() for t in ts)  # noqa: E731
    args = (plan, row_ptr, x, env, path_w, x, w, Y)
    grads = size(x, env, w, Y)
    return [
        ("allegro_env_embed", lambda **kw: binding.allegro_env_embed(plan, row_ptr, w, Y, **kw), size(env)),
        ("allegro_tp_forward", lambda **kw: binding.allegro_tp_forward(plan, row_ptr, x, env, path_w, **kw), size(x)),
        ("allegro_tp_backward", lambda **kw: binding.allegro_tp_backward(*args, **kw), grads),
        ("allegro_tp_backward_train", lambda **kw: binding.allegro_tp_backward_train(*args, **kw),
         grads + size(path_w) + max(16, binding.allegro_tp_backward_workspace(plan, n))),
        ("allegro_tp_backward_train_noalloc", lambda **kw: binding.allegro_tp_backward_train_noalloc(*args, **kw),
         grads + size(path_w)),
        ("allegro_sh_forward", lambda **kw: binding.allegro_sh_forward(plan, vec, **kw), size(Y)),
        ("allegro_sh_backward", lambda **kw: binding.allegro_sh_backward(plan, vec, Y, **kw), size(vec)),
        ("allegro_layer_forward", lambda **kw: binding.allegro_layer_forward(plan, L, H, row_ptr, h, x, Y, weights, **kw),
         size(h, x) + max(16, saved)),
        ("allegro_layer_backward", lambda **kw: binding.allegro_layer_backward(
            plan, L, H, row_ptr, h, x, Y, weights, _gpu(saved, dtype=torch.uint8), h, x, **kw),
         size(h, x, Y, *weights.values()) + max(16, scratch)),
    ]


ENTRIES = [(_latent_entries, i) for i in range(7)] + [(_layer_entries, i) for i in range(9)]


def test_every_entry_point_is_covered():
    names = {n for n in latent.EXPORTED + binding.EXPORTED
             if not n.endswith(("_workspace", "_buffers", "_last_error")) and "_plan_" not in n}
    assert {e[0] for e in _latent_entries() + _layer_entries()} == names


@pytest.mark.parametrize("entries,i", ENTRIES)
def test_what_a_call_allocates_belongs_to_its_stream(calls, entries, i):
    """Memory is reused in the order of the stream that it was allocated on: results and workspaces of a call on
    another stream than the current one are allocated on that stream, or the current stream's next tensor could
    take a workspace that the call still uses."""
    name, call, allocated = entries()[i]
    side = SimpleNamespace(cuda_stream=SIDE, device=torch.device("cuda", 0))
    call(stream=side)
    assert calls.launches == [(name, SIDE)]
    assert sum(n for n, _ in calls.allocated) == allocated
    assert all(s is side for _, s in calls.allocated)
    calls.launches.clear()
    calls.allocated.clear()
    call()
    assert calls.launches == [(name, CURRENT)]
    assert all(s is None for _, s in calls.allocated)


@pytest.mark.parametrize("entries,i", ENTRIES)
def test_calls_run_on_their_tensors_device(calls, entries, i):
    """The tensors' device is made current for the launch, and a stream of another device is refused."""
    name, call, _ = entries()[i]
    calls.device = 1
    call()
    assert calls.launches == [(name, CURRENT)] and calls.devices == [0] and calls.device == 1
    other = SimpleNamespace(cuda_stream=SIDE, device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="stream is one of cuda:1"):
        call(stream=other)
    assert len(calls.launches) == 1
