"""How the binding of the latent operators places its calls (no GPU): streams, allocations, devices.

The library's launches are replaced by a record of their arguments, and tensors of the CPU report a GPU.
"""

import contextlib
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")
latent = pytest.importorskip("paper_2504_16068_amd.latent",
                             reason="libraries not built (run __graft_entry__.build())")

SIDE, CURRENT = 0x51DE, 0xC0


class _OnGpu(torch.Tensor):
    def get_device(self):
        return 0


class _Lib:
    """The library with recorded launches; its host arithmetic is called."""

    def __init__(self, lib, launches, devices, device):
        self.lib, self.launches, self.devices, self.device = lib, launches, devices, device

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return getattr(self.lib, name)

        def launch(*args):
            self.launches.append((name, args[-1]))
            self.devices.append(self.device())
            return 0
        return launch


@pytest.fixture
def calls(monkeypatch):
    """Records: launches (name, stream handle) and the devices current at them, allocations (bytes, stream or None)."""
    rec = SimpleNamespace(launches=[], devices=[], allocated=[], stream=None, device=0)

    def empty(shape, dtype, device=None):
        t = torch.empty(shape, dtype=dtype)
        rec.allocated.append((t.numel() * t.element_size(), rec.stream))
        return t.as_subclass(_OnGpu)

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

    cuda = SimpleNamespace(stream=stream, device=device, current_device=lambda: rec.device)
    monkeypatch.setattr(latent, "torch", SimpleNamespace(empty=empty, cuda=cuda, Tensor=torch.Tensor, uint8=torch.uint8,
                                                         device=lambda *a: a))
    monkeypatch.setattr(latent, "_raw_stream", lambda index: CURRENT)
    monkeypatch.setattr(latent, "_current_device", lambda: rec.device, raising=False)
    monkeypatch.setattr(latent, "_lib", _Lib(latent.library(), rec.launches, rec.devices, lambda: rec.device))
    return rec


def _gpu(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


def _entries():
    """(name, call(**kw), allocated bytes of outputs, of workspace) of every entry point, nothing passed in."""
    m, k, n, g, f8 = 5000, 40, 24, 3, torch.float8_e4m3fn
    x, dy, w = _gpu(m, k), _gpu(m, n), _gpu(g, k, n)
    off, norm_w, rstd = _gpu(g + 1, dtype=torch.int64), _gpu(k), _gpu(m)
    return [
        ("allegro_group_rows", lambda **kw: latent.allegro_group_rows(_gpu(m, dtype=torch.int32), g, **kw),
         8 * (g + 1) + 4 * m, latent.allegro_group_rows_workspace(m, g)),
        ("allegro_grouped_matmul", lambda **kw: latent.allegro_grouped_matmul(x, w, off, **kw), 4 * m * n, 0),
        ("allegro_grouped_matmul_backward", lambda **kw: latent.allegro_grouped_matmul_backward(x, w, dy, off, **kw),
         4 * m * k + 4 * g * k * n, latent.allegro_grouped_matmul_workspace(m, k, n, g)),
        ("allegro_grouped_matmul_fp8", lambda **kw: latent.allegro_grouped_matmul_fp8(
            x.to(f8), _gpu(m, 1), _gpu(1, n, k).to(f8), _gpu(1, 1, 1), **kw), 2 * m * n, 0),
        ("allegro_rms_norm_forward", lambda **kw: latent.allegro_rms_norm_forward(x, norm_w, x, **kw),
         2 * 4 * m * k + 4 * m, 0),
        ("allegro_rms_norm_fp8", lambda **kw: latent.allegro_rms_norm_fp8(x, norm_w, x, **kw), m * k + 4 * m + 4 * m * k, 0),
        ("allegro_rms_norm_backward", lambda **kw: latent.allegro_rms_norm_backward(x, norm_w, rstd, x, **kw),
         4 * m * k + 4 * k, latent.allegro_rms_norm_workspace(m, k)),
    ]


def test_every_entry_point_is_covered():
    names = {n for n in latent.EXPORTED if not n.endswith(("_workspace", "_last_error"))}
    assert {e[0] for e in _entries()} == names


@pytest.mark.parametrize("i", range(7))
def test_what_a_call_allocates_belongs_to_its_stream(calls, i):
    """Memory is reused in the order of the stream that it was allocated on: results and workspaces of a call on
    another stream than the current one are allocated on that stream, or the current stream's next tensor could
    take a workspace that the call still uses."""
    name, call, outputs, workspace = _entries()[i]
    side = SimpleNamespace(cuda_stream=SIDE, device=torch.device("cuda", 0))
    call(stream=side)
    assert calls.launches == [(name, SIDE)]
    assert sum(n for n, _ in calls.allocated) == outputs + workspace
    assert all(s is side for _, s in calls.allocated)
    calls.launches.clear()
    calls.allocated.clear()
    call()
    assert calls.launches == [(name, CURRENT)]
    assert all(s is None for _, s in calls.allocated)


@pytest.mark.parametrize("i", range(7))
def test_calls_run_on_their_tensors_device(calls, i):
    """The tensors' device is made current for the launch, and a stream of another device is refused."""
    name, call, _, _ = _entries()[i]
    calls.device = 1
    call()
    assert calls.launches == [(name, CURRENT)] and calls.devices == [0] and calls.device == 1
    other = SimpleNamespace(cuda_stream=SIDE, device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="stream is one of cuda:1"):
        call(stream=other)
    assert len(calls.launches) == 1
