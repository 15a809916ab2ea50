"""Memory that a call allocates for itself comes from the pool of the stream that the call runs on (no GPU: allocations and launches are watched)."""
import contextlib

import numpy as np
import pytest
import torch


class Device(torch.Tensor):
    """A tensor on the host that says it is on a GPU."""

    is_cuda = property(lambda self: True)


def _on_gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Device)


@pytest.fixture
def watched(monkeypatch):
    """(the package's binding, what happened: ("alloc", the current stream at that time), ("launch", the call's stream))."""
    from paper_2605_08696_amd import binding, build
    if build.is_stale():
        build.build_lib()
    binding.lib()
    log, current = [], [None]

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before

    empty = torch.empty

    def alloc(*args, **kw):
        log.append(("alloc", current[0]))
        return empty(*args, **kw).as_subclass(Device)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", alloc)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: None)
    monkeypatch.setattr(binding, "_check", lambda rc: None)
    monkeypatch.setattr(binding, "_launch", lambda fn, args, first, others, stream: log.append(("launch", stream)))
    return binding, log


@pytest.mark.parametrize("stream", [None, "another"])
def test_the_scans_workspace(watched, stream):
    binding, log = watched
    H, P, N, T = 2, 64, 64, 2000
    xbc, dt, out = _on_gpu(T, H * P + 2 * N, dtype=torch.bfloat16), _on_gpu(T, H), _on_gpu(T, H * P, dtype=torch.bfloat16)
    off = np.array([0, T], dtype=np.int32)
    assert binding.selective_scan_workspace_bytes(binding.SRM_BF16, off, H, P, N) > 0
    binding.selective_scan(xbc, dt, _on_gpu(H), off, torch.tensor([0, T], dtype=torch.int32), out, stream=stream)
    assert log == [("alloc", stream), ("launch", stream)]


@pytest.mark.parametrize("stream", [None, "another"])
def test_a_mixer_blocks_slabs(watched, monkeypatch, stream):
    binding, log = watched

    class Library:
        def srm_mixer_block(self, *args):
            log.append(("launch", args[-1]))
            return 0

    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(binding, "_stream", lambda s: s)
    monkeypatch.setattr(binding.Model, "act_dtype", torch.bfloat16)
    monkeypatch.setattr(binding.Model, "state_torch_dtype", torch.float32)
    model = binding.Model.__new__(binding.Model)
    model._h, model.d, model.sd = None, 256, 256
    model.mixer_block(0, 3, 2, _on_gpu(2, 256), _on_gpu(2, 256), _on_gpu(2, 256, dtype=torch.bfloat16), stream=stream)
    assert log == [("alloc", stream), ("launch", stream)]
