"""Which workspaces the binding keeps, with a library and tensors that only pretend (no GPU)."""
import contextlib
import gc
import types
import weakref

import pytest
import torch

from paper_2112_04291_b200 import binding


class Scratch:
    """What the binding asks of a uint8 CUDA tensor."""
    is_cuda, dtype = True, torch.uint8

    def __init__(self, size, device):
        self.size, self.device = size, torch.device(device)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return id(self) & ~255

    def numel(self):
        return self.size

    def get_device(self):
        return self.device.index


@pytest.fixture
def registered(monkeypatch):
    """The library's side: by device, the address that it was told last."""
    told, current = {}, [0]

    def set_workspace(ptr, size, stream):
        told[current[0]] = (ptr, size)
        return 0

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d).index
        yield
        current[0] = before
    monkeypatch.setattr(binding, "lib", lambda: types.SimpleNamespace(fastsgd_set_workspace=set_workspace))
    monkeypatch.setattr(binding, "_stream_handle", lambda stream=None: 0)
    monkeypatch.setattr(binding.torch, "empty", lambda size, dtype, device: Scratch(size, device))
    monkeypatch.setattr(binding.torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(binding.torch.cuda, "device", device)
    for name, value in (("_workspace_keepalive", None), ("_workspaces", {}), ("_allocated", {}), ("_outgrown", [])):
        monkeypatch.setattr(binding, name, value, raising=False)
    return told


def test_a_workspace_that_becomes_too_small_stays_for_graphs_captured_with_it(registered):
    first = weakref.ref(binding._ensure(10_000, "cuda"))
    second = weakref.ref(binding._ensure(50_000, "cuda"))
    gc.collect()
    assert first() is not None and second() is not None and registered[0] == (second().data_ptr(), 50_000)
    assert binding._ensure(20_000, "cuda") is second()
    binding.set_workspace(Scratch(4_096, "cuda:0"))                  # one of the caller's own in between
    gc.collect()
    assert second() is not None and registered[0][1] == 4_096
    assert binding._ensure(50_000, "cuda") is second() and registered[0] == (second().data_ptr(), 50_000)


def test_a_callers_own_that_is_too_small_stays_as_well(registered):
    binding.set_workspace(Scratch(4_096, "cuda:0"))
    own = weakref.ref(binding._workspace_keepalive)
    binding._ensure(10_000, "cuda")
    gc.collect()
    assert own() is not None and binding._workspace_keepalive.numel() == 10_000
    binding.set_workspace(own())
    binding._ensure(10_000, "cuda")
    assert len(binding._outgrown) == 1


def test_what_is_kept_stays_within_three_times_the_largest(registered):
    for need in range(10_000, 2_000_000, 999):
        assert binding._ensure(need, "cuda").numel() >= need
    kept = [w.numel() for w in binding._allocated[0]]
    assert sum(kept) <= 3 * kept[-1] and kept[-1] <= 3_000_000


def test_each_device_keeps_its_own(registered):
    a = binding._ensure(10_000, "cuda:0")
    b = binding._ensure(20_000, "cuda:1")
    assert b.device == torch.device("cuda", 1) and registered == {0: (a.data_ptr(), 10_000), 1: (b.data_ptr(), 20_000)}
    assert binding._ensure(10_000, "cuda:0") is a and binding._ensure(20_000, "cuda:1") is b and binding._ensure(10_000, "cuda") is a
