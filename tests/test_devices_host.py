"""Calls without a handle run on their tensors' device, whichever is current.  (No device is
touched: the library's functions and torch's device calls are stand-ins here.)"""

import contextlib
import ctypes
import types

import pytest
import torch


class OnDevice1(torch.Tensor):
    """A host tensor that says it is on cuda:1."""
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", 1))

    def get_device(self):
        return 1

    def new_empty(self, shape, dtype=None):
        return there(torch.empty(shape, dtype=dtype or self.dtype))


def there(t):
    return t.as_subclass(OnDevice1)


@pytest.fixture
def b(monkeypatch):
    """The binding, with a library that notes which device was current at each call."""
    from paper_2009_04509_amd import binding
    now, seen = [0], []

    @contextlib.contextmanager
    def device(index):
        before, now[0] = now[0], index
        yield
        now[0] = before

    def call(name):
        return lambda *a: seen.append((name, now[0], a[-1])) or 0

    for name in ("pointid_checkpoint_save", "pointid_checkpoint_load", "pointid_gather", "pointid_gather_planes",
                 "pointid_downsample"):
        monkeypatch.setattr(binding.lib, name, call(name))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda d: types.SimpleNamespace(cuda_stream=100 + torch.device(d).index))
    monkeypatch.setattr(binding, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(binding, "_empty", lambda shape, dtype, device, stream: there(torch.empty(shape, dtype=dtype)))
    binding.seen, binding.now = seen, now
    yield binding
    del binding.seen, binding.now


def value(stream):
    return stream.value if isinstance(stream, ctypes.c_void_p) else stream


@pytest.mark.parametrize("current", [0, 1])
def test_the_tensors_device_is_current(b, current):
    b.now[0] = current
    x = there(torch.ones((4, 40), dtype=torch.bfloat16))
    c = b.pointid_checkpoint_save(x)
    b.pointid_checkpoint_load(c, torch.bfloat16)
    image, hits = there(torch.ones((64, 64))), there(torch.zeros((3, 2), dtype=torch.int32))
    b.pointid_gather(image, hits)
    b.pointid_gather_planes([image], there(torch.zeros((3, 3), dtype=torch.int32)))
    b.pointid_downsample(image, 2)
    assert [name for name, _, _ in b.seen] == ["pointid_checkpoint_save", "pointid_checkpoint_load", "pointid_gather",
                                               "pointid_gather_planes", "pointid_downsample"]
    assert all(on == 1 and value(stream) == 101 for _, on, stream in b.seen), b.seen
    assert b.now[0] == current
