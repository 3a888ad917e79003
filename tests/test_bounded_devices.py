"""Where the tensors of the rotary and bounded-cache calls may be: on the current CUDA device, since
the library launches on the current device whatever its pointers belong to. Stand-ins for tensors
carry the device's number, so that the refusals can be tested without a GPU (or a second one)."""
import ctypes

import pytest
import torch

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")


class OnDevice:
    """What the binding asks a contiguous tensor, and nothing behind it."""

    def __init__(self, device, shape, dtype):
        self.device_index, self.shape, self.dtype = device, torch.Size(shape), dtype
        self.nbytes = 1 << 20
        steps = []
        for n in reversed(shape):
            steps.insert(0, steps[0] * last if steps else 1)
            last = n
        self.steps = tuple(steps)

    def get_device(self):
        return self.device_index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self):
        return self.steps

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


class Lib:
    """The library, with its launching calls counted instead of made."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 64 if name.endswith("_bytes") else 0
        return call


def calls(device):
    """The four calls on tensors of `device`."""
    def t(shape, dtype=torch.bfloat16):
        return OnDevice(device, shape, dtype)

    def cache(capacity):
        c = object.__new__(fdp.Cache)
        c.streams, c.groups, c.capacity, c.head_dim = 2, 4, capacity, 64
        c.device, c.dtype, c.int32, c.float32 = device, torch.bfloat16, torch.int32, torch.float32
        c.pos, c.weight = t((2, 4, capacity), torch.int32), t((2, 4, capacity), torch.float32)
        c.ref, c._workspace = ctypes.byref(ctypes.c_int()), {}
        return c
    plan = object.__new__(fdp.Rotary)
    plan.head_dim, plan.axes, plan.int32, plan.handle = 64, 1, torch.int32, None
    q, new = t((2, 3, 16, 64)), t((2, 3, 4, 64))
    pos, err = t((2, 3), torch.int32), t((1,), torch.int32)
    x = t((6, 16, 64))
    return {
        "rotary": lambda **kw: fdp.op_rotary(plan, t((6,), torch.int32), x, x, **kw),
        "attention": lambda **kw: fdp.op_cache_attention(
            cache(100), q, pos, q, workspace=t((1 << 20,), torch.uint8), err=err, **kw),
        "insert": lambda **kw: fdp.op_cache_insert(cache(100), new, new, pos,
                                                   t((2, 4, 3), torch.int32), **kw),
        "compact": lambda **kw: fdp.op_cache_compact(
            cache(100), cache(10), t((2,), torch.int32), t((2, 4, 10), torch.int32), **kw),
    }


@pytest.fixture
def library(monkeypatch):
    lib = Lib()
    monkeypatch.setattr(fdp, "lib", lambda: lib)
    monkeypatch.setattr(fdp, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(fdp, "_get_device", lambda: 0)  # the current device
    return lib


@pytest.mark.parametrize("call", ["rotary", "attention", "insert", "compact"])
@pytest.mark.parametrize("stream", [None, 1 << 12])
def test_tensors_of_another_device_are_refused(library, call, stream):
    with pytest.raises(ValueError, match="cuda:1.*current device"):
        calls(1)[call](stream=stream)
    assert not [c for c in library.calls if c.startswith("fd_op")]
    calls(0)[call](stream=stream)
    assert len([c for c in library.calls if c.startswith("fd_op")]) == 1
