"""The status word of op_cache_attention: kernels read it while they wait and set bits in it, so it
has to be int32 memory of the call's device. Stand-ins for tensors, no GPU."""
import pytest
import torch

from test_bounded_devices import OnDevice, fdp, library  # noqa: F401


class Strided(OnDevice):
    def is_contiguous(self):
        return False


GOOD = [OnDevice(0, (1,), torch.int32), OnDevice(0, (), torch.int32), OnDevice(0, (4, 2), torch.int32)]
BAD = {
    "on the host": OnDevice(-1, (1,), torch.int32),
    "a host tensor": torch.zeros(1, dtype=torch.int32),
    "of another device": OnDevice(1, (1,), torch.int32),
    "64 bits": OnDevice(0, (1,), torch.int64),
    "one byte": OnDevice(0, (1,), torch.uint8),
    "fp32": OnDevice(0, (1,), torch.float32),
    "empty": OnDevice(0, (0,), torch.int32),
    "every second": Strided(0, (2,), torch.int32),
    "an address": 1 << 20,
}


def attention(err):
    S, G, C, D = 2, 4, 100, 64
    cache = object.__new__(fdp.Cache)
    cache.streams, cache.groups, cache.capacity, cache.head_dim = S, G, C, D
    cache.device, cache.dtype, cache.int32, cache.float32 = (0, torch.bfloat16, torch.int32,
                                                             torch.float32)
    cache.ref, cache._workspace = None, {}
    q = OnDevice(0, (S, 3, 16, D), torch.bfloat16)
    fdp.op_cache_attention(cache, q, OnDevice(0, (S, 3), torch.int32), q,
                           workspace=OnDevice(0, (1 << 20,), torch.uint8), err=err)


@pytest.mark.parametrize("name", BAD)
def test_what_is_no_status_word_is_refused(library, name):  # noqa: F811
    with pytest.raises((TypeError, ValueError), match="err"):
        attention(BAD[name])
    assert "fd_op_cache_attention" not in library.calls


def test_status_words(library):  # noqa: F811
    for err in GOOD:
        attention(err)
    assert library.calls.count("fd_op_cache_attention") == len(GOOD)


def test_the_library_asks_for_a_status_word():
    """Without one the library refuses the call (queries need one, gathering alone does not)."""
    from test_bounded_cache_args import INVALID, attend, cache
    assert attend(cache(), fdp.lib(), err=None) == INVALID
