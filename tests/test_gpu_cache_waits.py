"""The bounded waits of the attention over a bounded cache for many rows, without a GPU fault: a wait on
a barrier that nothing arrives at gives up by the clock and says so in the status word, and a call
whose status word says that something has given up ends soon and leaves the next call as it was."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
CHECK = 32  # the bit that the check's waits set


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_a_wait_gives_up_by_the_clock(which):
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fdp.debug_cache_wait_timeout(which, err)  # loads the kernel
    torch.cuda.synchronize()
    err.zero_()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start = time.perf_counter()
    begin.record()
    fdp.debug_cache_wait_timeout(which, err)
    end.record()
    torch.cuda.synchronize()
    assert int(err) == CHECK and time.perf_counter() - start < 1.0
    assert begin.elapsed_time(end) >= 1.0  # not before its limit of 1 ms
    # another wait has given up: it ends early, a wait for copies in flight does not
    err.fill_(1)
    begin.record()
    fdp.debug_cache_wait_timeout(which, err)
    end.record()
    torch.cuda.synchronize()
    assert int(err) == 1 | CHECK
    if which == 1:
        assert begin.elapsed_time(end) >= 1.0


@pytest.mark.parametrize("D,n", [(64, 300), (128, 300), (128, 20)])
def test_a_call_after_one_that_gave_up(D, n):
    gen = torch.Generator(device="cuda").manual_seed(D)
    S, G, H, C = 2, 2, 16, 3000
    k, v = (torch.randn(S, G, C, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    pos = torch.arange(C, device="cuda").int().expand(S, G, C).contiguous()
    cache = fdp.Cache(k, v, pos, torch.zeros(S, G, C, device="cuda"))
    q = torch.randn(S, n, H, D, generator=gen, device="cuda").bfloat16()
    q_pos = torch.full((S, n), C, dtype=torch.int32, device="cuda")
    work = torch.empty(fdp.cache_attention_workspace_bytes(cache, H, n), dtype=torch.uint8,
                       device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        out, w = torch.empty_like(q), torch.empty_like(cache.weight)
        fdp.op_cache_attention(cache, q, q_pos, out, weight_out=w, workspace=work, err=err)
        return out, w
    want = call()
    assert int(err) == 0
    err.fill_(CHECK)
    torch.cuda.synchronize()
    start = time.perf_counter()
    call()
    torch.cuda.synchronize()
    assert time.perf_counter() - start < 1.0 and int(err) & CHECK
    err.zero_()
    got = call()
    assert int(err) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v)


def test_arguments():
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for which in (-1, 4):
        with pytest.raises(fdp.FdError):
            fdp.debug_cache_wait_timeout(which, err)
    with pytest.raises(TypeError):
        fdp.debug_cache_wait_timeout(0, err.long())
    assert int(err) == 0
