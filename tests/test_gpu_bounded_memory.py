"""A BoundedStream's memory does not grow with the number of step sizes that it has seen, and what a
captured step or the caller still uses is not taken away."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402

S, H, G, D, C = 1, 8, 2, 64, 400


def inputs(n, at, gen):
    x = [torch.randn(S, n, h, D, generator=gen, device="cuda").bfloat16() for h in (H, G, G)]
    return x + [(at + torch.arange(n, device="cuda").int()).expand(S, n).contiguous()]


@pytest.mark.parametrize("turned", [False, True])
def test_many_step_sizes_take_no_more_memory(turned):
    gen = torch.Generator(device="cuda").manual_seed(0)
    b = BoundedStream(S, H, G, D, C, plan=fdp.Rotary(D) if turned else None, sinks=1, recent=8)
    at, sizes = 0, [300 - i for i in range(60)]
    start, held = torch.cuda.memory_allocated(), []
    for n in sizes:
        b.step(*inputs(n, at, gen))
        at += n
        held.append(torch.cuda.memory_allocated() - start)
    # the first ten sizes are the largest; half as much again for how the allocator rounds
    assert max(held[10:]) <= 1.5 * max(held[:10])
    b.check()


def test_an_output_stays_until_a_step_of_its_size():
    gen = torch.Generator(device="cuda").manual_seed(1)
    b = BoundedStream(S, H, G, D, C, sinks=1, recent=8)
    out = b.step(*inputs(7, 0, gen))
    want, at = out.clone(), 7
    for n in range(20, 50):
        b.step(*inputs(n, at, gen))
        at += n
    assert torch.equal(out, want)


def test_a_captured_step_keeps_its_buffers():
    """A graph of a one-token step is replayed after many other sizes have come and gone, and
    what they let go of has been overwritten."""
    def fresh():
        gen = torch.Generator(device="cuda").manual_seed(2)
        b = BoundedStream(S, H, G, D, C, plan=fdp.Rotary(D), sinks=1, recent=8)
        b.step(*inputs(C, 0, gen))
        return b, gen
    plain, gen = fresh()
    graphed, gen2 = fresh()
    for b, g in ((plain, gen), (graphed, gen2)):  # the size's buffers are there before the capture
        b.step(*inputs(1, C, g))
    x = inputs(1, C + 1, gen)
    inputs(1, C + 1, gen2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = graphed.step(*x)
    at = C + 1
    want = plain.step(*x)
    graph.replay()
    assert torch.equal(got, want)
    for round_ in range(3):
        for n in range(2, 30):
            at += n
            y = inputs(n, at, gen)
            plain.step(*y)
            graphed.step(*y)
        junk = [torch.full((1 << s,), float("nan"), device="cuda") for s in range(8, 22)
                for _ in range(8)]
        want = plain.step(*x)
        graph.replay()
        assert torch.equal(got, want)
        assert torch.equal(plain.cache.weight, graphed.cache.weight)
        assert all(bool(j.isnan().all()) for j in junk)
    plain.check(), graphed.check()


def test_buffers_that_another_stream_still_uses():
    """Buffers that were allocated on the default stream are used on a side stream, which is behind,
    and let go of: the default stream's next tensors must not get their memory yet."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    b = BoundedStream(S, H, G, D, C, plan=fdp.Rotary(D), sinks=1, recent=8)
    sizes = (64, 65, 66, 67, 68, 69)
    steps = [inputs(n, 100 * i, gen) for i, n in enumerate((64,) + sizes)]
    b.step(*steps[0])
    shapes = [(t.shape, t.dtype) for t in b._buffers.values()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        for x in steps[1:]:
            b.step(*x)
    assert ("slots", (S, G, 64)) not in b._buffers  # let go of while the side stream sleeps
    taken = [torch.full(shape, 77, dtype=dtype, device="cuda")
             for shape, dtype in shapes for _ in range(4)]
    assert not side.query()
    torch.cuda.synchronize()
    assert all(bool((t == 77).all()) for t in taken)
    b.check()
