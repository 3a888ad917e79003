"""A BoundedStream with its default settings follows the stream: what came last is in the cache,
long after the cache was full."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402


@pytest.mark.parametrize("n", [1, 8])
def test_the_newest_entries_are_kept(n):
    S, H, G, D, C = 1, 4, 2, 64, 64
    gen = torch.Generator(device="cuda").manual_seed(n)
    b = BoundedStream(S, H, G, D, C)
    for at in range(0, 4 * C, n):
        x = [torch.randn(S, n, h, D, generator=gen, device="cuda").bfloat16() for h in (H, G, G)]
        b.step(*x, (at + torch.arange(n, device="cuda").int()).expand(S, n).contiguous())
    newest = set(range(4 * C - C // 2, 4 * C))
    for g in range(G):
        held = set(b.cache.pos[0, g].tolist())
        assert newest <= held and {0, 1, 2, 3} <= held
    # cut down, half of the smaller cache is the newest too
    small = b.compact(C // 2, torch.full((S,), 4 * C, dtype=torch.int32, device="cuda"))
    for g in range(G):
        held = small.cache.pos[0, g].tolist()
        assert set(range(4 * C - C // 4, 4 * C)) <= set(held) and min(held) < 4
        assert any(4 <= p < 4 * C - C // 4 for p in held)
    b.check(), small.check()


def test_settings_that_are_given_hold():
    b = BoundedStream(1, 4, 2, 64, 64, recent=0)
    assert b.recent == 0
    small = b.compact(32, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert small.recent == 0 and small.sinks == b.sinks and small.decay == b.decay
