"""Steps of a BoundedStream on views of a fused projection [S][n][heads + 2 groups][D], and on keys
and values of different layouts, against the same steps on contiguous copies: equal bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402

H, G, D, C = 8, 2, 64, 48


@pytest.mark.parametrize("S", [1, 2])
@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("layout", ["fused", "k contiguous", "v contiguous", "group major"])
def test_steps_on_views(S, turned, layout):
    gen = torch.Generator(device="cuda").manual_seed(S)
    plan = fdp.Rotary(D, 32, "half") if turned else None
    views = BoundedStream(S, H, G, D, C, plan=plan, sinks=1, recent=8)
    copies = BoundedStream(S, H, G, D, C, plan=plan, sinks=1, recent=8)
    at = 0
    for n in (40, 1, 1, 5, 24, 1):
        x = torch.randn(S, n, H + 2 * G, D, generator=gen, device="cuda").bfloat16()
        q, k, v = x[:, :, :H], x[:, :, H:H + G], x[:, :, H + G:]
        if layout == "k contiguous":
            k = k.contiguous()
        elif layout == "v contiguous":
            v = v.contiguous()
        elif layout == "group major":
            v = v.transpose(1, 2).contiguous().transpose(1, 2)
        before = x.clone()
        pos = (at + torch.arange(n, device="cuda").int()).expand(S, n).contiguous()
        at += n
        got = views.step(q, k, v, pos)
        want = copies.step(q.contiguous(), k.contiguous(), v.contiguous(), pos)
        assert torch.equal(got, want) and torch.equal(x, before)
        for a, b in ((views.cache.k, copies.cache.k), (views.cache.v, copies.cache.v),
                     (views.cache.pos, copies.cache.pos),
                     (views.cache.weight, copies.cache.weight)):
            assert torch.equal(a, b)
    views.check(), copies.check()


def test_host_values_are_refused_in_any_layout():
    b = BoundedStream(1, H, G, D, C)
    q, k = (torch.zeros(1, 3, h, D, dtype=torch.bfloat16, device="cuda") for h in (H, G))
    pos = torch.arange(3, device="cuda").int()[None]
    for v in (k.cpu(), torch.zeros(1, 3, G + 1, D, dtype=torch.bfloat16)[:, :, :G]):
        with pytest.raises(TypeError):
            b.step(q, k, v, pos)
    assert b.filled == 0
