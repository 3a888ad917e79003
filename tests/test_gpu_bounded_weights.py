"""The weights that a BoundedStream's steps leave, slot by slot, against 64 bits.

The scores are taken from the keys and queries that the attention itself had (turned and rounded
to bf16), so what is left is the attention's own error: a probability is off by
eps = 2 (D + 8) 2^-23 A + 2^-18 of itself, A the largest sum of |q_d k_d| scale of any query and
slot (D products summed in fp32 and scaled; maximum, sum, logarithm and exponential 2^-18
together), and the decayed total and the sum round to fp32, 2^-22 of them together. Each step
starts from the weights that the library had before it, so that a step's error is its own.

The same bounds have to tell a step that forgets the decay, its own weights, or to start a new
entry at nothing: the mistakes are made in the reference."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("n,whole", [(1, False), (3, False), (24, True), (40, False)])
def test_weights_of_every_step(n, whole, turned):
    S, H, G, D, C, decay = 2, 8, 2, 64, 96, 0.9
    steps = 9 if n > 1 else 110
    gen = torch.Generator(device="cuda").manual_seed(n)
    b = BoundedStream(S, H, G, D, C, plan=fdp.Rotary(D, 32, "half") if turned else None, sinks=2,
                      recent=n, decay=decay)
    told = {"no decay": 0, "nothing added": 0, "a new entry keeps the old weight": 0}
    for step in range(steps):
        q, k, v = (torch.randn(S, n, h, D, generator=gen, device="cuda").bfloat16()
                   for h in (H, G, G))
        pos = (step * n + torch.arange(n, device="cuda").int()).expand(S, n).contiguous()
        before = b.cache.weight.double()
        b.step(q, k, v, pos, whole_chunk=whole)
        got = b.cache.weight.double()
        slots = b._buffers[("slots", (S, G, n))].long()
        reset = before.scatter(-1, slots, 0.0)
        q = (b._buffers[("q", q.shape)] if turned else q).double().view(S, n, G, H // G, D)
        where, keys = b.cache.pos.long(), b.cache.k.double()
        score = torch.einsum("sngid,sgjd->sngij", q, keys) / 8
        size = float((torch.einsum("sngid,sgjd->sngij", q.abs(), keys.abs()) / 8).max())
        last = pos[:, -1:].expand(S, n) if whole else pos
        seen = (where >= 0)[:, None, :, None] & (where[:, None, :, None]
                                                 <= last[:, :, None, None, None])
        added = torch.nan_to_num(torch.softmax(score.masked_fill(~seen, -math.inf), -1)).sum((1, 3))
        eps = 2 * (D + 8) * 2.0 ** -23 * size + 2.0 ** -18

        def fits(decayed, more):
            tol = eps * more + 2.0 ** -22 * (decayed + more)
            return bool(((got - decayed - more).abs() <= tol + 1e-30).all())
        assert fits(decay * reset, added)
        told["no decay"] += not fits(reset, added)
        told["nothing added"] += not fits(decay * reset, torch.zeros_like(added))
        told["a new entry keeps the old weight"] += not fits(decay * before, added)
    # the first step has nothing to decay, and slots hold no weight until the cache is full
    assert told["nothing added"] == steps and told["no decay"] >= steps - 1
    assert told["a new entry keeps the old weight"] >= steps - -(-C // n) - 1
    b.check()
