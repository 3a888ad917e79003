"""Insert over list lengths that bring every form of the selection: how many slots a thread holds
depends on the lists' length and on how many there are (one CTA a list from 77 lists on, clusters
of up to 8 below). Bit for bit against a sorted list."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

# lists, slots, new tokens, empty share
CASES = [
    (80, 1500, 1, 0.0), (80, 2048, 1, 0.01),      # one token, up to 2 slots a thread
    (80, 3000, 1, 0.0), (77, 12288, 1, 0.0),      # 3 to 12
    (80, 12289, 1, 0.01), (77, 24576, 1, 0.0),    # 13 to 24
    (77, 24577, 1, 0.0),                          # read again
    (80, 8193, 700, 0.01), (77, 12288, 5, 0.0),   # several tokens, 9 to 12
    (77, 12289, 3001, 0.01), (80, 20000, 2, 0.0), (77, 24576, 24000, 0.0),  # 13 to 24
    (77, 24577, 100, 0.01),                       # read again
    (1, 130000, 777, 0.001), (1, 130000, 1, 0.0),  # a cluster of 8, 16 slots a thread
    (1, 200000, 1, 0.001),                        # a cluster of 8, read again
    (3, 9000, 33, 0.0), (40, 9000, 1, 0.0), (40, 9000, 100, 0.01),  # clusters of 8 and 2
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("ties", [False, True])
def test_insert(case, ties):
    lists, C, n, empty = case
    D, sinks, recent = 64, 3, C // 5
    gen = torch.Generator(device="cuda").manual_seed(C + n)
    k = torch.zeros(lists, 1, C, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    pos = torch.rand(lists, 1, 2 * C, generator=gen, device="cuda").argsort(-1)[..., :C].int()
    pos[torch.rand(lists, 1, C, generator=gen, device="cuda") < empty] = -1
    weight = torch.rand(lists, 1, C, generator=gen, device="cuda")
    if ties:
        weight.mul_(5).floor_()
    cache = fdp.Cache(k, v, pos.clone(), weight.clone())
    k_new = torch.randn(lists, n, 1, D, generator=gen, device="cuda").bfloat16()
    v_new = torch.randn(lists, n, 1, D, generator=gen, device="cuda").bfloat16()
    new_pos = (2 * C + torch.arange(n, device="cuda").int()).expand(lists, n).contiguous()
    slots = torch.full((lists, 1, n), -9, dtype=torch.int32, device="cuda")
    fdp.op_cache_insert(cache, k_new, v_new, new_pos, slots, sinks=sinks, recent=recent)
    # stable sorts by weight, then by class, leave ties in the order of their slots
    cls = torch.where(pos < 0, 0, torch.where((pos < sinks) | (pos >= 2 * C - recent), 2, 1))
    by_weight = torch.where(pos < 0, 0.0, weight).sort(dim=-1, stable=True).indices
    order = by_weight.gather(-1, cls.gather(-1, by_weight).sort(dim=-1, stable=True).indices)
    want = order[..., :n].sort(-1).values
    assert torch.equal(slots.long(), want)
    assert torch.equal(cache.pos, pos.scatter(-1, want, new_pos[:, None]))
    assert torch.equal(cache.weight, weight.scatter(-1, want, 0.0))
    rows = want[..., None].expand(lists, 1, n, D)
    for x, new in ((k, k_new), (v, v_new)):
        assert torch.equal(x.gather(2, rows), new.transpose(1, 2))
        left = x.scatter(2, rows, 0.0)
        assert not bool(left.any())
