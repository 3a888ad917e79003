"""Layouts that users of the bounded cache have: a dimension of one entry with any stride, and
queries, keys and values that are views of one fused projection."""
import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402

D = 64


def bits(x):
    return x.contiguous().view(torch.int16)


def test_a_dimension_of_one_entry_may_have_any_stride():
    """Keys and values of one stream, one group or one token that come from different buffers: the
    strides that are never stepped differ."""
    gen = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").bfloat16()
    for S, G in ((1, 1), (1, 3), (3, 1)):
        C = 40
        k = randn(S, G, C, D)
        wide = randn(S + 1, G + 1, C, D)
        v = wide[:S, :G].contiguous() if S > 1 and G > 1 else wide.as_strided(
            (S, G, C, D), (k.stride(0) if S > 1 else 8 * wide.stride(0),
                           k.stride(1) if G > 1 else 16 * C * D, D, 1))
        pos = torch.full((S, G, C), -1, dtype=torch.int32, device="cuda")
        cache = fdp.Cache(k, v, pos, torch.zeros(S, G, C, device="cuda"))
        for n in (1, 2):
            k_new = randn(S, n, G, D)
            fused = randn(S, n, G + 2, D)
            # the token's stride differs where there is one token, the group's where there is one group
            v_new = fused[:, :, :G] if n == 1 and S == 1 else randn(S, n, G, D)
            new_pos = torch.arange(n, device="cuda").int().expand(S, n).contiguous()
            slots = torch.empty(S, G, n, dtype=torch.int32, device="cuda")
            cache.pos.fill_(-1)
            fdp.op_cache_insert(cache, k_new, v_new, new_pos, slots)
            assert torch.equal(bits(k[:, :, :n]), bits(k_new.transpose(1, 2)))
            assert torch.equal(bits(v[:, :, :n]), bits(v_new.transpose(1, 2)))


def test_strides_that_are_stepped_have_to_agree():
    x = torch.zeros(2, 2, 50, D, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(2, 50, 2, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    pos = torch.full((2, 2, 50), -1, dtype=torch.int32, device="cuda")
    weight = torch.zeros(2, 2, 50, device="cuda")
    with pytest.raises(ValueError):
        fdp.Cache(x, y, pos, weight)
    cache = fdp.Cache(x, torch.zeros_like(x), pos, weight)
    k = torch.zeros(2, 3, 2, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(2, 3, 4, D, dtype=torch.bfloat16, device="cuda")[:, :, 1:3]
    with pytest.raises(ValueError):
        fdp.op_cache_insert(cache, k, v, torch.zeros(2, 3, dtype=torch.int32, device="cuda"),
                            torch.empty(2, 2, 3, dtype=torch.int32, device="cuda"))
