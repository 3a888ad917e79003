"""The operators for training a residual block on tensors whose elements lie past 2^31, and on the longest
keys that they take. A layout changes no sum: the results are those of dense tensors, bit for bit."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

BF16, F32 = torch.bfloat16, torch.float32


def far(like, base, at, strides):
    """A copy of `like` in the buffer `base`, `at` elements from its beginning."""
    return base.as_strided(like.shape, (*strides, 1), at).copy_(like)


def attention(t, spans, like, work, err):
    T, H, D = t["q"].shape
    lse = torch.empty(H, T, device="cuda")
    fdp.op_span_attention(t["q"], t["k"], t["v"], spans, t["out"], lse, workspace=work, err=err)
    fdp.op_span_attention_bwd(t["q"], t["k"], t["v"], spans, t["out"], lse, t["dout"], t["dq"], t["dk"], t["dv"],
                              workspace=work, err=err)
    assert int(err) == 0
    return lse


@pytest.mark.parametrize("strides,period", [((1 << 25, 64), 512), ((64, 1 << 30), 130 * 64)],
                         ids=["tokens", "heads"])
def test_attention(strides, period):
    T, H, G, D = 130, 4, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    names = {"q": H, "k": G, "v": G, "out": H, "dout": H, "dq": H, "dk": G, "dv": G}
    dense = {n: torch.randn(T, h, D, generator=gen, device="cuda").to(BF16) for n, h in names.items()}
    spans = torch.tensor([(t // 3, t + 1) for t in range(T)], dtype=torch.int32, device="cuda")
    need = max(fdp.span_attention_workspace_bytes(T, T, H, G, D, backward=b) for b in (False, True))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    last = (T - 1) * strides[0] + (H - 1) * strides[1] + 8 * period + D
    assert last > 1 << 31
    base = torch.empty(last, dtype=BF16, device="cuda")
    wide = {n: far(x, base, i * period, strides) for i, (n, x) in enumerate(dense.items())}
    want = attention(dense, spans, dense, work, err)
    got = attention(wide, spans, dense, work, err)
    assert torch.equal(got, want)
    for n in dense:
        assert torch.equal(wide[n], dense[n]), n


def test_join_and_checkpoints():
    rows, width, stride = 5, 264, 1 << 29
    gen = torch.Generator(device="cuda").manual_seed(1)
    names = ("h", "b", "y", "u", "dy", "du", "dh", "db")
    dense = {n: torch.randn(rows, width, generator=gen, device="cuda").to(BF16) for n in names}
    base = torch.empty((rows - 1) * stride + 8 * 512, dtype=BF16, device="cuda")
    wide = {n: far(x, base, i * 512, (stride,)) for i, (n, x) in enumerate(dense.items())}
    post, pre = (1 + 0.1 * torch.randn(width, generator=gen, device="cuda") for _ in range(2))
    found = []
    for t in (dense, wide):
        r = [torch.empty(rows, device="cuda") for _ in range(2)]
        kept = [fdp.Checkpoint8.empty(rows, width) for _ in range(2)]
        sums = [torch.empty(width, device="cuda") for _ in range(2)]
        work = torch.empty(fdp.block_join_bwd_workspace_bytes(rows, width), dtype=torch.uint8, device="cuda")
        fdp.op_block_join(t["h"], t["b"], t["y"], t["u"], post_gain=post, pre_gain=pre, r_post=r[0], r_pre=r[1],
                          h_kept=kept[0], b_kept=kept[1])
        fdp.op_block_join_bwd(t["dy"], t["du"], t["h"], t["b"], t["dh"], t["db"], post_gain=post, pre_gain=pre,
                              r_post=r[0], r_pre=r[1], d_post=sums[0], d_pre=sums[1], workspace=work)
        alone = fdp.Checkpoint8.empty(rows, width)
        fdp.op_checkpoint_save(t["h"], alone)
        assert torch.equal(alone.codes, kept[0].codes) and torch.equal(alone.exps, kept[0].exps)
        found.append([*r, *sums, kept[0].codes, kept[0].exps, kept[1].codes, kept[1].exps])
        fdp.op_checkpoint_load(alone, t["du"])
    for a, b in zip(*found):
        assert torch.equal(a, b)
    for n in names:
        assert torch.equal(wide[n], dense[n]), n
    # transposed: 72 columns 2^26 elements apart
    kept, x = fdp.Checkpoint8.empty(rows, 72), torch.empty(72, rows, dtype=BF16, device="cuda")
    fdp.op_checkpoint_save(dense["h"][:, :72], kept)
    fdp.op_checkpoint_load(kept, x, transposed=True)
    base = torch.empty(71 * (1 << 26) + rows, dtype=BF16, device="cuda")
    got = base.as_strided((72, rows), (1 << 26, 1))
    fdp.op_checkpoint_load(kept, got, transposed=True)
    assert torch.equal(got, x)


def test_longest_keys():
    """2^24 keys, of which the queries see all, the last one, and 1000 in the middle. The values are whole
    numbers that most keys hold as zero, and all scores are 0 (the queries are zeros), so that every sum
    is known: out = sum v / n, dv = sum of dout / n, dk = 0."""
    S, D = 1 << 24, 64
    spans = torch.tensor([(0, S), (S - 1, S), (S // 2, S // 2 + 1000)], dtype=torch.int32, device="cuda")
    q = torch.zeros(3, 1, D, dtype=BF16, device="cuda")
    k = torch.ones(S, 1, D, dtype=BF16, device="cuda")
    v = torch.ones(S, 1, D, dtype=BF16, device="cuda")
    v[S // 2:S // 2 + 500] = 3
    v[S - 1] = 5
    out, lse = torch.empty_like(q), torch.empty(1, 3, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    need = max(fdp.span_attention_workspace_bytes(3, S, 1, 1, D, backward=b) for b in (False, True))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    fdp.op_span_attention(q, k, v, spans, out, lse, workspace=work, err=err)
    # the sums of ones up to 2^24 are exact; those in parts are, too
    assert torch.equal(out[:, 0, 0].float().cpu(), torch.tensor([1.0, 5.0, 2.0]))
    want = torch.tensor([math.log(S), 0.0, math.log(1000)])
    assert bool(((lse[0].cpu() - want).abs() <= 2.0 ** -21 * want).all())
    dout = torch.zeros_like(out)
    dout[1], dout[2] = 1, 1000
    dq, dk, dv = torch.ones_like(q), torch.ones_like(k), torch.ones_like(v)
    fdp.op_span_attention_bwd(q, k, v, spans, out, lse, dout, dq, dk, dv, workspace=work, err=err)
    assert int(err) == 0
    want = torch.zeros(S, device="cuda")
    want[S - 1] = 1
    want[S // 2:S // 2 + 1000] = 1
    # P is 1 / 1000 by an exponential (2^-21), rounded to 8 bits, as dv is
    assert bool(((dv[:, 0].float() - want[:, None]).abs() <= (2.0 ** -8 * 2 + 2.0 ** -15) * want[:, None]).all())
    assert not bool(dk.any())
    # dq = scale sum dS k: dS = P (dout . v - dout . out) sums to 0 up to its rounding, 2^-8 of 64 000 each
    assert bool((dq[0] == 0).all()) and bool((dq[1] == 0).all())
    assert bool((dq[2].float().abs() <= 0.125 * 64000 * 2.0 ** -7).all())
