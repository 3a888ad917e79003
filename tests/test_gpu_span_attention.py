"""Attention in spans of keys on the GPU against plain attention in 64 bits.

Tolerances. With A the largest sum of |q_d k_d| scale of any (query, key), a score's error in fp32 is at
most (D + 8) 2^-23 A (products are exact, sums and the scale round, tensor cores truncate), and maximum,
sum, logarithm and exponential add 2^-18 together; so a probability is relatively off by
eps = 2 (D + 8) 2^-23 A + 2^-18 (numerator and sum). Output: P is rounded to the type (u = 2^-8 or
2^-11; fp16 2^-25 of the row's largest at least, which a maximum kept up to 2^8 behind makes 2^-25 of 1)
and the result once more: (u + eps) sum p |v| + u |out|, fp16 outputs by 2^-25 at least. lse: the
score's error, and 2^-22 of its size and of the logarithm."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
BF16, FP16 = torch.bfloat16, torch.float16


def matrix(gen, tokens, heads, D, dtype, layout):
    if layout == "dense":
        x = torch.empty(tokens, heads, D, dtype=dtype, device="cuda")
    elif layout == "head_major":
        x = torch.empty(heads, tokens, D, dtype=dtype, device="cuda").transpose(0, 1)
    else:  # a part of a wider projection
        x = torch.full((tokens, heads + 2, D + 8), math.nan, dtype=dtype, device="cuda")[:, 1:heads + 1, 8:]
    return x.copy_(torch.randn(tokens, heads, D, generator=gen, device="cuda"))


def packed(lengths, pad=0, chunk=1, window=0, new=0):
    """Spans of sequences one behind another (causal by chunks, the last `window` of them; the last
    `new` tokens alone as queries), `pad` queries that see nothing behind them."""
    at, spans = 0, []
    for n in lengths:
        for p in range(max(0, n - new) if new else 0, n):
            c = p // chunk
            spans.append((at + (max(0, (c - window + 1) * chunk) if window else 0),
                          at + min(n, (c + 1) * chunk)))
        at += n
    return spans + [(0, 0)] * pad, at


def anywhere(T, S, seed, empty=0.3):
    """Spans in no order, some of them empty, some past the keys at either end."""
    rng = random.Random(seed)
    spans = []
    for _ in range(T):
        a, b = sorted(rng.randint(-5, S + 5) for _ in range(2))
        spans.append((b, a) if rng.random() < empty else (a, b))
    return spans


def make(spans, n_k, heads, groups, D, dtype, layout="dense", seed=0, size=1.0, nan=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = len(spans)
    s = {"q": matrix(gen, T, heads, D, dtype, layout), "k": matrix(gen, n_k, groups, D, dtype, layout),
         "v": matrix(gen, n_k, groups, D, dtype, layout),
         "dout": matrix(gen, T, heads, D, dtype, layout),
         "spans": torch.tensor(spans, dtype=torch.int32, device="cuda").view(T, 2)}
    if size != 1.0:
        s["q"].mul_(size)
    j = torch.arange(n_k, device="cuda")
    s["seen"] = (j >= s["spans"][:, :1]) & (j < s["spans"][:, 1:])
    if nan:  # what nothing sees, or sees nothing, may hold anything
        for n, there in (("q", s["seen"].any(1)), ("dout", s["seen"].any(1)), ("k", s["seen"].any(0)),
                         ("v", s["seen"].any(0))):
            s[n][~there] = math.nan
    return s


def run(s, scale=None, workspace_fill=255):
    T, H, D = s["q"].shape
    S, G = s["k"].shape[:2]
    out = torch.full_like(s["q"], 7.0)
    lse = torch.full((H, T), 7.0, device="cuda")
    need = fdp.span_attention_workspace_bytes(T, S, H, G, D)
    work = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(workspace_fill)  # (NaN)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fdp.op_span_attention(s["q"], s["k"], s["v"], s["spans"], out, lse, scale=scale, workspace=work,
                          err=err)
    assert int(err) == 0
    return out, lse


def heads_of(s, scale):
    """For every head: (h, its group, its queries, keys, values, scores, -inf where hidden, A)."""
    H, G, D = s["q"].shape[1], s["k"].shape[1], s["q"].shape[2]
    scale = D ** -0.5 if scale is None else scale
    rows, keys = s["seen"].any(1)[:, None], s["seen"].any(0)[:, None]
    for h in range(H):
        g = h // (H // G)
        q = torch.where(rows, s["q"][:, h], 0).double()
        k = torch.where(keys, s["k"][:, g], 0).double()
        v = torch.where(keys, s["v"][:, g], 0).double()
        x = (q @ k.t()) * scale
        size = float((q.abs() @ k.abs().t()).max()) * scale
        yield h, g, q, k, v, x.masked_fill(~s["seen"], -math.inf), size


def check(s, out, lse, scale=None):
    dtype, D = s["q"].dtype, s["q"].shape[2]
    u = U[dtype]
    for h, g, q, k, v, x, size in heads_of(s, scale):
        want_lse = torch.logsumexp(x, 1)
        p = torch.nan_to_num(torch.exp(x - want_lse[:, None]))
        want = p @ v
        score = (D + 8) * 2.0 ** -23 * size
        eps = 2 * score + 2.0 ** -18
        tol = (u + eps) * (p @ v.abs()) + u * want.abs()
        if dtype == FP16:
            tol = tol + 2.0 ** -25 * s["seen"].double() @ v.abs() + 2.0 ** -25
        off = (out[:, h].double() - want).abs()
        assert not bool((~(off <= tol)).any()), (h, float((off / tol).max()))
        none = want_lse == -math.inf
        assert torch.equal(lse[h] == -math.inf, none)
        assert not bool(out[:, h][none].any())
        off = (lse[h].double() - want_lse)[~none].abs()
        tol = score + 2.0 ** -18 + 2.0 ** -22 * (want_lse[~none].abs() + size)
        assert not bool((~(off <= tol)).any()), (h, float((off / tol).max()))


CASES = [
    # spans, heads, groups
    ("one", packed([1]), 1, 1),
    ("two_keys", packed([2]), 4, 2),
    ("short", packed([77, 50], pad=3), 6, 2),
    ("block", packed([128]), 4, 4),
    ("block_and_one", packed([129]), 2, 1),
    ("causal", packed([700]), 8, 2),
    ("ragged", packed([1, 200, 33, 128, 257, 5], pad=40), 10, 2),
    ("chunks", packed([600], chunk=150, window=2), 4, 1),
    ("chunks_wide", packed([1000], chunk=130, window=4), 3, 1),
    ("window", packed([500, 100], window=37), 7, 7),
    ("tokens", packed([300, 1, 1000, 64, 2000], new=1), 16, 4),
    ("few", packed([1500, 900], new=5), 8, 1),
    ("many_heads", packed([40]), 128, 1),
    ("odd_heads", packed([90]), 65, 1),
    ("long_past", packed([20000], new=3), 4, 1),
]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("name,spans,heads,groups", CASES, ids=[c[0] for c in CASES])
def test_masks(name, spans, heads, groups, dtype, D):
    s = make(spans[0], spans[1] + 3, heads, groups, D, dtype, seed=len(spans[0]))
    check(s, *run(s))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,S", [(1, 1), (5, 300), (200, 130), (333, 700)])
def test_spans_in_no_order(T, S, D):
    for seed in range(2):
        s = make(anywhere(T, S, seed), S, 6, 3, D, BF16, seed=seed)
        check(s, *run(s))


@pytest.mark.parametrize("layout", ["head_major", "part"])
@pytest.mark.parametrize("D", [64, 128])
def test_layouts(layout, D):
    spans, n = packed([150, 151])
    s = make(spans, n, 6, 2, D, FP16, layout=layout)
    check(s, *run(s))
    out = torch.full((n, 8, D + 8), 7.0, dtype=FP16, device="cuda")  # a part of a wider buffer
    lse = torch.empty(6, n, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    work = torch.empty(fdp.span_attention_workspace_bytes(n, n, 6, 2, D), dtype=torch.uint8, device="cuda")
    fdp.op_span_attention(s["q"], s["k"], s["v"], s["spans"], out[:, 1:7, 8:], lse, workspace=work, err=err)
    check(s, out[:, 1:7, 8:], lse)
    out[:, 1:7, 8:] = 7.0
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("D", [64, 128])
def test_sharp_and_flat_scores(D):
    spans, n = packed([400])
    for size, scale in ((30.0, None), (1e-3, None), (1.0, 2.5)):
        s = make(spans, n, 4, 2, D, BF16, size=size)
        check(s, *run(s, scale), scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_rising_scores(D):
    """Every block's scores are far above those before: the maximum moves all the time."""
    n = 1300
    s = make([(0, n)] * 64, n, 2, 2, D, BF16, nan=False)
    s["q"].fill_(1.0)
    s["k"].copy_((torch.arange(n, device="cuda") / 16)[:, None, None])
    check(s, *run(s, scale=1 / D), scale=1 / D)
    s["k"].copy_(s["k"].flip(0))
    check(s, *run(s, scale=1 / D), scale=1 / D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("level", [-300.0, 300.0])
def test_scores_far_from_zero(level, dtype, D):
    """Rows whose first keys come at any place, with scores far below or above zero, and steps of a few
    powers of two between the blocks."""
    n = 700
    for spans in (packed([n], window=300)[0], anywhere(260, n, 3)):
        s = make(spans, n, 2, 1, D, dtype, nan=False)
        s["q"].fill_(1.0)
        s["k"].copy_((level + 4 * (torch.arange(n, device="cuda") // 100 % 3))[:, None, None])
        check(s, *run(s, scale=1 / D), scale=1 / D)


def test_equal_calls_give_equal_bits():
    spans, n = packed([1, 200, 33, 128, 257, 5], pad=40)
    for D in (64, 128):
        s = make(spans, n, 8, 2, D, BF16)
        a, b = run(s, workspace_fill=0), run(s)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_streams_and_graphs():
    spans, n = packed([1000, 500], new=3)
    s = make(spans, n, 8, 2, 64, BF16)
    want = run(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    T, H = len(spans), 8
    out, lse = torch.empty_like(s["q"]), torch.empty(H, T, device="cuda")
    work = torch.empty(fdp.span_attention_workspace_bytes(T, n, H, 2, 64), dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda: fdp.op_span_attention(s["q"], s["k"], s["v"], s["spans"], out, lse,  # noqa: E731
                                         workspace=work, err=err)
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(2):
        out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    s["spans"][:, 1] -= 7  # other spans, the same graph
    want = run(s)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_no_queries_and_no_keys():
    s = make([], 50, 4, 2, 64, BF16)
    run(s)
    s = make([(0, 5)] * 9, 0, 4, 2, 64, BF16)
    out, lse = run(s)
    assert not bool(out.any()) and bool((lse == -math.inf).all())


def test_tensors_that_are_refused():
    spans, n = packed([40])
    s = make(spans, n, 4, 2, 64, BF16)
    out, lse = torch.empty_like(s["q"]), torch.empty(4, n, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def call(**kw):
        d = dict(q=s["q"], k=s["k"], v=s["v"], spans=s["spans"], out=out, lse=lse, workspace=work, err=err)
        d.update(kw)
        fdp.op_span_attention(**d)

    call()
    for bad in (dict(q=s["q"].cpu()), dict(k=s["k"].cpu()), dict(v=s["v"].half()), dict(q=s["q"][0]),
                dict(k=s["k"][..., :32]), dict(spans=s["spans"].long()), dict(spans=s["spans"][:5]),
                dict(out=out.half()), dict(out=out[:5]), dict(lse=lse.t()), dict(lse=lse.double()),
                dict(err=err.cpu()), dict(err=err.float()), dict(q=s["q"].transpose(0, 2))):
        with pytest.raises((TypeError, ValueError)):
            call(**bad)
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(err=None),
                dict(q=torch.empty(n, 5, 64, dtype=BF16, device="cuda"),
                     out=torch.empty(n, 5, 64, dtype=BF16, device="cuda"),
                     lse=torch.empty(5, n, device="cuda")),
                dict(k=s["k"][:, :1].expand(-1, 2, -1))):
        with pytest.raises(fdp.FdError):
            call(**bad)
