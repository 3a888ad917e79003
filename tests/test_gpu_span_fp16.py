"""Attention in spans of keys in fp16 where its range could cost digits: few large probabilities beside many
small ones, gradients of very different sizes beside each other.

Tolerances are those of test_gpu_span_attention.py and test_gpu_span_gradient.py without what these allow fp16 for
each key that a query sees. Forward: probabilities keep half a step, 2^-11, down to 2^-25 of the row's largest.
Gradient: dS is off by 2^-25 of the largest |dout| of its own row (dq) or of the rows that see the key (dk). (Where
values are so large that 2^-39 of dS's bound is more than that, half a step of P M is, too.)"""
import math

import pytest
import torch
from test_gpu_span_attention import FP16, U, check, heads_of, make, packed, run
from test_gpu_span_gradient import check as check_bwd
from test_gpu_span_gradient import run_bwd

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")


def sink_and_tail(top, place, n, rows, D, seed=0):
    """Queries whose score is `top` with one key and 0 with all the others; values around 1, those of the one 0."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k = torch.zeros(rows, 1, D, dtype=FP16, device="cuda"), torch.zeros(n, 1, D, dtype=FP16, device="cuda")
    q[..., 3], k[place, 0, 3] = 4.0, top / 4
    v = (0.5 + torch.rand(n, 1, D, generator=gen, device="cuda")).half()
    v[place] = 0
    return {"q": q, "k": k, "v": v, "spans": torch.tensor([(0, n)] * rows, dtype=torch.int32, device="cuda")}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("top", [12.0, 16.0, 17.25])
@pytest.mark.parametrize("place", [0, 25000, 49999])
def test_one_key_far_above_many(place, top, D):
    """50000 keys; enough row tiles that none is split, so that one maximum stands for all of them: the others'
    probabilities are 2^-17 to 2^-25 of it, 24 % to 0.16 % of the sum."""
    n, rows = 50000, 20000
    s = sink_and_tail(top, place, n, rows, D)
    assert fdp.span_attention_workspace_bytes(rows, n, 1, 1, D) == 0  # (no parts)
    out, lse = run(s, scale=1.0)
    total = math.exp(top) + n - 1
    want = s["v"][:, 0].double().sum(0) / total
    u, score = U[FP16], (D + 8) * 2.0 ** -23 * top
    tol = (2 * u + 2 * score + 2.0 ** -18) * want
    off = (out[:, 0].double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    off = (lse[0].double() - math.log(total)).abs()
    assert bool((off <= score + 2.0 ** -18 + 2.0 ** -22 * (math.log(total) + top)).all())


@pytest.mark.parametrize("D", [64, 128])
def test_one_key_far_above_many_in_parts(D):
    """The same of few queries, whose keys are walked in parts."""
    n, top = 50000, 16.0
    s = sink_and_tail(top, 20000, n, 3, D)
    assert fdp.span_attention_workspace_bytes(3, n, 1, 1, D) > 0
    out, lse = run(s, scale=1.0)
    total = math.exp(top) + n - 1
    want = s["v"][:, 0].double().sum(0) / total
    tol = (2 * U[FP16] + 2 * (D + 8) * 2.0 ** -23 * top + 2.0 ** -18) * want
    assert bool(((out[:, 0].double() - want).abs() <= tol).all())
    assert bool(((lse[0].double() - math.log(total)).abs() <= 1e-4).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("step", [0.02, 1 / 16, 0.5])
def test_rising_scores(step, D):
    """The maximum moves with every block, by less and by more than it may before sums are rescaled."""
    n = 1300
    s = make([(0, n)] * 64, n, 2, 2, D, FP16, nan=False)
    s["q"].fill_(1.0)
    for way in (1, -1):
        s["k"].copy_(((torch.arange(n, device="cuda") * step) * way)[:, None, None])
        check(s, *run(s, scale=1 / D), scale=1 / D)


def gradient(s, out, lse, scale=None):
    """{name: (value, tolerance)} of the formula in 64 bits from out and lse as they are."""
    T, H, D = s["q"].shape
    S, G = s["k"].shape[:2]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    c, u = D ** -0.5 if scale is None else scale, U[FP16]
    found = {n: [torch.zeros(shape, **f64) for _ in range(2)]
             for n, shape in (("dq", (T, H, D)), ("dk", (S, G, D)), ("dv", (S, G, D)))}
    rows = s["seen"].any(1)[:, None]
    seen = s["seen"].double()
    top = torch.where(rows, s["dout"].abs().amax(2), 0).double()  # of a row
    of_key = torch.stack([(seen * t[:, None]).amax(0) for t in top.view(T, G, -1).amax(2).t()], 1)
    for h, g, q, k, v, x, size in heads_of(s, scale):
        do = torch.where(rows, s["dout"][:, h], 0).double()
        l = torch.where(rows[:, 0], lse[h], 0).double()[:, None]
        p = torch.exp(x - l)
        e = (2 * (D + 8) * 2.0 ** -23 * size + 2.0 ** -18 + 2.0 ** -22 * float(l.abs().max())
             + (D + 8) * 2.0 ** -23 + max(S, T * (H // G)) * 2.0 ** -24)
        o = out[:, h].double()
        ds = p * (do @ v.t() - (do * o).sum(1, keepdim=True))
        off = (u + e) * p * (do.abs() @ v.abs().t() + (do * o).abs().sum(1, keepdim=True))
        for n, at, value, tol in (
                ("dq", h, c * ds @ k, c * (off + 2.0 ** -25 * top[:, h:h + 1] * seen) @ k.abs()),
                ("dk", g, c * ds.t() @ q, c * (off + 2.0 ** -25 * of_key[:, g] * seen).t() @ q.abs()),
                ("dv", g, p.t() @ do, ((u + e) * p + 2.0 ** -39 * seen).t() @ do.abs())):
            found[n][0][:, at] += value
            found[n][1][:, at] += tol
    return {n: (a, b + (u * a.abs()).clamp_min(2.0 ** -25)) for n, (a, b) in found.items()}


def owner(lengths):
    return torch.cat([torch.full((n,), i) for i, n in enumerate(lengths)]).cuda()


@pytest.mark.parametrize("heads,groups,D", [(4, 1, 64), (2, 2, 128)])
@pytest.mark.parametrize("small", [1, 0.01, 0.001])
@pytest.mark.parametrize("lengths", [[1700, 2500], [2500, 1700], [60, 50] * 8, [1, 130, 700, 5, 129]], ids=str)
def test_sequences_with_gradients_far_apart(lengths, small, heads, groups, D):
    """Packed sequences, every other one with gradients 1000, the rest with small ones: none takes digits from
    another, wherever they meet in a tile."""
    spans, n = packed(lengths, pad=3)
    s = make(spans, n, heads, groups, D, FP16, seed=len(lengths))
    far = torch.cat([owner(lengths) % 2 == 1, torch.ones(3, dtype=torch.bool, device="cuda")])
    s["dout"][far] *= 1000
    s["dout"][~far] *= small
    out, lse = run(s)
    check_bwd(run_bwd(s, out, lse), gradient(s, out, lse), s)


@pytest.mark.parametrize("heads,groups,D", [(6, 2, 64), (3, 3, 128)])
def test_rows_with_gradients_far_apart(heads, groups, D):
    """Every query and head has gradients of another size, chunks and windows between them."""
    spans, n = packed([900, 333], chunk=7, window=40)
    s = make(spans, n, heads, groups, D, FP16, seed=D)
    gen = torch.Generator(device="cuda").manual_seed(3)
    power = torch.randint(-8, 10, (len(spans), heads, 1), generator=gen, device="cuda")
    s["dout"].copy_(torch.ldexp(s["dout"].float(), power))
    out, lse = run(s)
    check_bwd(run_bwd(s, out, lse), gradient(s, out, lse), s)


@pytest.mark.parametrize("D", [64, 128])
def test_few_keys_of_many_rows_with_gradients_far_apart(D):
    """Keys walked in parts: 300 keys and 6000 rows, whose gradients grow 2^16-fold from the first to the last;
    each row sees the keys around its place."""
    rows, n = 6000, 300
    spans = [(t * n // rows - 2, t * n // rows + 3) for t in range(rows)]
    s = make(spans, n, 2, 1, D, FP16)
    s["dout"].copy_(torch.ldexp(s["dout"].float(), (torch.arange(rows, device="cuda") * 16 // rows - 6)[:, None, None]))
    out, lse = run(s)
    check_bwd(run_bwd(s, out, lse), gradient(s, out, lse), s)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("keys", [2, 3, 150])
@pytest.mark.parametrize("size", [500.0, 4000.0])
def test_large_values_along_the_gradient(size, keys, D):
    """Values of some size with signs that dout shares: dS = P (dout . v - dout . out) is past fp16's largest number,
    dq and dk (scores' factors are small) are not."""
    spans, n = packed([keys] * 40)
    s = make(spans, n, 4, 2, D, FP16, seed=keys, size=0.05)
    s["k"].mul_(0.05)
    gen = torch.Generator(device="cuda").manual_seed(1)
    sign = torch.randint(0, 2, (1, 1, D), generator=gen, device="cuda") * 2 - 1
    s["v"].copy_(sign * size * (torch.arange(n, device="cuda") % 2 * 2 - 1)[:, None, None])
    s["dout"].copy_((1.5 + 0.4 * torch.rand(s["dout"].shape, generator=gen, device="cuda")) * sign)
    out, lse = run(s)
    want = gradient(s, out, lse)
    assert all(float(v.abs().max()) < 60000 for v, _ in want.values())
    check_bwd(run_bwd(s, out, lse), want, s)


@pytest.mark.parametrize("heads,groups,D", [(4, 1, 64), (2, 2, 128)])
@pytest.mark.parametrize("lengths", [[700, 900, 3], [60, 50] * 8, [1, 130, 700, 5, 129]], ids=str)
@pytest.mark.parametrize("first", [0, 1])
def test_sequences_with_values_far_apart(first, lengths, heads, groups, D):
    """Packed sequences, every other one with values of thousands, the rest with small ones."""
    spans, n = packed(lengths)
    s = make(spans, n, heads, groups, D, FP16, seed=len(lengths))
    far = owner(lengths) % 2 == first
    s["v"][far] *= 3000
    s["v"][~far] *= 0.01
    s["dout"].mul_(4)
    out, lse = run(s)
    # (a result past 65504 is an infinity of fp16, whatever computes it)
    want = {m: (v, torch.where(v.abs() < 65000, t, math.inf)) for m, (v, t) in gradient(s, out, lse).items()}
    check_bwd(run_bwd(s, out, lse), want, s)


@pytest.mark.parametrize("dtype", [torch.bfloat16, FP16], ids=str)
@pytest.mark.parametrize("D", [64, 128])
def test_what_nothing_sees_has_no_effect(D, dtype):
    """Whatever is in keys that no query sees and in queries that see nothing, the results are the same bits."""
    layouts = [([(0, 200)] * 32 + [(0, 0)] * 64 + [(300, 310)] * 32 + [(100, 200)] * 40, 400),
               ([(40, 41), (7, 7), (130, 250)] + [(251 + t, 255 + t) for t in range(20)], 600),
               ([(5, 70)] * 300, 20000)]
    for spans, n in layouts:
        found = []
        for fill in (0.0, math.inf, math.nan, torch.finfo(dtype).max, -1000.0):
            s = make(spans, n, 6, 2, D, dtype, nan=False)
            for name, there in (("q", s["seen"].any(1)), ("dout", s["seen"].any(1)), ("k", s["seen"].any(0)),
                                ("v", s["seen"].any(0))):
                s[name][~there] = fill
            out, lse = run(s)
            found.append([out, lse, *run_bwd(s, out, lse).values()])
        for got in found[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got, found[0]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths", [[77, 60], [400, 300]], ids=str)
def test_captured_gradient_with_other_inputs(lengths, D):
    """Scales are of the inputs at every replay: a captured gradient with gradients, values and spans of other sizes
    gives the bits of a call of its own."""
    spans, n = packed(lengths)
    s = make(spans, n, 6, 2, D, FP16, nan=False)
    out, lse = run(s)
    got = {"d" + m: torch.empty_like(s[m]) for m in "qkv"}
    work = torch.empty(fdp.span_attention_workspace_bytes(n, n, 6, 2, D, backward=True), dtype=torch.uint8,
                       device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fdp.op_span_attention_bwd(s["q"], s["k"], s["v"], s["spans"], out, lse, s["dout"], *got.values(),
                                  workspace=work, err=err)
    for change in range(4):
        if change == 1:
            s["dout"][::2] *= 1000
        elif change == 2:
            s["v"][:n // 2] *= 2000
        elif change == 3:
            s["spans"][:, 0] = (s["spans"][:, 1] - 9).clamp_min(0)
        fresh = run(s)
        out.copy_(fresh[0])
        lse.copy_(fresh[1])
        want = run_bwd(s, out, lse)
        for x in got.values():
            x.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[m], want[m]) for m in got), change
    assert int(err) == 0
