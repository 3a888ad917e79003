"""The gradient of attention in spans of keys on the GPU against its formula in 64 bits and against
differences.

Tolerances, with those of the forward pass (test_gpu_span_attention.py): a probability is relatively off
by eps = 2 (D + 8) 2^-23 A + 2^-18 + 2^-22 |lse|, dout . v and delta by (D + 8) 2^-23 of their sums of
magnitudes M = |dout| . |v| and L = |dout| . |out|, and the products' sums of N terms in fp32 by N 2^-24
of their magnitudes; let e be the sum of these. P and dS are rounded to the type (u = 2^-8 or 2^-11).
So dv is off by (u + e) sum P |dout|, dS by (u + e) P (M + L), dq and dk by scale times the products of
that with |k| and |q|, and u of themselves. fp16: steps end at 2^-24: a result is off by 2^-25 at least, dS by
2^-25 of the largest |dout| (it is divided by the power of two in it), P by 2^-39."""
import math

import pytest
import torch
from test_gpu_span_attention import (BF16, CASES, FP16, U, anywhere, heads_of, make, matrix, packed,
                                     run)

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")


def run_bwd(s, out, lse, scale=None, into=None, workspace_fill=255):
    T, H, D = s["q"].shape
    S, G = s["k"].shape[:2]
    dq, dk, dv = into or (torch.full_like(s["q"], 7.0), torch.full_like(s["k"], 7.0),
                          torch.full_like(s["v"], 7.0))
    need = fdp.span_attention_workspace_bytes(T, S, H, G, D, backward=True)
    work = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(workspace_fill)  # (NaN)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fdp.op_span_attention_bwd(s["q"], s["k"], s["v"], s["spans"], out, lse, s["dout"], dq, dk, dv,
                              scale=scale, workspace=work, err=err)
    assert int(err) == 0
    return {"dq": dq, "dk": dk, "dv": dv}


def gradient(s, out, lse, scale=None):
    """{name: (value, tolerance)} of the formula in 64 bits from out and lse as they are."""
    T, H, D = s["q"].shape
    S, G = s["k"].shape[:2]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    c = D ** -0.5 if scale is None else scale
    u = U[s["q"].dtype]
    found = {n: [torch.zeros(shape, **f64) for _ in range(2)]
             for n, shape in (("dq", (T, H, D)), ("dk", (S, G, D)), ("dv", (S, G, D)))}
    rows = s["seen"].any(1)[:, None]
    top = float(torch.where(rows[..., None], s["dout"], 0).abs().max()) if T else 0.0
    low = 2.0 ** -25 * top if s["q"].dtype == FP16 else 0.0
    for h, g, q, k, v, x, size in heads_of(s, scale):
        do = torch.where(rows, s["dout"][:, h], 0).double()
        l = torch.where(rows[:, 0], lse[h], 0).double()[:, None]
        p = torch.exp(x - l)
        e = (2 * (D + 8) * 2.0 ** -23 * size + 2.0 ** -18 + 2.0 ** -22 * float(l.abs().max())
             + (D + 8) * 2.0 ** -23 + max(S, T * (H // G)) * 2.0 ** -24)
        o = out[:, h].double()
        ds = p * (do @ v.t() - (do * o).sum(1, keepdim=True))
        ds_off = (u + e) * p * (do.abs() @ v.abs().t() + (do * o).abs().sum(1, keepdim=True)) \
            + low * s["seen"]
        p_off = (u + e) * p + 2.0 ** -39 * s["seen"]
        for n, at, value, off in (("dq", h, c * ds @ k, c * ds_off @ k.abs()),
                                  ("dk", g, c * ds.t() @ q, c * ds_off.t() @ q.abs()),
                                  ("dv", g, p.t() @ do, p_off.t() @ do.abs())):
            found[n][0][:, at] += value
            found[n][1][:, at] += off
    step = 2.0 ** -25 if s["q"].dtype == FP16 else 1e-30
    return {n: (a, b + (u * a.abs()).clamp_min(step)) for n, (a, b) in found.items()}


def check(got, want, s):
    for n, (value, tol) in want.items():
        off = (got[n].double() - value).abs()
        bad = ~(off <= tol)
        assert not bool(bad.any()), (n, int(bad.sum()), float((off / tol).max()))
    rows, keys = s["seen"].any(1), s["seen"].any(0)
    assert not bool(got["dq"][~rows].any()) and not bool(got["dk"][~keys].any())
    assert not bool(got["dv"][~keys].any())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
@pytest.mark.parametrize("name,spans,heads,groups", CASES, ids=[c[0] for c in CASES])
def test_masks(name, spans, heads, groups, dtype, D):
    s = make(spans[0], spans[1] + 3, heads, groups, D, dtype, seed=len(spans[0]))
    out, lse = run(s)
    check(run_bwd(s, out, lse), gradient(s, out, lse), s)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,S", [(1, 1), (5, 300), (200, 130), (333, 700)])
def test_spans_in_no_order(T, S, D):
    for seed in range(2):
        s = make(anywhere(T, S, seed), S, 6, 3, D, BF16, seed=seed)
        out, lse = run(s)
        check(run_bwd(s, out, lse), gradient(s, out, lse), s)


def test_tiles_that_see_nothing_between_others():
    spans = [(0, 200)] * 32 + [(0, 0)] * 64 + [(300, 310)] * 32 + [(100, 200)] * 40
    s = make(spans, 400, 4, 1, 64, BF16)
    out, lse = run(s)
    check(run_bwd(s, out, lse), gradient(s, out, lse), s)


@pytest.mark.parametrize("layout", ["head_major", "part"])
@pytest.mark.parametrize("D", [64, 128])
def test_layouts(layout, D):
    spans, n = packed([150, 151])
    s = make(spans, n, 6, 2, D, FP16, layout=layout)
    out, lse = run(s)
    gen = torch.Generator(device="cuda").manual_seed(1)
    into = [matrix(gen, n, heads, D, FP16, layout) for heads in (6, 2, 2)]
    check(run_bwd(s, out, lse, into=into), gradient(s, out, lse), s)


@pytest.mark.parametrize("D", [64, 128])
def test_sharp_and_flat_scores(D):
    spans, n = packed([400])
    for size, scale in ((30.0, None), (1e-3, None), (1.0, 2.5)):
        s = make(spans, n, 4, 2, D, BF16, size=size)
        out, lse = run(s, scale)
        check(run_bwd(s, out, lse, scale), gradient(s, out, lse, scale), s)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", [1e-4, 3e-6, 0.0, 2000.0])
def test_small_and_large_gradients_in_fp16(size, D):
    spans, n = packed([300, 70], pad=2)
    s = make(spans, n + 2, 4, 2, D, FP16)
    s["dout"].mul_(size)
    out, lse = run(s)
    want = gradient(s, out, lse)
    got = run_bwd(s, out, lse)
    fits = {m: (v, torch.where(v.abs() < 60000, t, math.inf)) for m, (v, t) in want.items()}
    check(got, fits, s)


def test_against_differences():
    """The kernels' gradient along a direction against central differences of the attention in 64 bits."""
    spans, n = packed([50, 41], chunk=3)
    s = make(spans, n, 4, 2, 64, BF16)
    out, lse = run(s)
    got, want = run_bwd(s, out, lse), gradient(s, out, lse)
    gen = torch.Generator(device="cuda").manual_seed(5)

    def loss(t):
        total = 0.0
        for h in range(4):
            x = t["q"][:, h] @ t["k"][:, h // 2].t() / 8
            p = torch.softmax(x.masked_fill(~s["seen"], -math.inf), 1)
            total += float((p @ t["v"][:, h // 2] * s["dout"][:, h].double()).sum())
        return total

    for name in "qkv":
        way = torch.randn(s[name].shape, generator=gen, device="cuda", dtype=torch.float64)
        sides = []
        for sign in (1e-4, -1e-4):
            t = {m: s[m].double() for m in "qkv"}
            t[name] = t[name] + sign * way
            sides.append(loss(t))
        found = float((got["d" + name].double() * way).sum())
        # out's rounding moves delta by u L, which the tolerance has once already
        room = 2 * float((want["d" + name][1] * way.abs()).sum())
        assert abs(found - (sides[0] - sides[1]) / 2e-4) <= room


def test_equal_calls_give_equal_bits():
    spans, n = packed([1, 200, 33, 128, 257, 5], pad=40)
    for D in (64, 128):
        s = make(spans, n + 40, 8, 2, D, BF16)
        out, lse = run(s)
        a, b = run_bwd(s, out, lse, workspace_fill=0), run_bwd(s, out, lse)
        assert all(torch.equal(a[m], b[m]) for m in a)


def test_streams_and_graphs():
    spans, n = packed([300, 500])
    s = make(spans, n, 8, 2, 64, BF16)
    out, lse = run(s)
    want = run_bwd(s, out, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = {"d" + m: torch.empty_like(s[m]) for m in "qkv"}
    work = torch.empty(fdp.span_attention_workspace_bytes(n, n, 8, 2, 64, backward=True),
                       dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda: fdp.op_span_attention_bwd(s["q"], s["k"], s["v"], s["spans"], out, lse,  # noqa: E731
                                             s["dout"], *got.values(), workspace=work, err=err)
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert all(torch.equal(got[m], want[m]) for m in got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(2):
        for x in got.values():
            x.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[m], want[m]) for m in got)
    assert int(err) == 0


def test_no_queries_and_no_keys():
    s = make([], 50, 4, 2, 64, BF16)
    out, lse = run(s)
    got = run_bwd(s, out, lse)
    assert not bool(got["dk"].any()) and not bool(got["dv"].any())
    s = make([(0, 5)] * 9, 0, 4, 2, 64, BF16)
    out, lse = run(s)
    assert not bool(run_bwd(s, out, lse)["dq"].any())


def test_tensors_that_are_refused():
    spans, n = packed([40])
    s = make(spans, n, 4, 2, 64, BF16)
    out, lse = run(s)
    work = torch.empty(fdp.span_attention_workspace_bytes(n, n, 4, 2, 64, backward=True),
                       dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(**kw):
        d = dict(q=s["q"], k=s["k"], v=s["v"], spans=s["spans"], out=out, lse=lse, dout=s["dout"],
                 dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]), dv=torch.empty_like(s["v"]),
                 workspace=work, err=err)
        d.update(kw)
        fdp.op_span_attention_bwd(**d)

    call()
    for bad in (dict(dout=s["dout"].cpu()), dict(dout=s["dout"].half()), dict(dq=s["k"]),
                dict(dk=s["q"]), dict(dv=torch.empty(n, 2, 64, device="cuda")), dict(lse=lse[:2]),
                dict(out=out[:3]), dict(workspace=None), dict(workspace=work[:-1])):
        with pytest.raises((TypeError, ValueError)):
            call(**bad)
    for bad in (dict(scale=-1.0), dict(err=None), dict(dk=torch.empty(n, 1, 64, dtype=BF16,
                                                                     device="cuda").expand(-1, 2, -1))):
        with pytest.raises(fdp.FdError):
            call(**bad)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [0, 150, 299])
def test_largest_gradient_of_many_tiles(at, D):
    """300 row tiles, one of which has gradients 2000 times as large (fp16's are scaled by the largest)."""
    spans, n = packed([30, 20])
    s = make(spans, n, 300, 300, D, FP16)
    s["dout"].mul_(0.01)
    s["dout"][:, at].mul_(2000)
    out, lse = run(s)
    check(run_bwd(s, out, lse), gradient(s, out, lse), s)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=str)
def test_queries_that_see_one_key(dtype, D):
    """Their probability is 1 whatever the score: dq is zero, dk has nothing of them, dv their dout."""
    T = 300
    one = [(t, t + 1) for t in range(T)]
    s = make(one, T, 6, 2, D, dtype)
    out, lse = run(s)
    got = run_bwd(s, out, lse)
    assert not bool(got["dq"].any()) and not bool(got["dk"].any())
    check(got, gradient(s, out, lse), s)
    # among others: every third query sees one key, another one sees those and more
    mixed = [(t, t + 1) if t % 3 else (max(0, t - 40), t + 1) for t in range(T)]
    s = make(mixed, T, 6, 2, D, dtype)
    out, lse = run(s)
    got = run_bwd(s, out, lse)
    check(got, gradient(s, out, lse), s)
    alone = [t for t in range(T) if t % 3] + [0]
    assert not bool(got["dq"][alone].any()) and bool(got["dq"][3:][::3].any(-1).all())
