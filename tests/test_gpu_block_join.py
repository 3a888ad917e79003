"""The join between two blocks and its gradient on the GPU against the formulas in 64 bits.

Tolerances. A sum over a row is at most 32 sums in a thread, 5 in a warp and 16 over warps, on rounded
squares: 64 roundings of 2^-24 with those of the mean, so a norm's factor is relatively off by less than
E = 2^-18 (a root halves it, root and division add less than is left). Everything else is a few
products: an expression is off by at most E times the same expression in magnitudes (every term's
absolute value, differences as sums), twice that where two norms or a sum over tokens (a block's rows
and the blocks' partial sums, fewer than 64 each in these tests) come in; an output's own rounding adds
U = half a step of its type relative to its value, and for fp16 half of its smallest step, 2^-24, where
the value is below 2^-14 (steps get no smaller there)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

E = 2.0 ** -18
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
F32 = torch.float32


def rounding(value, dtype):
    """Half a step of dtype at value."""
    return (U[dtype] * value.abs()).clamp_min(2.0 ** -25 if dtype == torch.float16 else 0.0)


EPS = 1e-6


def make(rows, width, dtype, stream, gate_tokens, post, pre, seed=0, wide=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def matrix(x, to):
        if not wide:
            return x.to(to).contiguous()
        y = torch.full((rows, width + 24), math.nan, dtype=to, device="cuda")[:, 8:8 + width]
        return y.copy_(x)

    s = {"h": matrix(2 * randn(rows, width), stream), "b": matrix(randn(rows, width), dtype),
         "dy": matrix(randn(rows, width), stream), "du": matrix(randn(rows, width), dtype),
         "post": 1 + 0.2 * randn(width) if post else None,
         "pre": 1 + 0.2 * randn(width) if pre else None,
         "gate": randn(-(-rows // gate_tokens), width) if gate_tokens else None,
         "gate_tokens": gate_tokens, "scale": 0.7}
    if not pre:
        s["du"] = None
    return s


def gates(s):
    """The gate of every token, 64 bits."""
    rows = s["b"].shape[0]
    if s["gate"] is None:
        return torch.ones(1, 1, dtype=torch.float64, device="cuda")
    return s["gate"].double()[torch.arange(rows, device="cuda") // s["gate_tokens"]]


def forward(s):
    """{name: (value, tolerance)} in 64 bits."""
    h, b = s["h"].double(), s["b"].double()
    r = 1 / torch.sqrt(b.square().mean(1) + EPS) if s["post"] is not None else torch.ones_like(b[:, 0])
    z = s["scale"] * gates(s) * b * r[:, None]
    if s["post"] is not None:
        z = z * s["post"].double()
    y = h + z
    y_off = 2 * E * z.abs() + 2.0 ** -24 * y.abs()
    found = {"y": (y, y_off + rounding(y, s["h"].dtype))}
    if s["post"] is not None:
        found["r_post"] = (r, E * r)
    if s["pre"] is not None:
        rp = 1 / torch.sqrt(y.square().mean(1) + EPS)
        # the mean of y^2 moves by twice mean(|y| y_off) at most (and its square), the root by half
        rp_off = E * rp + rp ** 3 * ((y.abs() + y_off) * y_off).mean(1)
        u = y * rp[:, None] * s["pre"].double()
        found["r_pre"] = (rp, rp_off)
        found["u"] = (u, rounding(u, s["b"].dtype) + E * u.abs()
                      + (y.abs() * rp_off[:, None] + 2 * y_off * rp[:, None]) * s["pre"].double().abs())
    return found


def run(s, **kw):
    rows, width = s["b"].shape
    out = {"y": torch.full_like(s["h"], 9.0)}
    if s["post"] is not None:
        out["r_post"] = torch.empty(rows, device="cuda")
    if s["pre"] is not None:
        out["r_pre"], out["u"] = torch.empty(rows, device="cuda"), torch.full_like(s["b"], 9.0)
    fdp.op_block_join(s["h"], s["b"], out["y"], out.get("u"), post_gain=s["post"], pre_gain=s["pre"],
                      gate=s["gate"], gate_tokens=s["gate_tokens"], scale=s["scale"], eps=EPS,
                      r_post=out.get("r_post"), r_pre=out.get("r_pre"), **kw)
    return out


def check(got, want):
    for name, (value, tol) in want.items():
        off = (got[name].double() - value).abs()
        bad = ~(off <= tol + 1e-30)
        assert not bool(bad.any()), (name, int(bad.sum()), float((off / (tol + 1e-30)).max()))


SIZES = [(1, 8), (5, 40), (3, 256), (6, 264), (130, 512), (7, 520), (2, 1024), (611, 1024),
         (3, 1536), (700, 2048), (9, 4096), (620, 4096), (5, 4104), (620, 8192), (1, 8192)]
FORMS = [(torch.bfloat16, F32), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16),
         (torch.float16, F32)]


@pytest.mark.parametrize("rows,width", SIZES)
@pytest.mark.parametrize("dtype,stream", FORMS, ids=str)
def test_forward(rows, width, dtype, stream):
    gate_tokens = [0, 1, 2, rows, 3 * rows][(rows + width // 8) % 5]
    s = make(rows, width, dtype, stream, gate_tokens, True, True, seed=width)
    kept = fdp.Checkpoint8.empty(rows, width), fdp.Checkpoint8.empty(rows, width)
    check(run(s, h_kept=kept[0], b_kept=kept[1]), forward(s))
    for k, x in zip(kept, (s["h"], s["b"])):  # as the call of its own gives them
        want = fdp.Checkpoint8.empty(rows, width)
        fdp.op_checkpoint_save(x, want)
        assert torch.equal(k.codes, want.codes) and torch.equal(k.exps, want.exps)


@pytest.mark.parametrize("post,pre,gate_tokens", [(0, 0, 0), (0, 0, 7), (1, 0, 0), (0, 1, 1),
                                                  (0, 1, 50)])
@pytest.mark.parametrize("wide", [False, True])
def test_forward_parts(post, pre, gate_tokens, wide):
    for width in (72, 1024):
        s = make(33, width, torch.bfloat16, F32, gate_tokens, post, pre, seed=gate_tokens, wide=wide)
        check(run(s), forward(s))


@pytest.mark.parametrize("width", [256, 1024, 4096])
def test_in_place(width):
    s = make(40, width, torch.bfloat16, F32, 1, True, True)
    want = run(s)
    fdp.op_block_join(s["h"], s["b"], s["h"], s["b"], post_gain=s["post"], pre_gain=s["pre"],
                      gate=s["gate"], gate_tokens=1, scale=s["scale"], eps=EPS)
    assert torch.equal(s["h"], want["y"]) and torch.equal(s["b"], want["u"])


# ------------------------------------------------------------------------------ gradient
def values(kept):
    of = torch.arange(kept.shape[1], device="cuda") // 32
    return torch.ldexp(kept.codes.double(), kept.exps.long()[:, of] - 127)


def gradient(s, r_post, r_pre, h, b):
    """{name: (value, tolerance)} in 64 bits: the tolerance is the formula in magnitudes."""
    one = torch.ones(1, dtype=torch.float64, device="cuda")
    gate, scale = gates(s), s["scale"]
    post = s["post"].double() if s["post"] is not None else one
    rp = r_post.double()[:, None] if s["post"] is not None else one
    n = b * rp
    q = scale * gate * post
    d = s["dy"].double() if s["dy"] is not None else torch.zeros_like(b)
    D = d.abs()
    found = {}
    if s["pre"] is not None:
        r, du = r_pre.double()[:, None], s["du"].double()
        m, M = (h + q * n) * r, (h.abs() + (q * n).abs()) * r
        g = du * s["pre"].double()
        found["d_pre"] = ((du * m).sum(0), 2 * E * (du.abs() * M).sum(0))
        d = d + r * (g - m * (g * m).mean(1, keepdim=True))
        D = D + r * (g.abs() + M * (g.abs() * M).mean(1, keepdim=True))
    found["dh"] = (d, 2 * E * D + rounding(d, s["h"].dtype))
    wn, WN = scale * d * n, scale * D * n.abs()
    if s["gate"] is not None:
        rows = torch.arange(len(b), device="cuda") // s["gate_tokens"]
        sums = torch.zeros(2, *s["gate"].shape, dtype=torch.float64, device="cuda")
        sums[0].index_add_(0, rows, wn * post)
        sums[1].index_add_(0, rows, WN * post.abs())
        found["d_gate"] = (sums[0], 4 * E * sums[1])
    if s["post"] is not None:
        found["d_post"] = ((wn * gate).sum(0), 4 * E * (WN * gate.abs()).sum(0))
        db = rp * (q * d - n * (q * d * n).mean(1, keepdim=True))
        DB = rp * (q.abs() * D + n.abs() * (q.abs() * D * n.abs()).mean(1, keepdim=True))
    else:
        db, DB = q * d, q.abs() * D
    found["db"] = (db, 4 * E * DB + rounding(db, s["b"].dtype))
    return found


def run_bwd(s, fwd, h, b, into=None):
    rows, width = s["b"].shape
    out = {"dh": torch.full_like(s["h"], 9.0), "db": torch.full_like(s["b"], 9.0)}
    for n in ("post", "pre", "gate"):
        if s[n] is not None:
            out["d_" + n] = torch.full_like(s[n], 9.0)
    if into is not None:
        out.update(into)
    work = torch.empty(fdp.block_join_bwd_workspace_bytes(rows, width), dtype=torch.uint8,
                       device="cuda").fill_(255)  # (NaN)
    fdp.op_block_join_bwd(s["dy"], s["du"], h, b, out["dh"], out["db"], post_gain=s["post"],
                          pre_gain=s["pre"], gate=s["gate"], gate_tokens=s["gate_tokens"],
                          scale=s["scale"], r_post=fwd.get("r_post"), r_pre=fwd.get("r_pre"),
                          d_post=out.get("d_post"), d_pre=out.get("d_pre"),
                          d_gate=out.get("d_gate"), workspace=work)
    return out


@pytest.mark.parametrize("rows,width", SIZES)
@pytest.mark.parametrize("dtype,stream", FORMS, ids=str)
def test_gradient(rows, width, dtype, stream):
    for gate_tokens in {0, 1, 3, max(1, rows // 3), rows, 2 * rows}:
        s = make(rows, width, dtype, stream, gate_tokens, True, True, seed=rows + gate_tokens)
        fwd = run(s)
        want = gradient(s, fwd["r_post"], fwd["r_pre"], s["h"].double(), s["b"].double())
        got = run_bwd(s, fwd, s["h"], s["b"])
        check(got, want)
        again = run_bwd(s, fwd, s["h"], s["b"])
        assert all(torch.equal(got[n], again[n]) for n in got)
        kept = [fdp.Checkpoint8.empty(rows, width) for _ in range(2)]
        for x, k in zip((s["h"], s["b"]), kept):
            fdp.op_checkpoint_save(x, k)
        want = gradient(s, fwd["r_post"], fwd["r_pre"], values(kept[0]), values(kept[1]))
        check(run_bwd(s, fwd, *kept), want)


@pytest.mark.parametrize("post,pre,gate_tokens", [(0, 0, 0), (0, 0, 7), (0, 0, 33), (1, 0, 0), (0, 1, 1),
                                                  (0, 1, 50), (1, 0, 33), (1, 1, 0)])
@pytest.mark.parametrize("wide", [False, True])
def test_gradient_parts(post, pre, gate_tokens, wide):
    for rows, width in ((33, 72), (33, 1024), (1, 8192)):
        s = make(rows, width, torch.bfloat16, F32, gate_tokens, post, pre, seed=gate_tokens, wide=wide)
        if pre and gate_tokens == 1:
            s["dy"] = None  # nothing comes back along the stream
        fwd = run(s)
        check(run_bwd(s, fwd, s["h"], s["b"]),
              gradient(s, fwd.get("r_post"), fwd.get("r_pre"), s["h"].double(), s["b"].double()))


def test_gradient_in_place_and_parts_not_wanted():
    s = make(70, 1024, torch.bfloat16, F32, 9, True, True)
    fwd = run(s)
    want = run_bwd(s, fwd, s["h"], s["b"])
    t = {n: x.clone() if isinstance(x, torch.Tensor) else x for n, x in s.items()}
    got = run_bwd(t, fwd, t["h"], t["b"], into={"dh": t["dy"], "db": t["du"]})
    assert all(torch.equal(got[n], want[n]) for n in want)
    got = run_bwd(s, fwd, s["h"], s["b"], into={"dh": None, "d_post": None, "d_pre": None,
                                                 "d_gate": None})
    assert torch.equal(got["db"], want["db"])


def test_gradient_against_differences():
    """The kernels' gradient along a direction against central differences of the formulas in 64 bits."""
    s = make(12, 64, torch.float16, F32, 5, True, True, seed=3)
    fwd = run(s)
    got = run_bwd(s, fwd, s["h"], s["b"])
    gen = torch.Generator(device="cuda").manual_seed(9)
    names = {"h": "dh", "b": "db", "post": "d_post", "pre": "d_pre", "gate": "d_gate"}
    for name, grad in names.items():
        way = torch.randn(s[name].shape, generator=gen, device="cuda", dtype=torch.float64)
        sides = []
        for sign in (1e-5, -1e-5):
            t = dict(s)
            t[name] = s[name].double() + sign * way
            found = {n: t[n].double() if isinstance(t[n], torch.Tensor) else t[n] for n in t}
            h, b, gate = found["h"], found["b"], found["gate"][torch.arange(12, device="cuda") // 5]
            y = h + s["scale"] * gate * found["post"] * b / torch.sqrt(b.square().mean(1, True) + EPS)
            u = y * found["pre"] / torch.sqrt(y.square().mean(1, True) + EPS)
            sides.append(float((y * s["dy"].double()).sum() + (u * s["du"].double()).sum()))
        want = (sides[0] - sides[1]) / 2e-5
        # differences: third derivatives times 1e-10, and 64-bit rounding / 1e-5; the gradient's own
        # rounding is U of each element at most
        size = float((got[grad].double().abs() * way.abs()).sum())
        assert abs(float((got[grad].double() * way).sum()) - want) <= (U[torch.float16] + 1e-5) * size


def test_no_tokens():
    s = make(0, 64, torch.bfloat16, F32, 0, True, True)
    fwd = run(s)
    got = run_bwd(s, fwd, s["h"], s["b"])
    assert not got["d_post"].any() and not got["d_pre"].any()


def test_streams_and_graphs():
    s = make(100, 1024, torch.bfloat16, F32, 30, True, True)
    fwd = run(s)
    want = run_bwd(s, fwd, s["h"], s["b"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f2 = run(s)
        got = run_bwd(s, f2, s["h"], s["b"])
    side.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f3 = run(s)
        got = run_bwd(s, f3, s["h"], s["b"])
    for _ in range(2):
        for x in got.values():
            x.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)


def test_tensors_that_are_refused():
    s = make(4, 64, torch.bfloat16, F32, 0, True, True)
    y, u = torch.empty_like(s["h"]), torch.empty_like(s["b"])

    def call(**kw):
        d = dict(h=s["h"], b=s["b"], y=y, u=u, post_gain=s["post"], pre_gain=s["pre"])
        d.update(kw)
        fdp.op_block_join(**d)

    call()
    for bad in (dict(h=s["h"].cpu()), dict(b=s["b"].cpu()), dict(y=y.half()), dict(u=u.half()),
                dict(u=None), dict(pre_gain=None), dict(post_gain=s["post"][:32]),
                dict(gate=s["post"][None], gate_tokens=0), dict(gate=s["post"][None], gate_tokens=1),
                dict(r_post=torch.empty(5, device="cuda")), dict(h=s["h"].t()),
                dict(b_kept=fdp.Checkpoint8.empty(4, 72)), dict(y=y[:, :32])):
        with pytest.raises((TypeError, ValueError)):
            call(**bad)
    for bad in (dict(eps=-1.0), dict(eps=math.nan), dict(scale=math.inf)):
        with pytest.raises(fdp.FdError):
            call(**bad)
    with pytest.raises(ValueError, match="workspace"):
        fdp.op_block_join_bwd(s["dy"], s["du"], s["h"], s["b"], y, u, post_gain=s["post"],
                              pre_gain=s["pre"], r_post=s["h"][:, 0].contiguous(),
                              r_pre=s["h"][:, 0].contiguous())


@pytest.mark.parametrize("rows", [3, 70, 700])
def test_one_gate_for_any_number_of_tokens(rows, monkeypatch):
    """The library's gate_rows past rows, up to the largest int (the binding cuts it to the tokens there are)."""
    s = make(rows, 256, torch.bfloat16, F32, rows, True, True)
    want = run(s)
    want_bwd = run_bwd(s, want, s["h"], s["b"])
    view = fdp._join_view

    def wide(*args):
        j = view(*args)
        j.gate_rows = 2 ** 31 - 1
        return j

    monkeypatch.setattr(fdp, "_join_view", wide)
    got = run(s)
    got_bwd = run_bwd(s, got, s["h"], s["b"])
    assert all(torch.equal(got[n], want[n]) for n in want)
    assert all(torch.equal(got_bwd[n], want_bwd[n]) for n in want_bwd)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_two_calls_at_once(dtype):
    """Two joins with their gradients on two streams, each with a workspace of its own, give what they give alone."""
    cases = [make(rows, 1024, dtype, F32, 7, True, True, seed=rows) for rows in (300, 2000)]
    alone = []
    for s in cases:
        fwd = run(s)
        alone.append((fwd, run_bwd(s, fwd, s["h"], s["b"])))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        found = []
        for s, stream in zip(cases, streams):
            with torch.cuda.stream(stream):
                fwd = run(s)
                found.append((fwd, run_bwd(s, fwd, s["h"], s["b"])))
        torch.cuda.synchronize()
        for got, want in zip(found, alone):
            for a, b in zip(got, want):
                assert all(torch.equal(a[n], b[n]) for n in b if isinstance(b[n], torch.Tensor))
