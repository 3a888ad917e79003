"""A residual attention block's training pass through the operators together, against autograd of the same
formulas in 64 bits.

Tolerance, relative in the 2-norm: a rounding to bfloat16 is off by 2^-8 at most, and up to ten lie on a
gradient's way (u, qkv, P, out, b; db, dout, P or dS, dqkv, du); an activation in 8 bits is off by half a
step, 1/127 of the largest of 32 at most, which for normal values is 2.1 of their root mean square: half of
that on average, 0.5 % each for u, h and b. Together below 5.5 %."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300 import ResidualAttention  # noqa: E402

BOUND = 10 * 2.0 ** -8 + 3 * 0.005


def spans_of(lengths, pad):
    at, spans = 0, []
    for n in lengths:
        spans += [(at, at + p + 1) for p in range(n)]
        at += n
    return torch.tensor(spans + [(0, 0)] * pad, dtype=torch.int32, device="cuda")


def make(lengths, pad, width, heads, groups, head_dim, gate_tokens, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    T = sum(lengths) + pad
    w = {"w_qkv": randn((heads + 2 * groups) * head_dim, width) / math.sqrt(width),
         "w_out": randn(width, heads * head_dim) / math.sqrt(heads * head_dim),
         "post_gain": 1 + 0.1 * randn(width), "pre_gain": 1 + 0.1 * randn(width),
         "gate": 0.5 + 0.2 * randn(-(-T // gate_tokens), width)}
    w["w_qkv"], w["w_out"] = w["w_qkv"].bfloat16().float(), w["w_out"].bfloat16().float()
    x = {"h": randn(T, width), "u": randn(T, width).bfloat16(), "dy": randn(T, width),
         "du": randn(T, width).bfloat16()}
    return T, w, x, spans_of(lengths, pad)


def exact(w, x, spans, heads, groups, D, gate_tokens, scale):
    """Gradients of sum(y dy) + sum(u_next du) in 64 bits, by autograd."""
    p = {n: t.double().requires_grad_() for n, t in w.items()}
    h, u = (x[n].double().requires_grad_() for n in ("h", "u"))
    T = h.shape[0]
    qkv = u @ p["w_qkv"].t()
    q = qkv[:, :heads * D].view(T, heads, D)
    k = qkv[:, heads * D:(heads + groups) * D].view(T, groups, D).repeat_interleave(heads // groups, 1)
    v = qkv[:, (heads + groups) * D:].view(T, groups, D).repeat_interleave(heads // groups, 1)
    j = torch.arange(T, device="cuda")
    seen = (j >= spans[:, :1]) & (j < spans[:, 1:])
    s = torch.einsum("thd,jhd->htj", q, k) / math.sqrt(D)
    a = torch.softmax(s.masked_fill(~seen, -1e30), -1) * seen
    b = torch.einsum("htj,jhd->thd", a, v).reshape(T, -1) @ p["w_out"].t()
    n = b / torch.sqrt(b.square().mean(1, True) + 1e-6)
    gate = p["gate"][torch.arange(T, device="cuda") // gate_tokens]
    y = h + scale * gate * n * p["post_gain"]
    u_next = y / torch.sqrt(y.square().mean(1, True) + 1e-6) * p["pre_gain"]
    ((y * x["dy"].double()).sum() + (u_next * x["du"].double()).sum()).backward()
    return {"y": y, "u_next": u_next, "dh": h.grad, "du": u.grad, **{m: t.grad for m, t in p.items()}}


@pytest.mark.parametrize("lengths,pad,width,heads,groups,D,gate_tokens", [
    ([100, 27, 1], 0, 256, 4, 2, 64, 200), ([300, 200, 12], 8, 512, 6, 2, 128, 1),
    ([1000], 24, 1024, 16, 4, 64, 300)])
def test_training_pass(lengths, pad, width, heads, groups, D, gate_tokens):
    T, w, x, spans = make(lengths, pad, width, heads, groups, D, gate_tokens)
    block = ResidualAttention(T, width, heads, groups, D, w["w_qkv"], w["w_out"], w["post_gain"], w["pre_gain"],
                              w["gate"], gate_tokens, scale=0.7)
    want = exact(w, x, spans, heads, groups, D, gate_tokens, 0.7)
    for _ in range(2):  # the second pass finds the buffers of the first
        y, u_next = block.forward(x["h"], x["u"], spans)
        dh, du, g = block.backward(x["dy"], x["du"])
        block.check()
        got = {"y": y, "u_next": u_next, "dh": dh, "du": du, **g}
        for name, value in want.items():
            off = float((got[name].double() - value.detach()).norm() / value.detach().norm())
            assert off <= BOUND, (name, off)


def test_captured_pass():
    T, w, x, spans = make([90, 38], 0, 256, 4, 2, 64, 64)
    block = ResidualAttention(T, 256, 4, 2, 64, w["w_qkv"], w["w_out"], w["post_gain"], w["pre_gain"], w["gate"], 64)
    y, u_next = block.forward(x["h"], x["u"], spans)
    dh, du, g = block.backward(x["dy"], x["du"])
    want = [t.clone() for t in (y, u_next, dh, du, *g.values())]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, u_next = block.forward(x["h"], x["u"], spans)
        dh, du, g = block.backward(x["dy"], x["du"])
    for t in (y, dh, du, *g.values()):
        t.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, u_next, dh, du, *g.values()), want))
    block.check()


def test_sizes_that_are_refused():
    T, w, x, spans = make([90, 38], 0, 256, 4, 2, 64, 64)
    with pytest.raises(ValueError):
        ResidualAttention(T - 1, 256, 4, 2, 64, w["w_qkv"], w["w_out"], w["post_gain"], w["pre_gain"])


def test_example_runs_and_its_gradients():
    """Two blocks of the example: the gradient of its loss along the weights against central differences of the
    same stack in 64 bits (a loss of squares: the bound is that of two blocks, twice)."""
    import importlib.util
    import os
    import random
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "train_residual.py")
    spec = importlib.util.spec_from_file_location("train_residual", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    assert all(math.isfinite(v) for v in ex.main(["--steps", "3", "--tokens", "256"]))

    T, W, H, G, D = 128, 64, 2, 1, 64
    blocks, params = ex.make_blocks(T, W, H, G, D)
    x, target, spans = ex.batch(T, W, random.Random(0), torch.Generator(device="cuda").manual_seed(1))
    ex.train_step(blocks, params, x, target, spans)

    def loss(weights):
        h, u = x.double(), (x / x.square().mean(1, keepdim=True).sqrt()).bfloat16().double()
        j = torch.arange(T, device="cuda")
        seen = (j >= spans[:, :1]) & (j < spans[:, 1:])
        for p in weights:
            qkv = u @ p["w_qkv"].t()
            q, k, v = qkv[:, :H * D].view(T, H, D), qkv[:, H * D:H * D + D], qkv[:, H * D + D:]
            s = torch.einsum("thd,jd->htj", q, k) / math.sqrt(D)
            a = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
            b = torch.einsum("htj,jd->thd", a, v).reshape(T, -1) @ p["w_out"].t()
            h = h + p["gate"] * p["post_gain"] * b / torch.sqrt(b.square().mean(1, True) + 1e-6)
            u = h / torch.sqrt(h.square().mean(1, True) + 1e-6) * p["pre_gain"]
        return float((h - target.double()).square().mean())

    gen = torch.Generator(device="cuda").manual_seed(2)
    base = [{n: (t.bfloat16() if n.startswith("w_") else t).double() for n, t in p.items()} for p in params]
    for i, p in enumerate(params):
        for name, t in p.items():
            if float(t.grad.abs().max()) == 0.0:
                assert i == 1 and name == "pre_gain"  # the last block's next norm is not used
                continue
            # along the gradient itself, so that what is compared is not a small difference
            way = t.grad.double() / t.grad.double().norm() + 0.1 * torch.randn(
                t.shape, generator=gen, device="cuda", dtype=torch.float64) / math.sqrt(t.numel())
            sides = []
            for sign in (1e-4, -1e-4):
                moved = [dict(b) for b in base]
                moved[i][name] = moved[i][name] + sign * way
                sides.append(loss(moved))
            want = (sides[0] - sides[1]) / 2e-4
            found = float((t.grad.double() * way).sum())
            assert abs(found - want) <= 2 * BOUND * float(t.grad.double().norm()) * float(way.norm()), (i, name)


def test_inputs_that_are_refused():
    T, w, x, spans = make([90, 38], 0, 256, 4, 2, 64, 64)
    block = ResidualAttention(T, 256, 4, 2, 64, w["w_qkv"], w["w_out"], w["post_gain"], w["pre_gain"], w["gate"], 64)
    wide = torch.zeros(T, 512, dtype=torch.bfloat16, device="cuda")[:, :256]
    for u in (x["u"].float(), x["u"].half(), wide, x["u"][:-8], x["u"].cpu(), x["u"][:, :128].contiguous()):
        with pytest.raises((TypeError, ValueError)):
            block.forward(x["h"], u, spans)
    for s in (spans.long(), spans[:-8], spans.cpu(), spans.flatten()):
        with pytest.raises((TypeError, ValueError)):
            block.forward(x["h"], x["u"], s)
    for h in (x["h"].half(), x["h"][:, :128], x["h"].cpu()):
        with pytest.raises((TypeError, ValueError, RuntimeError)):  # (the library refuses a mix of types)
            block.forward(h, x["u"], spans)
    y, u_next = block.forward(x["h"], x["u"], spans)  # works as before
    want = block.forward(x["h"], x["u"], spans)
    assert torch.equal(y, want[0]) and torch.equal(u_next, want[1])
