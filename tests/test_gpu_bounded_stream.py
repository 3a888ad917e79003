"""A whole bounded stream (rotation, eviction, attention with gathered weights) step by step
against 64-bit attention over the entries that the cache should hold.

The reference follows the library in which slots it gives up (the choice depends on the last
bits of the weights) and checks the choice by the library's own weights; what the slots then
hold, the outputs and the weights are its own. Tolerances as for the attention alone: P and the
output are rounded to bf16, 2^-8 each of sum p |v| and of the output; the rotated keys and queries are
bf16 too, on both sides from the same 64-bit rotation up to one rounding, which moves a score by at
most 2^-8 of sum |q k| scale: probabilities by exp of that."""
import math
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("n,whole", [(1, False), (3, False), (24, True), (40, False)])
def test_steps_against_the_reference(n, whole):
    S, H, G, D, C, steps = 2, 8, 2, 64, 96, 9 if n > 1 else 110
    gen = torch.Generator(device="cuda").manual_seed(n)
    plan = fdp.Rotary(D, 32, "half")
    b = BoundedStream(S, H, G, D, C, plan=plan, sinks=2, recent=n, decay=0.9)
    weight = torch.zeros(S, G, C, dtype=torch.float64, device="cuda")
    keys = torch.zeros(S, G, C, D, dtype=torch.float64, device="cuda")
    values = torch.zeros_like(keys)
    where = torch.full((S, G, C), -1, dtype=torch.int64, device="cuda")
    for step in range(steps):
        q = torch.randn(S, n, H, D, generator=gen, device="cuda").bfloat16()
        k = torch.randn(S, n, G, D, generator=gen, device="cuda").bfloat16()
        v = torch.randn(S, n, G, D, generator=gen, device="cuda").bfloat16()
        pos = (step * n + torch.arange(n, device="cuda").int()).expand(S, n).contiguous()
        before = b.cache.weight.clone()
        out = b.step(q, k, v, pos, whole_chunk=whole).double()
        slots = b._buffers[("slots", (S, G, n))].long()

        # the slots: first n by (class, weight, index)
        kept = torch.where(where < 0, 0,
                           torch.where((where < 2) | (where >= step * n - n), 2, 1))
        for s in range(S):
            for g in range(G):
                order = sorted((int(kept[s, g, j]), float(before[s, g, j]) if kept[s, g, j] else 0.0,
                                j) for j in range(C))
                assert sorted(j for _, _, j in order[:n]) == slots[s, g].tolist()

        # rotation in 64 bits, rounded once
        def turn(x):
            half = 16
            f = 10000.0 ** (-torch.arange(half, device="cuda").double() / half)
            a = pos.double()[..., None, None] * f
            x = x.double()
            lo, hi = x[..., :half], x[..., half:2 * half]
            y = torch.cat([lo * a.cos() - hi * a.sin(), lo * a.sin() + hi * a.cos(), x[..., 32:]], -1)
            return y.bfloat16().double()
        q, k, v = turn(q), turn(k).transpose(1, 2), v.double().transpose(1, 2)
        rows = slots[..., None].expand(S, G, n, D)
        keys.scatter_(2, rows, k)
        values.scatter_(2, rows, v)
        where.scatter_(2, slots, pos.long()[:, None].expand(S, G, n))
        weight.scatter_(2, slots, 0.0)
        assert torch.equal(b.cache.pos.long(), where)
        x = q.view(S, n, G, H // G, D)
        score = torch.einsum("sngid,sgjd->sngij", x, keys) / 8
        size = float((torch.einsum("sngid,sgjd->sngij", x.abs(), keys.abs()) / 8).max())
        last = pos[:, -1:].expand(S, n) if whole else pos
        seen = (where[:, None, :, None] >= 0) & (where[:, None, :, None] <=
                                                 last[:, :, None, None, None])
        p = torch.nan_to_num(torch.softmax(score.masked_fill(~seen, -math.inf), -1))
        want = torch.einsum("sngij,sgjd->sngid", p, values).reshape(S, n, H, D)
        bound = torch.einsum("sngij,sgjd->sngid", p, values.abs()).reshape(S, n, H, D)
        # one bf16 unit of q or k where the two rotations round apart (2^-8 of half the terms at
        # most a handful; counted as all of them)
        eps = math.expm1(2 * 2.0 ** -8 * size)
        assert bool(((out - want).abs() <= (2.0 ** -8 + eps) * bound + 2.0 ** -8 * want.abs()).all())
        weight = 0.9 * weight + p.sum((1, 3))
        # the library's own weights go on from here, so errors do not pile up over the steps
        assert bool(((b.cache.weight.double() - weight).abs() <= (eps + 1e-5) * weight.clamp_min(1e-6)
                     + eps * 10).all())
        weight = b.cache.weight.double()
    b.check()


def test_compact_to_a_smaller_stream():
    S, H, G, D = 2, 4, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(0)
    b = BoundedStream(S, H, G, D, 500, sinks=3, recent=20)
    pos = torch.arange(300, dtype=torch.int32, device="cuda").expand(S, 300).contiguous()
    b.step(torch.randn(S, 300, H, D, generator=gen, device="cuda").bfloat16(),
           torch.randn(S, 300, G, D, generator=gen, device="cuda").bfloat16(),
           torch.randn(S, 300, G, D, generator=gen, device="cuda").bfloat16(), pos)
    now = torch.full((S,), 300, dtype=torch.int32, device="cuda")
    small = b.compact(100, now)
    assert small.filled == 100 and bool((small.cache.pos >= 0).all())
    for s in range(S):
        for g in range(G):
            kept = small.cache.pos[s, g].tolist()
            assert kept == sorted(kept) and kept[:3] == [0, 1, 2] and kept[-20:] == list(range(280, 300))
            rest = set(range(3, 280)) - set(kept)
            w = b.cache.weight[s, g]
            assert max(float(w[j]) for j in rest) <= min(float(w[j]) for j in kept[3:-20])
    wide = b.compact(400, now)  # more than there is: everything, and empty slots
    assert wide.filled == 300 and torch.equal(wide.cache.pos[..., :300], b.cache.pos[..., :300])
    assert bool((wide.cache.pos[..., 300:] == -1).all())
    small.check()


def test_steps_in_a_graph():
    """Steps of a full cache, captured once and replayed, against steps that are not."""
    S, H, G, D, C = 2, 8, 2, 64, 64

    def fresh():
        b = BoundedStream(S, H, G, D, C, plan=fdp.Rotary(D), sinks=1, recent=8)
        gen = torch.Generator(device="cuda").manual_seed(4)
        pos = torch.arange(C, dtype=torch.int32, device="cuda").expand(S, C).contiguous()
        x = [torch.randn(S, C, h, D, generator=gen, device="cuda").bfloat16() for h in (H, G, G)]
        b.step(*x, pos)
        return b, gen
    plain, gen = fresh()
    graphed, _ = fresh()
    q, k, v = (torch.empty(S, 1, h, D, dtype=torch.bfloat16, device="cuda") for h in (H, G, G))
    pos = torch.full((S, 1), C, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # loads the kernels, on a cache that is not used after
        fresh()[0].step(q.zero_(), k.zero_(), v.zero_(), pos)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = graphed.step(q, k, v, pos)
        pos.add_(1)
    for _ in range(20):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        want = plain.step(q, k, v, pos.clone())
        graph.replay()
        assert torch.equal(got, want) and torch.equal(graphed.cache.pos, plain.cache.pos)
        assert torch.equal(graphed.cache.weight, plain.cache.weight)
    plain.check(), graphed.check()


def test_example_runs():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "bounded_stream.py"),
                        "--tokens", "1200", "--capacity", "320"], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    window, used = (float(line.split(": ")[1].split()[0]) for line in r.stdout.strip().splitlines())
    assert used < 0.5 * window


def test_steps_on_another_stream_and_of_no_tokens():
    """Everything runs on the current stream, a chunk's common position too."""
    S, H, G, D, C = 2, 8, 2, 64, 64
    gen = torch.Generator(device="cuda").manual_seed(6)
    x = [[torch.randn(S, n, h, D, generator=gen, device="cuda").bfloat16() for h in (H, G, G)]
         for n in (48, 16, 0, 40)]
    pos, start = [], 0
    for q, _, _ in x:
        pos.append((start + torch.arange(q.shape[1], device="cuda").int()).expand(S, -1).contiguous())
        start += q.shape[1]

    def run():
        b = BoundedStream(S, H, G, D, C, plan=fdp.Rotary(D), sinks=1, recent=8)
        return [b.step(*t, p, whole_chunk=True).clone() for t, p in zip(x, pos)], b
    want, a = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(5_000_000)  # the current stream of the calls is behind the default one
        got, b = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(s, t) for s, t in zip(got, want)) and want[2].shape[1] == 0
    assert torch.equal(a.cache.weight, b.cache.weight) and torch.equal(a.cache.pos, b.cache.pos)
    a.check(), b.check()
