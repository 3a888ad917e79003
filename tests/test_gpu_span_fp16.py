"""Attention in spans of keys in fp16 where its range could cost digits: few large probabilities beside many
small ones.

Tolerances are those of test_gpu_span_attention.py without what it allows fp16 for each key that a query sees:
probabilities keep half a step, 2^-11, down to 2^-25 of the row's largest."""
import math

import pytest
import torch
from test_gpu_span_attention import FP16, U, check, make, run

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
