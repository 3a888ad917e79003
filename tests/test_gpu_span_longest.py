"""Attention in spans over the most keys that it takes, 2^24, with its gradient, against 64 bits.

Tolerances are those of test_gpu_span_attention.py and test_gpu_span_gradient.py, with the sums counted as they are
made: a part of `blocks` key blocks adds up in fp32 eight steps of 16 keys each (a tensor core's step truncates: 2^-23),
its exponentials by block (2^-24), and the parts once more. fp16: P and dS have the steps that the library's header
states, 2^-36 of the row's largest (forward), 2^-39 (P) and 2^-39 of dS's bound (gradient), where that is more."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
S, D, H, STEP = 1 << 24, 64, 2, 1 << 20
SPANS = [(0, S), (S - 1, S), (S // 2, S // 2 + 1000), (100, S - 77)]


def roundings(blocks):
    """The most on the way of a sum over the keys, 2^-24 each, with 100 parts of it at least (and fewer than 400)."""
    return 2 * 8 * (blocks // 100) + 400


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
def test_longest_keys_with_gradients(dtype):
    T, c, u = len(SPANS), D ** -0.5, U[dtype]
    gen = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    q, dout = randn(T, H, D).to(dtype), (1000 * randn(T, H, D)).to(dtype)
    k, v = (torch.empty(S, 1, D, dtype=dtype, device="cuda") for _ in range(2))
    for i in range(0, S, STEP):
        x = randn(STEP, 1, D)
        k[i:i + STEP] = x
        v[i:i + STEP] = 1 + 0.5 * x + 0.3 * randn(STEP, 1, D)
    spans = torch.tensor(SPANS, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(H, T, device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    need = max(fdp.span_attention_workspace_bytes(T, S, H, 1, D, backward=b) for b in (False, True))
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fdp.op_span_attention(q, k, v, spans, out, lse, workspace=work, err=err)
    fdp.op_span_attention_bwd(q, k, v, spans, out, lse, dout, dq, dk, dv, workspace=work, err=err)
    assert int(err) == 0

    sums = roundings(S // 128) * 2.0 ** -24
    fp16 = dtype == torch.float16
    rows = torch.arange(T, device="cuda").repeat_interleave(H)  # a row for each token and head
    q64, do = q.double().view(T * H, D), dout.double().view(T * H, D)
    o64, l64 = out.double().view(T * H, D), lse.t().double().reshape(T * H, 1)

    def chunks():
        for i in range(0, S, STEP):
            j = torch.arange(i, i + STEP, device="cuda")
            seen = (j >= spans[rows, :1]) & (j < spans[rows, 1:])
            x = (q64 @ k[i:i + STEP, 0].double().t()) * c
            yield i, seen, x.masked_fill(~seen, -math.inf), v[i:i + STEP, 0].double(), k[i:i + STEP, 0].double()

    # forward
    want_lse = torch.full((T * H, 1), -math.inf, dtype=torch.float64, device="cuda")
    size, most = 0.0, torch.full_like(want_lse, -math.inf)
    for i, seen, x, _, k64 in chunks():
        want_lse = torch.logaddexp(want_lse, torch.logsumexp(x, 1, keepdim=True))
        most = torch.maximum(most, x.amax(1, keepdim=True))
        size = max(size, float((q64.abs() @ k64.abs().t()).max()) * c)
    score = (D + 8) * 2.0 ** -23 * size
    off = (l64 - want_lse).abs()
    assert bool((off <= score + 2.0 ** -18 + sums + 2.0 ** -22 * (want_lse.abs() + size)).all())
    want, tol = torch.zeros_like(o64), torch.zeros_like(o64)
    for i, seen, x, v64, _ in chunks():
        p = torch.exp(x - want_lse)
        want += p @ v64
        tol += (u + 2 * score + 2.0 ** -18 + sums) * (p @ v64.abs())
        if fp16:
            tol += 2.0 ** -36 * torch.exp(most - want_lse) * (seen.double() @ v64.abs())
    off = (o64 - want).abs()
    assert bool((off <= tol + (u * want.abs()).clamp_min(2.0 ** -25 if fp16 else 0)).all()), float((off / tol).max())

    # gradient, from out and lse as they are
    e = 2 * score + 2.0 ** -18 + 2.0 ** -22 * float(l64.abs().max()) + (D + 8) * 2.0 ** -23
    delta, L = (do * o64).sum(1, keepdim=True), (do * o64).abs().sum(1, keepdim=True)
    bound = do.abs().sum(1, keepdim=True) * (2 * float(v.abs().max()) + o64.abs().amax(1, keepdim=True))
    floor = 2.0 ** -39 * bound if fp16 else torch.zeros_like(bound)
    one = (spans[rows, 1:] - spans[rows, :1]) == 1  # (P is 1, dS 0)
    want, tol = torch.zeros_like(o64), torch.zeros_like(o64)
    for i, seen, x, v64, k64 in chunks():
        p = torch.exp(x - l64)
        ds = (p * (do @ v64.t() - delta)).masked_fill(one, 0.0)
        ds_off = ((u + e) * p * (do.abs() @ v64.abs().t() + L) + floor * seen).masked_fill(one, 0.0)
        want += c * ds @ k64
        tol += c * (ds_off + sums * ds.abs()) @ k64.abs()
        key_off = ds_off if not fp16 else (u + e) * p * (do.abs() @ v64.abs().t() + L) + seen * (
            floor * seen).amax(0, keepdim=True)
        for name, got, value, room in (
                ("dk", dk, c * ds.t() @ q64, c * key_off.t() @ q64.abs()),
                ("dv", dv, p.t() @ do, ((u + e) * p + (2.0 ** -39 if fp16 else 0) * seen).t() @ do.abs())):
            off = (got[i:i + STEP, 0].double() - value).abs()
            room = room + (u * value.abs()).clamp_min(2.0 ** -25 if fp16 else 1e-30)
            assert bool((off <= room).all()), (name, i, float((off / room).max()))
            assert bool((got[i:i + STEP, 0] != 0).any())
    off = (dq.double().view(T * H, D) - want).abs()
    tol += (u * want.abs()).clamp_min(2.0 ** -25 if fp16 else 1e-30)
    assert bool((off <= tol).all()), float((off / tol).max())
    assert bool((tol[[0, 1, 6, 7]] < 0.5 * want[[0, 1, 6, 7]].abs().amax(1, keepdim=True)).all())
