"""Rotary positions (fd_op_rotary) against the formula in 64 bits.

Tolerance, element by element: the phase reaches sincospif as a 24-bit fraction of half a turn
(2^-25 of at most pi: 1e-7 rad each way), sine and cosine are within 2 ulp (2.4e-7), the products
and their sum round three times (1.8e-7): |error| <= 8e-7 m (|a| + |b|), and one rounding to the
output's type (2^-8 bf16, 2^-11 fp16, 2^-24 fp32 of the value; fp16 2^-25 at least)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def frequencies(dims, base=10000.0, scaling="none", factor=1.0, trained=1, fast=32.0, slow=1.0):
    out = []
    for d in dims:
        b = base * factor ** (d / (d - 2)) if scaling == "base" and d > 2 else base
        row = []
        for i in range(d // 2):
            f = b ** (-2.0 * i / d)
            if scaling == "linear":
                f /= factor
            if scaling == "blend":
                n = trained * f / (2 * math.pi)
                g = min(1.0, max(0.0, (n - slow) / (fast - slow)))
                f = g * f + (1 - g) * f / factor
            row.append(f)
        out.append(row)
    return out


def reference(x, pos, freqs, rot, layout, amplitude=1.0, backward=False):
    """(values, bound on |a| + |b|) in 64 bits; pos [T][axes]."""
    x = x.double()
    angle = torch.cat([pos[:, a:a + 1].double() * torch.tensor(f, dtype=torch.float64,
                                                               device=x.device)
                       for a, f in enumerate(freqs)], 1)[:, None]
    c, s = amplitude * angle.cos(), amplitude * angle.sin() * (-1 if backward else 1)
    y, size = x.clone(), torch.zeros_like(x)
    i = torch.arange(rot // 2, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + rot // 2)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia] = size[..., ib] = abs(amplitude) * (a.abs() + b.abs())
    return y, size


def check(got, want, size, phase=0.0):
    tol = (8e-7 + phase) * size + ROUND[got.dtype] * want.abs()
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), float(((got.double() - want).abs() - tol).max())


CASES = [
    # tokens, q heads, k heads, head_dim, axis dims, layout, dtype
    (1, 16, 4, 64, (24, 20, 20), "interleaved", torch.bfloat16),
    (1, 1, 0, 2, (2,), "half", torch.float32),
    (7, 3, 1, 64, (64,), "half", torch.float16),
    (129, 5, 2, 128, (64,), "half", torch.bfloat16),
    (33, 8, 8, 96, (30, 2), "interleaved", torch.bfloat16),
    (20, 4, 3, 80, (20,), "half", torch.float32),
    (20, 4, 3, 80, (20,), "interleaved", torch.float16),
    (11, 2, 1, 7, (2, 2), "half", torch.float16),
    (11, 2, 1, 5, (4,), "interleaved", torch.float32),
    (50, 2, 2, 256, (96, 96, 64), "half", torch.float32),
    (3, 1, 1, 255, (2,), "half", torch.bfloat16),
    (1563, 16, 4, 64, (24, 20, 20), "interleaved", torch.bfloat16),
    (4099, 32, 8, 128, (128,), "half", torch.float16),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("backward", [False, True])
def test_turns_queries_and_keys(case, backward):
    T, qh, kh, D, dims, layout, dtype = case
    gen = torch.Generator(device="cuda").manual_seed(T + D)
    q = torch.randn(T, qh, D, generator=gen, device="cuda").to(dtype)
    k = torch.randn(T, kh, D, generator=gen, device="cuda").to(dtype) if kh else None
    pos = torch.randint(-1000, 100000, (T, len(dims)), generator=gen, device="cuda").int()
    plan = fdp.Rotary(D, sum(dims), layout, dims)
    q_out = torch.full_like(q, math.nan)
    k_out = torch.full_like(k, math.nan) if kh else None
    fdp.op_rotary(plan, pos, q, q_out, k, k_out, backward=backward)
    for x, y in ((q, q_out),) + (((k, k_out),) if kh else ()):
        want, size = reference(x, pos, frequencies(dims), sum(dims), layout, backward=backward)
        check(y, want, size)
        assert torch.equal(y[..., sum(dims):], x[..., sum(dims):])


@pytest.mark.parametrize("scaling", ["linear", "base", "blend"])
def test_scaled_frequencies(scaling):
    T, D, dims = 257, 64, (24, 20, 20) if scaling != "blend" else (64,)
    q = torch.randn(T, 4, D, device="cuda")
    pos = torch.randint(0, 1000000, (T, len(dims)), device="cuda").int()
    plan = fdp.Rotary(D, D, "half", dims, base=500.0, scaling=scaling, factor=4.0,
                      trained_len=4096, fast_turns=32.0, slow_turns=1.0, amplitude=1.125)
    out = torch.empty_like(q)
    fdp.op_rotary(plan, pos, q, out)
    freqs = frequencies(dims, 500.0, scaling, 4.0, 4096)
    want, size = reference(q, pos, freqs, D, "half", 1.125)
    # 64-bit pow may differ by an ulp between libraries: 2^-52 of up to 10^6 rad on each side
    check(out, want, size, phase=2 * 1e6 * 2.0 ** -52)


def test_positions_at_the_ends_of_int32():
    pos = torch.tensor([[2 ** 31 - 1], [-2 ** 31], [2 ** 30 + 1], [16777217], [0]],
                       dtype=torch.int32, device="cuda")
    q = torch.randn(5, 2, 32, device="cuda")
    out = torch.empty_like(q)
    fdp.op_rotary(fdp.Rotary(32), pos, q, out)
    want, size = reference(q, pos, frequencies((32,)), 32, "interleaved")
    # the reference's own angle, 2^31 rad in 64 bits, and the plan's frequency: 2^31 2^-52 each
    check(out, want, size, phase=2 * 2.0 ** -21)
    assert torch.equal(out[4], q[4])


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("rot", [32, 64])
def test_in_place_and_strided(layout, rot):
    T, D = 37, 64
    fused = torch.randn(T, 8, D, device="cuda").bfloat16()  # queries, keys and values together
    pos = torch.arange(T, device="cuda").int()
    plan = fdp.Rotary(D, rot, layout)
    before = fused.clone()
    fdp.op_rotary(plan, pos, fused[:, :5], fused[:, :5], fused[:, 5:7], fused[:, 5:7])
    want, size = reference(before[:, :7], pos[:, None], frequencies((rot,)), rot, layout)
    check(fused[:, :7], want, size)
    assert torch.equal(fused[:, 7], before[:, 7])
    # head-major memory, an odd offset into it, and tokens backwards in the output
    flat = torch.randn(3 * T * D + 1, device="cuda").bfloat16()[1:]
    x = flat.view(3, T, D).transpose(0, 1)
    y = torch.empty(T, 3, D, dtype=torch.bfloat16, device="cuda")
    fdp.op_rotary(plan, pos, x, y)
    want, size = reference(x, pos[:, None], frequencies((rot,)), rot, layout)
    check(y, want, size)


def test_gradient_is_the_difference_quotient():
    """<dy, R(x + h d) - R(x)> / h = <R^T dy, d>: the map is linear, so the quotient is exact up to
    rounding, 16 terms of at most 2^-22 |dy| |d| each side over n elements."""
    T, D = 64, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, d, dy = (torch.randn(T, 4, D, generator=gen, device="cuda") for _ in range(3))
    pos = torch.randint(0, 50000, (T, 3), generator=gen, device="cuda").int()
    plan = fdp.Rotary(D, D, "interleaved", (24, 20, 20), amplitude=0.75)
    y0, y1, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    fdp.op_rotary(plan, pos, x, y0)
    fdp.op_rotary(plan, pos, x + d, y1)
    fdp.op_rotary(plan, pos, dy, dx, backward=True)
    left = float((dy.double() * (y1.double() - y0.double())).sum())
    right = float((dx.double() * d.double()).sum())
    assert abs(left - right) <= 16 * 2.0 ** -22 * float(dy.norm()) * float((x.norm() + d.norm()))


def test_gradient_undoes_the_turn():
    x = torch.randn(100, 6, 128, device="cuda")
    pos = torch.randint(0, 10000, (100,), device="cuda").int()
    plan = fdp.Rotary(128, 96, "half")
    y, z = torch.empty_like(x), torch.empty_like(x)
    fdp.op_rotary(plan, pos, x, y)
    fdp.op_rotary(plan, pos, y, z, backward=True)
    a = x[..., :48].abs() + x[..., 48:96].abs()
    assert bool(((z - x)[..., :96].abs() <= 4 * 8e-7 * torch.cat([a, a], -1) + 1e-7).all())


def test_agrees_with_the_decoders_table():
    """The temporal band of the decoder's own 3D-RoPE: cos and sin of a chunk's table."""
    t, frames = 40000, 4
    table = torch.empty(frames, 12, 2, device="cuda")
    fdp.op_rope_table(t, frames, 10000.0, table)
    x = torch.zeros(frames, 1, 64, device="cuda")
    x[..., 0:24:2] = 1.0
    pos = torch.zeros(frames, 3, dtype=torch.int32, device="cuda")
    pos[:, 0] = torch.arange(frames) + t * frames
    out = torch.empty_like(x)
    fdp.op_rotary(fdp.Rotary(64, 64, "interleaved", (24, 20, 20)), pos, x, out)
    assert float((out[:, 0, :24].reshape(frames, 12, 2) - table).abs().max()) <= 8e-7 + 2.0 ** -24


def test_nothing_to_do():
    plan = fdp.Rotary(64)
    q = torch.empty(0, 4, 64, device="cuda")
    fdp.op_rotary(plan, torch.empty(0, dtype=torch.int32, device="cuda"), q, q)
    q = torch.empty(3, 0, 64, device="cuda")
    fdp.op_rotary(plan, torch.zeros(3, dtype=torch.int32, device="cuda"), q, q)


def test_another_stream():
    x = torch.randn(2000, 16, 64, device="cuda").bfloat16()
    pos = torch.arange(2000, device="cuda").int()
    plan = fdp.Rotary(64)
    a, b = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fdp.op_rotary(plan, pos, x, a, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    fdp.op_rotary(plan, pos, x, b)
    assert torch.equal(a, b)
