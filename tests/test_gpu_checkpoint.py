"""Checkpoints in 8 bits on the GPU: codes and exponents against the format's definition in whole
numbers, restored values against the codes (both exact, so nothing has a tolerance)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

TYPES = [torch.bfloat16, torch.float16, torch.float32]
STEP_MOST = {torch.float32: 3.4028234663852886e38, torch.bfloat16: 3.3895313892515355e38,
             torch.float16: 65504.0}


def by_definition(x):
    """(codes, exponents' bytes) of x [rows][width], block by block."""
    rows, width = x.shape
    codes = torch.zeros(rows, width, dtype=torch.int8)
    exps = torch.zeros(rows, -(-width // 32), dtype=torch.uint8)
    for r, row in enumerate(x.double().cpu().tolist()):
        for j in range(0, width, 32):
            block = row[j:j + 32]
            if not all(math.isfinite(v) for v in block):
                exps[r, j // 32] = 255
                continue
            top, e = max(abs(v) for v in block), -126
            while top > 127 * 2.0 ** e:
                e += 1
            most = 63 if e == 122 else 127
            exps[r, j // 32] = e + 127
            codes[r, j:j + 32] = torch.tensor(
                [max(-most, min(most, round(math.ldexp(v, -e)))) for v in block])
    return codes, exps


def values(codes, exps, dtype):
    """What codes stand for, in dtype."""
    of = torch.arange(codes.shape[1]) // 32
    x = torch.ldexp(codes.double(), exps.long()[:, of] - 127)
    x[exps[:, of] == 255] = math.nan
    if dtype == torch.float16:
        x = torch.where(x.abs() == 65536, x.clamp(-65504, 65504), x)
    return x.to(dtype)


def activations(rows, width, dtype, seed, kind="spread"):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, width, generator=gen)
    if kind == "spread":
        x *= torch.exp(3 * torch.randn(rows, 1, generator=gen))
        x *= torch.exp(2 * torch.randn(width, generator=gen))
    elif kind == "ties":  # the first of a block is 127 steps: codes of half steps go to the even one
        x = (torch.randint(-254, 255, (rows, width), generator=gen) / 2).float()
        x[:, ::32] = 127
    elif kind == "edges":  # the largest magnitude at the borders of 127 steps
        x = torch.rand(rows, width, generator=gen)
        x[:, ::32] = torch.tensor([1.0, 127 / 128, 1 - 2.0 ** -8, 127 / 64, 2.0])[
            torch.arange(rows) % 5, None]
    return x.to(dtype)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0)) \
        and torch.equal(a.isnan(), b.isnan())


def kept_of(x):
    kept = fdp.Checkpoint8.empty(*x.shape)
    kept.codes.fill_(99), kept.exps.fill_(7)
    fdp.op_checkpoint_save(x, kept)
    return kept


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width,kind", [
    (1, 8, "spread"), (3, 24, "spread"), (5, 32, "edges"), (7, 40, "ties"), (33, 64, "spread"),
    (130, 136, "spread"), (2, 8200, "spread"), (129, 1024, "ties"), (10, 1536, "edges")])
def test_codes_are_those_of_the_definition(dtype, rows, width, kind):
    x = activations(rows, width, dtype, rows + width, kind)
    kept = kept_of(x.cuda())
    codes, exps = by_definition(x)
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.exps.cpu(), exps)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,width", [(1, 8), (3, 40), (127, 136), (128, 128), (129, 264),
                                        (300, 1032)])
@pytest.mark.parametrize("transposed", [False, True])
def test_restored_values(dtype, rows, width, transposed):
    kept = kept_of(activations(rows, width, dtype, rows * width).cuda())
    want = values(kept.codes.cpu(), kept.exps.cpu(), dtype)
    if transposed:
        want = want.t()
    x = torch.full(want.shape, 3.0, dtype=dtype, device="cuda")
    fdp.op_checkpoint_load(kept, x, transposed=transposed)
    assert same(x.cpu(), want)
    # rows of a wider buffer, whose other elements stay; the transposed ones at an odd address
    lead, pad = (3, 5) if transposed else (8, 8)
    wide = torch.full((want.shape[0], want.shape[1] + lead + pad
                       + (0 if transposed else -want.shape[1] % 8)), 3.0, dtype=dtype, device="cuda")
    part = wide[:, lead:lead + want.shape[1]]
    fdp.op_checkpoint_load(kept, part, transposed=transposed)
    assert same(part.cpu(), want)
    part.fill_(3.0)
    assert bool((wide == 3.0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_special_values(dtype):
    x = torch.zeros(9, 64, dtype=dtype)
    most = STEP_MOST[dtype]
    x[1, 5] = math.nan
    x[2, 40] = -math.inf
    x[3, 0], x[3, 1], x[3, 33] = most, -most, most / 2
    x[4, 3] = torch.finfo(dtype).tiny
    x[5, 3] = torch.finfo(dtype).smallest_normal / 4 if dtype != torch.float16 else 6e-8
    x[6] = -0.0
    x[7, :32] = most
    x[8] = -1.0
    kept = kept_of(x.cuda())
    codes, exps = by_definition(x)
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.exps.cpu(), exps)
    back = torch.empty_like(x, device="cuda")
    fdp.op_checkpoint_load(kept, back)
    assert same(back.cpu(), values(codes, exps, dtype))
    finite = torch.isfinite(x).view(9, 2, 32).all(-1)[..., None].expand(9, 2, 32).reshape(9, 64)
    assert torch.equal(torch.isfinite(back.cpu()), finite)
    # half a step at most; but a whole one for a step of 2^122: 63.5 to 64 of them (2^128 is infinite)
    # stay at 63, and the largest finite number is less than 64
    step = torch.ldexp(torch.ones(9, 2, dtype=torch.float64), exps.long() - 127)
    most_off = torch.where(exps == 249, step, step / 2).repeat_interleave(32, 1)
    off = (back.cpu().double() - x.double()).abs()
    assert bool((off <= most_off)[finite].all())


def test_rows_with_strides_other_streams_and_graphs():
    x = activations(65, 200, torch.bfloat16, 1).cuda()
    wide = torch.zeros(65, 216, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:208] = x
    want = kept_of(x)
    got = kept_of(wide[:, 8:208])
    assert torch.equal(got.codes, want.codes) and torch.equal(got.exps, want.exps)
    every_other = torch.zeros(130, 200, dtype=torch.bfloat16, device="cuda")
    every_other[::2] = x
    got = kept_of(every_other[::2])
    assert torch.equal(got.codes, want.codes) and torch.equal(got.exps, want.exps)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, back = fdp.Checkpoint8.empty(65, 200), torch.empty(200, 65, device="cuda").bfloat16()
    with torch.cuda.stream(side):
        fdp.op_checkpoint_save(x, got)
        fdp.op_checkpoint_load(got, back, transposed=True)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    again = torch.empty_like(back)
    with torch.cuda.graph(g):
        fdp.op_checkpoint_save(x, got)
        fdp.op_checkpoint_load(got, again, transposed=True)
    x.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(again.float(), back.float() * 2)
    assert torch.equal(got.codes, want.codes) and torch.equal(got.exps[got.exps > 1],
                                                             want.exps[want.exps > 1] + 1)


def test_no_rows():
    kept = fdp.Checkpoint8.empty(0, 64)
    fdp.op_checkpoint_save(torch.empty(0, 64, device="cuda"), kept)
    fdp.op_checkpoint_load(kept, torch.empty(64, 0, device="cuda"), transposed=True)


def test_tensors_that_are_refused():
    kept = fdp.Checkpoint8.empty(4, 64)
    for bad in (torch.zeros(4, 64), torch.zeros(4, 72, device="cuda"),
                torch.zeros(64, 4, device="cuda").t(), torch.zeros(4, 64, device="cuda").double()):
        with pytest.raises((TypeError, ValueError)):
            fdp.op_checkpoint_save(bad, kept)
    with pytest.raises(fdp.FdError):
        fdp.op_checkpoint_save(torch.zeros(4, 65, device="cuda")[:, 1:], kept)  # not 16-byte aligned
    with pytest.raises(ValueError):
        fdp.op_checkpoint_load(kept, torch.zeros(4, 64, device="cuda"), transposed=True)
    with pytest.raises(ValueError):
        fdp.Checkpoint8(kept.codes, torch.zeros(4, 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        fdp.Checkpoint8(torch.zeros(4, 64, dtype=torch.int8), kept.exps)
