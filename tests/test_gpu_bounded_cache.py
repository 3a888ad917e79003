"""The bounded cache on the GPU: attention that gathers weights against plain 64-bit attention,
eviction against a sorted list.

Tolerances of the attention. With A the largest sum of |q_d k_d| scale of any (query, slot), a
score's error in fp32 is at most (D + 8) 2^-23 A (products are exact, sums and the scale round,
tensor cores truncate), and maximum, sum, logarithm and exponential add 2^-18 together; so a
probability is relatively off by eps = 2 (D + 8) 2^-23 A + 2^-18 (numerator and sum). Weights:
eps times the gathered sum, and 2^-22 of the decayed weight and the sum. Output: P is rounded to
the cache's type (u = 2^-8 or 2^-11; fp16 2^-25 of the row's largest at least) and the result
once more: (u + eps) sum p |v| + u |out|."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
NAN = math.nan


def make_cache(S, G, C, D, dtype, gen, layout="dense", empty=0.0, now=None):
    """A cache after many replacements: scattered positions below `now`, NaN in empty slots."""
    def rows():
        if layout == "dense":
            x = torch.empty(S, G, C, D, dtype=dtype, device="cuda")
        elif layout == "slot_major":  # [S][C][G][D]
            x = torch.empty(S, C, G, D, dtype=dtype, device="cuda").transpose(1, 2)
        else:  # rows in a wider buffer, the first elements of it not ours
            x = torch.empty(S, G, C + 3, D + 8, dtype=dtype, device="cuda")[:, :, 2:C + 2, 8:]
        return x.copy_(torch.randn(S, G, C, D, generator=gen, device="cuda"))
    now = 2 * C + 5 if now is None else now
    pos = torch.rand(S, G, now, generator=gen, device="cuda").argsort(-1)[..., :C].int()
    gone = torch.rand(S, G, C, generator=gen, device="cuda") < empty
    pos = torch.where(gone, -1 - pos, pos).contiguous()
    k, v = rows(), rows()
    k.masked_fill_(gone[..., None], NAN)
    v.masked_fill_(gone[..., None], NAN)
    weight = torch.rand(S, G, C, generator=gen, device="cuda")
    return fdp.Cache(k, v, pos, weight)


def reference(cache, used, q, q_pos, scale, decay, dtype):
    """(out, its tolerance, weight_out, its tolerance) in 64 bits."""
    S, n, H, D = q.shape
    G = cache.groups
    per = H // G
    out = torch.zeros(S, n, H, D, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    weight = decay * cache.weight.double()
    wtol = 2.0 ** -22 * weight.abs()
    u = U[dtype]
    for s in range(S):
        for g in range(G):
            pos = cache.pos[s, g, :used]
            at = torch.nonzero(pos >= 0)[:, 0]
            if not at.numel() or not n:
                continue
            k, v = cache.k[s, g, at].double(), cache.v[s, g, at].double()
            x = q[s, :, g * per:(g + 1) * per].double()                     # [n][per][D]
            score = torch.einsum("thd,jd->thj", x, k) * scale
            size = float((torch.einsum("thd,jd->thj", x.abs(), k.abs()) * abs(scale)).max())
            seen = (pos[at][None] <= q_pos[s][:, None])[:, None]
            score = score.masked_fill(~seen, -math.inf)
            p = torch.nan_to_num(torch.softmax(score, -1))
            eps = 2 * (D + 8) * 2.0 ** -23 * size + 2.0 ** -18
            o = p @ v
            out[s, :, g * per:(g + 1) * per] = o
            low = 2.0 ** -25 * p.amax(-1, keepdim=True) * v.abs().sum(0) \
                if dtype == torch.float16 else 0.0
            tol[s, :, g * per:(g + 1) * per] = (u + eps) * (p @ v.abs()) + u * o.abs() + low
            total = p.sum((0, 1))
            weight[s, g].index_add_(0, at, total)
            wtol[s, g].index_add_(0, at, (eps + 2.0 ** -22) * total)
    return out, tol + 1e-30, weight, wtol + 1e-30


def attend(cache, q, q_pos, used=None, scale=None, decay=1.0, weights=True, in_place=False):
    S, n, H, D = q.shape
    out = torch.full((S, n, H, D), NAN, dtype=q.dtype, device="cuda")
    w = None
    if weights:
        w = cache.weight if in_place else torch.full_like(cache.weight, NAN)
    work = torch.full((fdp.cache_attention_workspace_bytes(cache, H, n, used) // 4 + 1,), NAN,
                      device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fdp.op_cache_attention(cache, q, q_pos, out, weight_out=w, used=used, scale=scale,
                           decay=decay, workspace=work, err=err)
    assert int(err) == 0
    return out, w


def check(cache, q, q_pos, used=None, scale=None, decay=1.0, in_place=False):
    D = q.shape[-1]
    n = cache.capacity if used is None else used
    want, tol, weight, wtol = reference(cache, n, q, q_pos, D ** -0.5 if scale is None else scale,
                                        decay, q.dtype)
    out, w = attend(cache, q, q_pos, used, scale, decay, in_place=in_place)
    over = (out.double() - want).abs() - tol
    assert not bool((~(over <= 0)).any()), ("out", float(over.nan_to_num(1e9).max()))
    over = (w.double() - weight).abs()[..., :n] - wtol[..., :n]
    assert not bool((~(over <= 0)).any()), ("weight", float(over.nan_to_num(1e9).max()))
    return out, w


CASES = [
    # streams, queries, heads, groups, D, capacity, used, dtype, layout, mask, empty
    (1, 1, 1, 1, 64, 1, 1, torch.bfloat16, "dense", "chunk", 0.0),
    (1, 1, 16, 4, 64, 1000, 999, torch.bfloat16, "dense", "causal", 0.0),
    (3, 1, 6, 2, 128, 257, 257, torch.float16, "slot_major", "causal", 0.3),
    (2, 1, 8, 1, 64, 6240, 6240, torch.bfloat16, "wide", "chunk", 0.02),
    (2, 3, 10, 2, 128, 4099, 4099, torch.bfloat16, "dense", "causal", 0.0),
    (5, 2, 7, 7, 64, 130, 127, torch.float16, "dense", "causal", 0.5),
    (1, 5, 3, 1, 128, 33, 31, torch.float16, "wide", "early", 0.0),
    (2, 17, 8, 2, 64, 300, 300, torch.bfloat16, "slot_major", "causal", 0.1),
    (1, 33, 16, 4, 64, 1561, 1561, torch.bfloat16, "dense", "chunk", 0.0),
    (2, 40, 12, 4, 128, 700, 641, torch.float16, "wide", "early", 0.2),
    (1, 257, 16, 4, 64, 6240, 6240, torch.bfloat16, "dense", "causal", 0.01),
    (2, 131, 10, 2, 128, 1030, 1025, torch.float16, "slot_major", "causal", 0.05),
    (1, 1560, 16, 4, 64, 3120, 3120, torch.bfloat16, "dense", "chunk", 0.0),
    (1, 300, 1, 1, 128, 129, 128, torch.bfloat16, "dense", "early", 0.0),
    (1, 128, 1, 1, 64, 20000, 20000, torch.float16, "dense", "causal", 0.0),
    (3, 50, 24, 3, 64, 97, 90, torch.float16, "dense", "causal", 0.9),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_attention_and_weights(case):
    S, n, H, G, D, C, used, dtype, layout, mask, empty = case
    gen = torch.Generator(device="cuda").manual_seed(S * 1000 + n * 10 + C)
    cache = make_cache(S, G, C, D, dtype, gen, layout, empty)
    q = (1.5 * torch.randn(S, n, H, D, generator=gen, device="cuda")).to(dtype)
    now = 2 * C + 5
    q_pos = torch.full((S, n), now - 1, dtype=torch.int32, device="cuda")
    if mask == "causal":
        q_pos = torch.randint(0, now, (S, n), generator=gen, device="cuda").int()
    elif mask == "early":  # some queries come before every entry, one at a negative position
        q_pos = torch.randint(-2, 6, (S, n), generator=gen, device="cuda").int()
    check(cache, q, q_pos, used, decay=0.75)


@pytest.mark.parametrize("n", [1, 200])
def test_rows_and_caches_that_see_nothing(n):
    """Empty streams give zeros and leave the decayed weights, and do not disturb the others."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    cache = make_cache(3, 2, 300, 64, torch.bfloat16, gen)
    cache.pos[1] = -7
    cache.k[1] = NAN
    cache.v[1] = math.inf
    cache.pos[2, 1] = 2 ** 31 - 1
    q = torch.randn(3, n, 4, 64, generator=gen, device="cuda").bfloat16()
    q_pos = torch.full((3, n), 2 ** 31 - 2, dtype=torch.int32, device="cuda")
    out, w = check(cache, q, q_pos, decay=0.5)
    assert not bool(out[1].any()) and torch.equal(w[1], 0.5 * cache.weight[1])
    assert not bool(out[2, :, 2:].any())


@pytest.mark.parametrize("n", [1, 150])
def test_weights_in_place_or_not_gathered(n):
    gen = torch.Generator(device="cuda").manual_seed(6)
    cache = make_cache(2, 2, 500, 128, torch.float16, gen)
    q = torch.randn(2, n, 4, 128, generator=gen, device="cuda").half()
    q_pos = torch.full((2, n), 2000, dtype=torch.int32, device="cuda")
    out, w = check(cache, q, q_pos, decay=0.9)
    before = cache.weight.clone()
    alone, _ = attend(cache, q, q_pos, weights=False)
    assert torch.equal(alone, out) and torch.equal(cache.weight, before)
    again, same = attend(cache, q, q_pos, decay=0.9, in_place=True)
    assert torch.equal(again, out) and torch.equal(same, w)


@pytest.mark.parametrize("n", [1, 100])
def test_large_scores_and_equal_bits(n):
    """Scores in the hundreds (one slot takes almost all), equal calls equal bits."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    cache = make_cache(1, 2, 1500, 64, torch.bfloat16, gen)
    q = (40 * torch.randn(1, n, 8, 64, generator=gen, device="cuda")).bfloat16()
    q_pos = torch.randint(0, 3000, (1, n), generator=gen, device="cuda").int()
    for scale in (1.0, 0.01):
        a, wa = check(cache, q, q_pos, scale=scale)
        b, wb = attend(cache, q, q_pos, scale=scale)
        assert torch.equal(a, b) and torch.equal(wa, wb)


@pytest.mark.parametrize("D,n", [(64, 700), (128, 700), (128, 1)])
def test_many_calls_in_a_row_give_equal_bits(D, n):
    """Calls back to back over a long cache with empty slots: a copy that is used before it has
    landed, or overwritten before it has been used, shows as other bits sooner or later."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    cache = make_cache(2, 4, 8191, D, torch.float16, gen, empty=0.01)
    q = torch.randn(2, n, 16, D, generator=gen, device="cuda").half()
    q_pos = torch.randint(8000, 16387, (2, n), generator=gen, device="cuda").int()
    want, weight = attend(cache, q, q_pos)
    out, w = torch.empty_like(want), torch.empty_like(weight)
    work = torch.empty(fdp.cache_attention_workspace_bytes(cache, 16, n), dtype=torch.uint8,
                       device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    differ = torch.zeros(1, dtype=torch.int64, device="cuda")
    for _ in range(60):
        for _ in range(4):
            fdp.op_cache_attention(cache, q, q_pos, out, weight_out=w, workspace=work, err=err)
        differ += (out != want).sum() + (w != weight).sum()
    assert int(err) == 0 and int(differ) == 0


@pytest.mark.parametrize("n", [1, 40])
def test_strided_queries_and_outputs(n):
    gen = torch.Generator(device="cuda").manual_seed(8)
    cache = make_cache(2, 2, 200, 64, torch.bfloat16, gen)
    fused = torch.randn(n, 2, 8, 64, generator=gen, device="cuda").bfloat16()
    q = fused[:, :, 2:6].transpose(0, 1)
    q_pos = torch.full((2, n), 500, dtype=torch.int32, device="cuda")
    want, tol, _, _ = reference(cache, 200, q, q_pos, 0.125, 1.0, torch.bfloat16)
    buf = torch.full((2, 4, n, 72), 3.0, dtype=torch.bfloat16, device="cuda")
    out = buf[..., :64].transpose(1, 2)
    work = torch.empty(fdp.cache_attention_workspace_bytes(cache, 4, n), dtype=torch.uint8,
                       device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    fdp.op_cache_attention(cache, q, q_pos, out, workspace=work, err=err)
    assert bool(((out.double() - want).abs() <= tol).all())
    assert bool((buf[..., 64:] == 3.0).all())


@pytest.mark.parametrize("heads", [1, 3, 16])
@pytest.mark.parametrize("order", ["ascending", "descending", "mixed", "steps"])
@pytest.mark.parametrize("D", [64, 128])
def test_masks_over_a_cache_in_order(heads, order, D):
    """Rows of one tile that see different parts of it: entries in the order of their positions,
    queries at positions in the cache, before it and after it."""
    n, C = 150, 500
    gen = torch.Generator(device="cuda").manual_seed(heads)
    cache = make_cache(2, 1, C, D, torch.bfloat16, gen, empty=0.02)
    cache.pos.copy_(torch.where(cache.pos < 0, -1, torch.arange(C, device="cuda").int()))
    t = torch.arange(C - 100, C - 100 + n, device="cuda").int()
    t = {"ascending": t, "descending": t.flip(0), "steps": t // 7 * 7,
         "mixed": torch.randint(-4, C + 4, (n,), generator=gen, device="cuda").int()}[order]
    q = torch.randn(2, n, heads, D, generator=gen, device="cuda").bfloat16()
    check(cache, q, torch.stack([t, t - 250]).contiguous())


def test_no_queries_no_slots():
    gen = torch.Generator(device="cuda").manual_seed(9)
    cache = make_cache(2, 2, 300, 64, torch.bfloat16, gen)
    q = torch.randn(2, 3, 4, 64, device="cuda").bfloat16()
    q_pos = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    out, w = attend(cache, q, q_pos, used=0)
    assert not bool(out.any()) and bool(w.isnan().all())
    out, w = attend(cache, q[:, :0], q_pos[:, :0].contiguous(), decay=0.25)
    assert torch.equal(w, 0.25 * cache.weight)
    empty = fdp.Cache(cache.k[:0], cache.v[:0], cache.pos[:0], cache.weight[:0])
    attend(empty, q[:0], q_pos[:0])


def test_offsets_past_32_bits():
    """Streams 2^31 + 4096 elements apart (offsets past 2^32 bytes and past 2^31 elements)."""
    apart = 2 ** 31 + 4096
    flat_k = torch.empty(apart + 2 * 64 * 64, dtype=torch.bfloat16, device="cuda")
    flat_v = torch.empty_like(flat_k)
    gen = torch.Generator(device="cuda").manual_seed(10)
    view = [x.as_strided((2, 2, 64, 64), (apart, 64 * 64, 64, 1)) for x in (flat_k, flat_v)]
    for x in view:
        x.copy_(torch.randn(2, 2, 64, 64, generator=gen, device="cuda"))
    pos = torch.arange(64, device="cuda").int().expand(2, 2, 64).contiguous()
    cache = fdp.Cache(*view, pos, torch.rand(2, 2, 64, generator=gen, device="cuda"))
    for n in (1, 64):
        q = torch.randn(2, n, 4, 64, generator=gen, device="cuda").bfloat16()
        check(cache, q, torch.full((2, n), 50, dtype=torch.int32, device="cuda"))
    check_insert(cache, 5, 2, 8, gen)


def test_another_stream():
    gen = torch.Generator(device="cuda").manual_seed(11)
    cache = make_cache(2, 4, 3000, 64, torch.bfloat16, gen)
    for n in (1, 300):
        q = torch.randn(2, n, 16, 64, generator=gen, device="cuda").bfloat16()
        q_pos = torch.full((2, n), 9000, dtype=torch.int32, device="cuda")
        want, w = attend(cache, q, q_pos)
        work = torch.empty(fdp.cache_attention_workspace_bytes(cache, 16, n), dtype=torch.uint8,
                           device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, w2 = torch.empty_like(q), torch.empty_like(w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        fdp.op_cache_attention(cache, q, q_pos, out, weight_out=w2, workspace=work, err=err,
                               stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want) and torch.equal(w, w2)


# ------------------------------------------------------------------------------ eviction
def ranked(pos, weight, newest, sinks, recent):
    """Slots in the order in which they are given up, and their classes."""
    def value(w):
        return (1, 0.0) if math.isnan(w) else (0, w + 0.0 if w else 0.0)
    keys = []
    for j, (p, w) in enumerate(zip(pos, weight)):
        if p < 0:
            keys.append((0, (0, 0.0), j))
        else:
            keys.append((2 if p < sinks or p >= newest - recent else 1, value(w), j))
    return sorted(keys)


def check_insert(cache, n, sinks, recent, gen, in_place=False, first=None):
    S, G, C, D = cache.streams, cache.groups, cache.capacity, cache.head_dim
    k_new = torch.randn(S, n, G, D, generator=gen, device="cuda").to(cache.dtype)
    v_new = torch.randn(S, n, G, D, generator=gen, device="cuda").to(cache.dtype)
    first = 3 * C if first is None else first
    new_pos = (first + torch.arange(n, device="cuda").int()).expand(S, n).contiguous()
    slots = torch.full((S, G, n), -9, dtype=torch.int32, device="cuda")
    k, v = cache.k.clone(), cache.v.clone()
    pos, weight = cache.pos.clone(), cache.weight.clone()
    pos_out = cache.pos if in_place else torch.full_like(pos, -9)
    weight_out = cache.weight if in_place else torch.full_like(weight, NAN)
    fdp.op_cache_insert(cache, k_new, v_new, new_pos, slots, pos_out=pos_out,
                        weight_out=weight_out, sinks=sinks, recent=recent)
    want = torch.zeros_like(slots).cpu()
    pl, wl = pos.cpu().tolist(), weight.cpu().tolist()
    for s in range(S):
        for g in range(G):
            order = ranked(pl[s][g], wl[s][g], first, sinks, recent)
            want[s, g] = torch.tensor(sorted(j for _, _, j in order[:n]), dtype=torch.int32)
    want = want.cuda()
    assert torch.equal(slots, want)
    at = want.long()
    pos.scatter_(-1, at, new_pos[:, None].expand(S, G, n))
    weight.scatter_(-1, at, 0.0)
    rows = at[..., None].expand(S, G, n, D)
    k.scatter_(2, rows, k_new.transpose(1, 2))
    v.scatter_(2, rows, v_new.transpose(1, 2))
    assert torch.equal(pos_out, pos)
    for got, exp in ((weight_out, weight), (cache.k, k), (cache.v, v)):
        bits = torch.int32 if got.dtype == torch.float32 else torch.int16
        assert torch.equal(got.contiguous().view(bits), exp.contiguous().view(bits))


INSERTS = [
    # streams, groups, D, capacity, new, dtype, layout, sinks, recent, empty
    (1, 1, 64, 1, 1, torch.bfloat16, "dense", 0, 0, 0.0),
    (1, 1, 64, 1, 1, torch.bfloat16, "dense", 5, 9, 1.0),
    (8, 4, 64, 6240, 1, torch.bfloat16, "dense", 4, 256, 0.0),
    (2, 3, 128, 1000, 1, torch.float16, "slot_major", 0, 0, 0.1),
    (2, 3, 128, 1000, 7, torch.float16, "wide", 4, 100, 0.0),
    (1, 4, 64, 6240, 1560, torch.bfloat16, "dense", 4, 1560, 0.03),
    (3, 2, 64, 97, 97, torch.float16, "dense", 4, 10, 0.2),
    (1, 2, 64, 33, 32, torch.bfloat16, "dense", 1000, 10, 0.0),
    (1, 1, 64, 20011, 3001, torch.bfloat16, "dense", 16, 10 ** 6, 0.0),
    (80, 1, 64, 1025, 100, torch.bfloat16, "dense", 0, 300, 0.5),
    (77, 1, 64, 33000, 129, torch.bfloat16, "dense", 2, 5000, 0.01),
    (77, 1, 64, 30000, 1, torch.bfloat16, "dense", 2, 5000, 0.0),
    (80, 1, 64, 8192, 8192, torch.bfloat16, "dense", 2, 5000, 0.0),
    (2, 1, 64, 65537, 20000, torch.float16, "dense", 2, 5000, 0.0),
]


@pytest.mark.parametrize("case", INSERTS, ids=str)
@pytest.mark.parametrize("in_place", [False, True])
def test_insert_takes_the_least_used_slots(case, in_place):
    S, G, D, C, n, dtype, layout, sinks, recent, empty = case
    gen = torch.Generator(device="cuda").manual_seed(C + n)
    cache = make_cache(S, G, C, D, dtype, gen, layout, empty)
    check_insert(cache, n, sinks, recent, gen, in_place)


@pytest.mark.parametrize("n", [1, 2, 50, 299])
def test_ties_and_odd_weights(n):
    """Equal weights, both zeros, negative ones, infinities and NaN; empty slots whose weights
    are NaN; a stream whose entries are all protected."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    cache = make_cache(3, 4, 300, 64, torch.bfloat16, gen, empty=0.1)
    values = torch.tensor([0.0, -0.0, 1.0, 1.0, -1.0, math.inf, -math.inf, NAN, 1e-40, -1e-40],
                          device="cuda")
    cache.weight.copy_(values[torch.randint(0, 10, cache.weight.shape, generator=gen,
                                            device="cuda")])
    cache.weight[1] = 0.5
    cache.weight[cache.pos < 0] = NAN
    cache.pos[2] = cache.pos[2].clamp_min(890)
    check_insert(cache, n, 3, 10, gen)


def test_insert_nothing_copies_the_rest():
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = make_cache(2, 2, 77, 64, torch.bfloat16, gen, empty=0.2)
    check_insert(cache, 0, 3, 10, gen)


COMPACTS = [
    # streams, groups, D, capacity, used, keep, dtype, layout, sinks, recent, empty
    (1, 1, 64, 1, 1, 1, torch.bfloat16, "dense", 0, 0, 0.0),
    (1, 4, 64, 6240, 6240, 1560, torch.bfloat16, "dense", 4, 256, 0.0),
    (2, 3, 128, 1000, 990, 990, torch.float16, "wide", 4, 100, 0.1),
    (2, 3, 128, 1000, 990, 980, torch.float16, "slot_major", 4, 100, 0.3),
    (2, 2, 64, 500, 400, 300, torch.bfloat16, "dense", 0, 0, 0.6),
    (2, 1, 64, 50, 50, 1, torch.bfloat16, "dense", 0, 0, 1.0),
    (1, 2, 128, 20011, 20011, 4099, torch.float16, "dense", 16, 1000, 0.01),
    (80, 1, 64, 33000, 33000, 129, torch.bfloat16, "dense", 2, 50, 0.01),
    (80, 1, 64, 8192, 8192, 8100, torch.bfloat16, "dense", 2, 50, 0.0),
    (80, 1, 64, 8193, 8193, 8000, torch.float16, "dense", 2, 50, 0.001),
    (1, 1, 64, 100000, 100000, 50000, torch.bfloat16, "dense", 2, 50, 0.001),
]


@pytest.mark.parametrize("case", COMPACTS, ids=str)
@pytest.mark.parametrize("ties", [False, True])
def test_compact_keeps_the_most_used(case, ties):
    S, G, D, C, used, keep, dtype, layout, sinks, recent, empty = case
    gen = torch.Generator(device="cuda").manual_seed(C + keep)
    src = make_cache(S, G, C, D, dtype, gen, layout, empty)
    if ties:
        src.weight.copy_((src.weight * 4).floor())
    now = torch.full((S,), 2 * C + 5, dtype=torch.int32, device="cuda")
    dst = fdp.Cache(torch.full((S, G, keep, D), NAN, dtype=dtype, device="cuda"),
                    torch.full((S, G, keep, D), NAN, dtype=dtype, device="cuda"),
                    torch.full((S, G, keep), -9, dtype=torch.int32, device="cuda"),
                    torch.full((S, G, keep), NAN, device="cuda"))
    came = torch.full((S, G, keep), -9, dtype=torch.int32, device="cuda")
    fdp.op_cache_compact(src, dst, now, came, used=used, sinks=sinks, recent=recent)
    want = torch.full((S, G, keep), -1, dtype=torch.int32)
    pl, wl = src.pos.cpu().tolist(), src.weight.cpu().tolist()
    for s in range(S):
        for g in range(G):
            order = ranked(pl[s][g][:used], wl[s][g][:used], 2 * C + 5, sinks, recent)
            kept = sorted(j for c, _, j in order[used - keep:] if c)
            want[s, g, :len(kept)] = torch.tensor(kept, dtype=torch.int32)
    want = want.cuda()
    assert torch.equal(came, want)
    at, none = want.clamp_min(0).long(), want < 0
    rows = at[..., None].expand(S, G, keep, D)
    assert torch.equal(dst.pos, torch.where(none, -1, src.pos.gather(-1, at)))
    assert torch.equal(dst.weight, torch.where(none, 0.0, src.weight.gather(-1, at)))
    for x, y in ((src.k, dst.k), (src.v, dst.v)):
        assert torch.equal(y, torch.where(none[..., None], 0.0, x.gather(2, rows)))


def test_the_binding_refuses_what_the_library_would_misread():
    gen = torch.Generator(device="cuda").manual_seed(12)
    c = make_cache(2, 2, 100, 64, torch.bfloat16, gen)
    q = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    q_pos = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    work = torch.empty(fdp.cache_attention_workspace_bytes(c, 4, 1), dtype=torch.uint8,
                       device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def attention(**kw):
        d = dict(q=q, q_pos=q_pos, out=torch.empty_like(q), workspace=work, err=err)
        d.update(kw)
        fdp.op_cache_attention(c, d.pop("q"), d.pop("q_pos"), d.pop("out"), **d)

    attention()
    for bad in (dict(q=q.half()), dict(q=q[:1]), dict(q=q[..., :32]), dict(q_pos=q_pos.long()),
                dict(out=q[:, :0]), dict(workspace=None), dict(workspace=work[:16]),
                dict(weight_out=c.weight[:1]), dict(q=q.cpu()), dict(q_pos=q_pos.cpu())):
        with pytest.raises((TypeError, ValueError)):
            attention(**bad)
    with pytest.raises(fdp.FdError):
        attention(used=101)
    with pytest.raises(TypeError):
        fdp.Cache(c.k.float(), c.v.float(), c.pos, c.weight)
    with pytest.raises(ValueError):
        fdp.Cache(c.k, c.v.transpose(1, 2).contiguous().transpose(1, 2), c.pos, c.weight)
    with pytest.raises(ValueError):
        fdp.Cache(c.k, c.v, c.pos[:, :1], c.weight)
    new = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(2, 2, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        fdp.op_cache_insert(c, new, new, q_pos, slots[:, :1])
    with pytest.raises(TypeError):
        fdp.op_cache_insert(c, new.half(), new, q_pos, slots)
    x = torch.zeros(3, 2, 64, device="cuda")
    with pytest.raises(ValueError):
        fdp.op_rotary(fdp.Rotary(64), torch.zeros(4, dtype=torch.int32, device="cuda"), x, x)
    with pytest.raises(TypeError):
        fdp.op_rotary(fdp.Rotary(64), torch.zeros(3, device="cuda"), x, x)
    with pytest.raises(ValueError):
        fdp.op_rotary(fdp.Rotary(32), torch.zeros(3, dtype=torch.int32, device="cuda"), x, x)
