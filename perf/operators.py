"""The operators of a bounded key/value cache, in their plain form and through the library.

A stream that never ends keeps a cache of fixed size: each new token's query and key are turned
by its position (rotary), the new keys and values take the slots of the entries that attention
has used least (cache insert), attention over the cache adds every entry's weight to its running
total (cache attention), and a long first pass is cut down to the cache's size once (cache
compact). The sizes are those of the streaming decoder's presets (16 heads in 4 groups of head
dimension 64, 1560 tokens a chunk, a window of 4 chunks) and generic ones of long contexts.

`own` chooses what run() computes with: elementary torch operations in 32 bits, or the library.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
TURN_BITS = 64   # a position's phase is counted in 2^-64 turns, modulo one turn


def listed():
    return [
        # one new token in each of 8 streams of the 480p decoder: its time-row-column positions
        {"name": "rotary_token", "op": "rotary", "tokens": 8, "q_heads": 16, "k_heads": 4,
         "head_dim": 64, "rot_dim": 64, "layout": "interleaved", "axis_dims": "24,20,20",
         "scaling": "none", "dtype": "bf16", "backward": False, "most_pos": 100000},
        # gradient of a refinement chunk's queries and keys (4 x 1560 tokens) in training
        {"name": "rotary_chunk_grad", "op": "rotary", "tokens": 6240, "q_heads": 16, "k_heads": 4,
         "head_dim": 64, "rot_dim": 64, "layout": "interleaved", "axis_dims": "24,20,20",
         "scaling": "none", "dtype": "fp32", "backward": True, "most_pos": 100000},
        # a long context at once: half of each head turned, frequencies stretched 8 times
        {"name": "rotary_long", "op": "rotary", "tokens": 40001, "q_heads": 32, "k_heads": 8,
         "head_dim": 128, "rot_dim": 64, "layout": "half", "axis_dims": "64",
         "scaling": "blend", "dtype": "bf16", "backward": False, "most_pos": 1000000},
        # one token of each of 8 streams against a cache as large as the 480p window
        {"name": "attend_token", "op": "attend", "streams": 8, "queries": 1, "heads": 16,
         "groups": 4, "head_dim": 64, "used": 6240, "dtype": "bf16", "mask": "causal",
         "empty": 0.0, "fresh": False},
        # one token of 2 streams over a long, not quite full cache
        {"name": "attend_token_long", "op": "attend", "streams": 2, "queries": 1, "heads": 32,
         "groups": 8, "head_dim": 128, "used": 65537, "dtype": "bf16", "mask": "causal",
         "empty": 0.02, "fresh": False},
        # a chunk of the 480p decoder over its window, every token seeing the whole chunk
        {"name": "attend_chunk", "op": "attend", "streams": 1, "queries": 1560, "heads": 16,
         "groups": 4, "head_dim": 64, "used": 6240, "dtype": "bf16", "mask": "chunk",
         "empty": 0.0, "fresh": False},
        # a prompt's part of 2 streams, causal, odd sizes, fp16
        {"name": "attend_prompt", "op": "attend", "streams": 2, "queries": 2001, "heads": 32,
         "groups": 8, "head_dim": 128, "used": 8191, "dtype": "fp16", "mask": "causal",
         "empty": 0.01, "fresh": False},
        # the next token of 8 streams takes a slot of a full cache
        {"name": "insert_token", "op": "insert", "streams": 8, "groups": 4, "head_dim": 64,
         "capacity": 6240, "new": 1, "dtype": "bf16", "sinks": 4, "recent": 256, "empty": 0.0},
        # the next chunk of 8 streams takes a quarter of the slots
        {"name": "insert_chunk", "op": "insert", "streams": 8, "groups": 4, "head_dim": 64,
         "capacity": 6240, "new": 1560, "dtype": "bf16", "sinks": 4, "recent": 1560,
         "empty": 0.03},
        # the window of one 480p stream cut to one chunk's size
        {"name": "compact_window", "op": "compact", "streams": 1, "groups": 4, "head_dim": 64,
         "used": 6240, "keep": 1560, "dtype": "bf16", "sinks": 4, "recent": 256, "empty": 0.0},
        # long prompts of 4 streams cut to a small cache
        {"name": "compact_long", "op": "compact", "streams": 4, "groups": 8, "head_dim": 128,
         "used": 32771, "keep": 4099, "dtype": "fp16", "sinks": 16, "recent": 1000,
         "empty": 0.01},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["rotary", "attend", "attend", "insert", "compact"])
    if op == "rotary":
        head_dim = rng.choice([32, 64, 80, 96, 128])
        rot_dim = rng.choice([r for r in (16, 20, 32, 48, 64, 128) if r <= head_dim])
        axes = rng.choice([1, 1, 2, 3])
        first = rot_dim // axes // 2 * 2
        dims = [rot_dim - (axes - 1) * first] + [first] * (axes - 1)
        case = {"op": op, "tokens": _log(rng, 1, 40001), "q_heads": rng.randint(1, 32),
                "k_heads": rng.randint(1, 8), "head_dim": head_dim, "rot_dim": rot_dim,
                "layout": rng.choice(["interleaved", "half"]),
                "axis_dims": ",".join(str(d) for d in dims),
                "scaling": rng.choice(["none", "linear", "base", "blend"]),
                "dtype": rng.choice(["bf16", "fp16", "fp32"]),
                "backward": rng.random() < 0.4, "most_pos": _log(rng, 100, 1000000)}
        if case["dtype"] == "fp32":
            case["tokens"] = min(case["tokens"], 20000)
        return case
    groups = rng.choice([1, 2, 3, 4, 6, 8])
    head_dim = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "fp16"])
    empty = rng.choice([0.0, 0.01, 0.3])
    streams = _log(rng, 1, 16)
    if op == "attend":
        queries = rng.choice([1, 1, 2, 3, _log(rng, 4, 2001), _log(rng, 4, 2001)])
        per_group = rng.choice([1, 2, 3, 4, 5, 6, 8])
        used = max(queries, _log(rng, 1, 65537))
        # no more scores than the prompt's case, no more keys and values than the long token's
        while (streams * groups * per_group * queries * used > 10 ** 9
               or streams * groups * used * head_dim > 130 * 10 ** 6):
            if streams > 1:
                streams //= 2
            elif groups > 1:
                groups //= 2
            else:
                used = max(queries, used // 2)
        return {"op": op, "streams": streams, "queries": queries, "heads": groups * per_group,
                "groups": groups, "head_dim": head_dim, "used": used, "dtype": dtype,
                "mask": rng.choice(["causal", "chunk"]), "empty": empty,
                "fresh": streams > 1 and rng.random() < 0.3}
    if op == "insert":
        capacity = _log(rng, 16, 32771)
        new = rng.choice([1, 1, _log(rng, 1, max(1, capacity // 3))])
        return {"op": op, "streams": streams, "groups": groups, "head_dim": head_dim,
                "capacity": capacity, "new": new, "dtype": dtype, "sinks": rng.choice([0, 4, 16]),
                "recent": rng.randint(0, capacity // 2), "empty": empty}
    used = _log(rng, 16, 32771)
    return {"op": op, "streams": min(streams, 4), "groups": groups, "head_dim": head_dim,
            "used": used, "keep": _log(rng, 1, used), "dtype": dtype,
            "sinks": rng.choice([0, 4, 16]), "recent": rng.randint(0, used // 8), "empty": empty}


# ------------------------------------------------------------------------------ the inputs
def _axis_dims(case):
    return [int(d) for d in case["axis_dims"].split(",")]


#: stretched contexts: 8 times the 8192 positions trained on, base 10000
FACTOR, TRAINED, FAST, SLOW, BASE = 8.0, 8192, 32.0, 1.0, 10000.0


def _frequencies(case):
    """Radians per position and the axis of every pair, in 64 bits."""
    freq, axis = [], []
    for a, d in enumerate(_axis_dims(case)):
        base = BASE
        if case["scaling"] == "base" and d > 2:
            base *= FACTOR ** (d / (d - 2))
        for i in range(d // 2):
            f = base ** (-2 * i / d)
            if case["scaling"] == "linear":
                f /= FACTOR
            elif case["scaling"] == "blend":
                keep = min(1.0, max(0.0, (TRAINED * f / (2 * math.pi) - SLOW) / (FAST - SLOW)))
                f = keep * f + (1 - keep) * f / FACTOR
            freq.append(f)
            axis.append(a)
    return freq, axis


def _amplitude(case):
    return 0.1 * math.log(FACTOR) + 1 if case["scaling"] == "blend" else 1.0


def _filled(gen, streams, groups, slots, now, empty):
    """Positions of a cache after many replacements: `slots` of the `now` positions so far in no
    order, -1 where a slot is empty."""
    dev = "cuda"
    pos = torch.rand(streams, groups, now, generator=gen, device=dev).argsort(-1)[..., :slots]
    gone = torch.rand(streams, groups, slots, generator=gen, device=dev) < empty
    return torch.where(gone, -1, pos).to(torch.int32).contiguous()


def _totals(gen, shape):
    """Accumulated attention: a few entries hold most of it, and many hold exactly nothing."""
    x = torch.rand(shape, generator=gen, device="cuda")
    y = torch.rand(shape, generator=gen, device="cuda")
    return torch.where(y < 0.1, 0.0, 0.05 * x.clamp_min(1e-6).log().neg() ** 3).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    s = {"case": case}
    op = case["op"]
    if op == "rotary":
        t, d = case["tokens"], case["head_dim"]
        dims = _axis_dims(case)
        s["q"] = randn(t, case["q_heads"], d)
        s["k"] = randn(t, case["k_heads"], d)
        s["pos"] = torch.randint(0, case["most_pos"], (t, len(dims)), generator=gen,
                                 device="cuda").to(torch.int32)
        freq, axis = _frequencies(case)
        # phase per position in 2^-64 turns, as signed 64-bit integers
        inc = [round(f / (2 * math.pi) * 2.0 ** TURN_BITS) % 2 ** TURN_BITS for f in freq]
        s["inc"] = torch.tensor([i - 2 ** 64 if i >= 2 ** 63 else i for i in inc], device="cuda")
        s["axis"] = torch.tensor(axis, device="cuda")
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        if own:
            from paper_2607_14898_gb300 import flashdec as fdp
            s["plan"] = fdp.Rotary(d, rot_dim=case["rot_dim"], layout=case["layout"],
                                   axis_dims=dims, base=BASE, scaling=case["scaling"],
                                   factor=FACTOR, trained_len=TRAINED, fast_turns=FAST,
                                   slow_turns=SLOW, amplitude=_amplitude(case))
        return s
    S, G, D = case["streams"], case["groups"], case["head_dim"]
    slots = case["capacity"] if op == "insert" else case["used"]
    s["k"], s["v"] = randn(S, G, slots, D), randn(S, G, slots, D)
    s["weight"] = _totals(gen, (S, G, slots))
    now = slots + slots // 2 + 8  # positions so far: a third of them has been dropped
    s["pos"] = _filled(gen, S, G, slots, now, case["empty"])
    if case.get("fresh"):
        s["pos"][0] = -1  # a stream that has only begun: its cache holds nothing yet
    gone = (s["pos"] < 0)[..., None]
    s["k"].masked_fill_(gone, math.nan)  # an empty slot's bytes are whatever was there
    s["v"].masked_fill_(gone, math.nan)
    if op == "attend":
        n = case["queries"]
        s["q"] = randn(S, n, case["heads"], D)
        # the queries are the newest n positions, which are in the cache or have been dropped
        t = torch.arange(now - n, now, device="cuda", dtype=torch.int32)
        if case["mask"] == "chunk":
            t = torch.full_like(t, now - 1)
        s["q_pos"] = t.expand(S, n).contiguous()
        s["out"] = torch.empty_like(s["q"])
        s["weight_out"] = torch.empty_like(s["weight"])
        s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if own:
            from paper_2607_14898_gb300 import flashdec as fdp
            s["cache"] = fdp.Cache(s["k"], s["v"], s["pos"], s["weight"])
            s["work"] = torch.empty(
                fdp.cache_attention_workspace_bytes(s["cache"], case["heads"], n),
                dtype=torch.uint8, device="cuda")
    elif op == "insert":
        n = case["new"]
        s["k_new"], s["v_new"] = randn(S, n, G, D), randn(S, n, G, D)
        s["new_pos"] = torch.arange(now, now + n, device="cuda",
                                    dtype=torch.int32).expand(S, n).contiguous()
        s["pos_out"], s["weight_out"] = torch.empty_like(s["pos"]), torch.empty_like(s["weight"])
        s["slots"] = torch.empty(S, G, n, dtype=torch.int32, device="cuda")
        if own:
            from paper_2607_14898_gb300 import flashdec as fdp
            s["cache"] = fdp.Cache(s["k"], s["v"], s["pos"], s["weight"])
    else:
        keep = case["keep"]
        s["now"] = torch.full((S,), now, dtype=torch.int32, device="cuda")
        s["k_out"] = torch.empty(S, G, keep, D, dtype=dtype, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
        s["pos_out"] = torch.empty(S, G, keep, dtype=torch.int32, device="cuda")
        s["weight_out"] = torch.empty(S, G, keep, device="cuda")
        s["slots"] = torch.empty(S, G, keep, dtype=torch.int32, device="cuda")
        if own:
            from paper_2607_14898_gb300 import flashdec as fdp
            s["cache"] = fdp.Cache(s["k"], s["v"], s["pos"], s["weight"])
            s["dst"] = fdp.Cache(s["k_out"], s["v_out"], s["pos_out"], s["weight_out"])
    return s


# ------------------------------------------------------------------------------ the plain form
def _plain_rotary(s):
    case = s["case"]
    r = case["rot_dim"]
    # turns modulo one from the wrapped 64-bit phase, then angles in 32 bits
    phase = s["pos"].long()[:, s["axis"]] * s["inc"]
    angle = (phase >> 32).float() * (2 * math.pi / 2.0 ** 32)
    c = (angle.cos() * _amplitude(case))[:, None]
    w = (angle.sin() * _amplitude(case))[:, None]
    if case["backward"]:
        w = -w

    def turn(x):
        y = x.float()
        if case["layout"] == "interleaved":
            a, b = y[..., 0:r:2], y[..., 1:r:2]
            head = torch.stack([a * c - b * w, a * w + b * c], -1).flatten(-2)
        else:
            a, b = y[..., :r // 2], y[..., r // 2:r]
            head = torch.cat([a * c - b * w, a * w + b * c], -1)
        return torch.cat([head, y[..., r:]], -1).to(x.dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


DECAY = 0.98


def _plain_attend(s):
    case = s["case"]
    S, n, H, D = s["q"].shape
    G = case["groups"]
    q = s["q"].float().view(S, n, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(S, G, -1, D)
    live = s["pos"] >= 0
    k = torch.where(live[..., None], s["k"].float(), 0.0)
    v = torch.where(live[..., None], s["v"].float(), 0.0)
    scores = (q @ k.transpose(-1, -2)).view(S, G, H // G, n, -1) * (1 / math.sqrt(D))
    seen = live[:, :, None] & (s["pos"][:, :, None] <= s["q_pos"][:, None, :, None])
    scores = scores.masked_fill(~seen[:, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = (p.view(S, G, -1, p.shape[-1]) @ v).view(S, G, H // G, n, D)
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(S, n, H, D).to(s["q"].dtype),
            "weight": s["weight"] * DECAY + p.sum((2, 3))}


def _plain_order(s, newest, sinks, recent):
    """The slots of each (stream, group) in the order in which they are given up: empty ones,
    then the unprotected and the protected by their weight; equal ones by their index."""
    pos = s["pos"].long()
    kept = (pos < sinks) | (pos >= newest.long()[:, None, None] - recent)
    rank = torch.where(pos < 0, 0, torch.where(kept, 2, 1))
    weight = torch.where(pos < 0, 0.0, s["weight"])
    by_weight = weight.sort(dim=-1, stable=True).indices
    by_rank = rank.gather(-1, by_weight).sort(dim=-1, stable=True).indices
    return by_weight.gather(-1, by_rank)


def _plain_insert(s):
    case = s["case"]
    n = case["new"]
    order = _plain_order(s, s["new_pos"][:, 0], case["sinks"], case["recent"])
    slots = order[..., :n].sort(-1).values
    rows = slots[..., None].expand(-1, -1, -1, case["head_dim"])
    s["k"].scatter_(2, rows, s["k_new"].transpose(1, 2))
    s["v"].scatter_(2, rows, s["v_new"].transpose(1, 2))
    new_pos = s["new_pos"][:, None].expand(slots.shape)
    return {"slots": slots.to(torch.int32), "pos": s["pos"].scatter(-1, slots, new_pos),
            "weight": s["weight"].scatter(-1, slots, 0.0), "k": s["k"], "v": s["v"]}


def _plain_compact(s):
    case = s["case"]
    keep = case["keep"]
    order = _plain_order(s, s["now"], case["sinks"], case["recent"])
    last = order[..., order.shape[-1] - keep:]
    # kept entries in the order of their slots, empty places at the end
    none = s["pos"].gather(-1, last) < 0
    slots = torch.where(none, s["pos"].shape[-1], last).sort(-1).values
    none = slots == s["pos"].shape[-1]
    at = torch.where(none, 0, slots)
    rows = at[..., None].expand(-1, -1, -1, case["head_dim"])
    return {"slots": torch.where(none, -1, slots).to(torch.int32),
            "k": torch.where(none[..., None], 0.0, s["k"].gather(2, rows)).to(s["k"].dtype),
            "v": torch.where(none[..., None], 0.0, s["v"].gather(2, rows)).to(s["v"].dtype),
            "pos": torch.where(none, -1, s["pos"].gather(-1, at)).to(torch.int32),
            "weight": torch.where(none, 0.0, s["weight"].gather(-1, at))}


# ------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if not own:
        return {"rotary": _plain_rotary, "attend": _plain_attend, "insert": _plain_insert,
                "compact": _plain_compact}[case["op"]](s)
    from paper_2607_14898_gb300 import flashdec as fdp
    if case["op"] == "rotary":
        fdp.op_rotary(s["plan"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"],
                      backward=case["backward"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["op"] == "attend":
        fdp.op_cache_attention(s["cache"], s["q"], s["q_pos"], s["out"],
                               weight_out=s["weight_out"], decay=DECAY, workspace=s["work"],
                               err=s["err"])
        return {"out": s["out"], "weight": s["weight_out"]}
    if case["op"] == "insert":
        fdp.op_cache_insert(s["cache"], s["k_new"], s["v_new"], s["new_pos"], s["slots"],
                            pos_out=s["pos_out"], weight_out=s["weight_out"],
                            sinks=case["sinks"], recent=case["recent"])
        return {"slots": s["slots"], "pos": s["pos_out"], "weight": s["weight_out"],
                "k": s["k"], "v": s["v"]}
    fdp.op_cache_compact(s["cache"], s["dst"], s["now"], s["slots"], sinks=case["sinks"],
                         recent=case["recent"])
    return {"slots": s["slots"], "k": s["k_out"], "v": s["v_out"], "pos": s["pos_out"],
            "weight": s["weight_out"]}


def work(case):
    esz = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "rotary":
        heads = case["q_heads"] + case["k_heads"]
        return {"bytes": case["tokens"] * (heads * case["head_dim"] * esz * 2
                                           + 4 * len(_axis_dims(case))),
                "flops": case["tokens"] * heads * case["rot_dim"] * 3}
    lists = case["streams"] * case["groups"]
    row = case["head_dim"] * esz * 2  # a key and a value
    if case["op"] == "attend":
        n, H, D, used = case["queries"], case["heads"], case["head_dim"], case["used"]
        live = used * (1 - case["empty"])
        return {"bytes": int(lists * (live * row + used * 12)
                             + case["streams"] * n * (H * D * esz * 2 + 4)),
                "flops": int(4 * case["streams"] * H * n * live * D)}
    if case["op"] == "insert":
        return {"bytes": lists * (case["capacity"] * 16 + case["new"] * (2 * row + 8)),
                "flops": lists * case["capacity"]}
    return {"bytes": lists * (case["used"] * 8 + case["keep"] * (2 * row + 12)),
            "flops": lists * case["used"]}


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        freq, axis = _frequencies(case)
        r, half = case["rot_dim"], case["rot_dim"] // 2
        pos = s["pos"].double()
        z = torch.stack([torch.polar(torch.full_like(pos[:, a], _amplitude(case)),
                                     pos[:, a] * (-f if case["backward"] else f))
                         for f, a in zip(freq, axis)], -1)[:, None]
        found = {}
        for name in ("q", "k"):
            x = s[name].double()
            if case["layout"] == "interleaved":
                y = torch.view_as_complex(x[..., :r].unflatten(-1, (half, 2)).contiguous()) * z
                head = torch.view_as_real(y).flatten(-2)
            else:
                y = torch.complex(x[..., :half], x[..., half:r]) * z
                head = torch.cat([y.real, y.imag], -1)
            found[name] = torch.cat([head, x[..., r:]], -1)
        return found
    S, G = case["streams"], case["groups"]
    if case["op"] == "attend":
        per, D = case["heads"] // G, case["head_dim"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        weight = s["weight"].double() * DECAY
        for i in range(S):
            for g in range(G):
                at = torch.nonzero(s["pos"][i, g] >= 0)[:, 0]
                if not at.numel():
                    continue
                k, v = s["k"][i, g][at].double(), s["v"][i, g][at].double()
                hide = s["pos"][i, g][at][None, :] > s["q_pos"][i][:, None]
                for h in range(g * per, (g + 1) * per):
                    x = torch.einsum("td,jd->tj", s["q"][i, :, h].double(), k) / math.sqrt(D)
                    x = torch.logsumexp(x.masked_fill(hide, -math.inf), 1, keepdim=True).neg() + x
                    p = torch.where(hide, 0.0, x.exp())
                    out[i, :, h] = p @ v
                    weight[i, g].index_add_(0, at, p.sum(0))
        return {"out": out, "weight": weight}
    # the others move values: which ones, by a list of (class, weight, slot) for each cache
    found = {n: s[n].double().cpu().clone() for n in ("k", "v", "weight")}
    if case["op"] == "compact":
        found = {n: torch.zeros(s[n + "_out"].shape, dtype=torch.float64) for n in found}
    for i in range(S):
        newest = int(s["new_pos"][i, 0] if case["op"] == "insert" else s["now"][i])
        for g in range(G):
            pos, weight = s["pos"][i, g].tolist(), s["weight"][i, g].tolist()
            order = sorted(
                (0, 0.0, j) if p < 0 else
                (2 if p < case["sinks"] or p >= newest - case["recent"] else 1, weight[j], j)
                for j, p in enumerate(pos))
            if case["op"] == "insert":
                slots = sorted(j for _, _, j in order[:case["new"]])
                found["k"][i, g, slots] = s["k_new"][i, :, g].double().cpu()
                found["v"][i, g, slots] = s["v_new"][i, :, g].double().cpu()
                found["weight"][i, g, slots] = 0.0
            else:
                slots = sorted(j for c, _, j in order[len(order) - case["keep"]:] if c)
                for n in found:
                    found[n][i, g, :len(slots)] = s[n][i, g, slots].double().cpu()
    return {"slots": None, "pos": None, **found}
