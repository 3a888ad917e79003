"""The operators of a residual block in training, in their plain form and through the library.

Attention in which every query sees a span of keys (packed sequences, chunks of a clip with a
window, new tokens against long pasts), and its gradient, which computes the probabilities again
from the log-sum-exp; the join between two blocks (the norm after a block, its gate and residual
scale, the residual sum, the norm before the next block) and its gradient; checkpoints of
activations in 8 bits, which the join writes of what it reads and its gradient reads, and which
are restored as they were or transposed for a weight gradient. The sizes are those of the
streaming decoder's presets (width 1024, 16 heads in 4 groups of head dimension 64, 1560 tokens
a chunk, a window of 4 chunks) and generic ones.

`own` chooses what run() computes with: elementary torch operations, or the library.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
BLOCK = 32  # elements of a row that share a checkpoint's exponent


def listed():
    return [
        # the next token of 8 streams, each over its own past (480p windows of ragged fill)
        {"name": "attend_token", "op": "attend", "seqs": 8, "tokens": 49920, "new": 1, "chunk": 1,
         "window": 0, "pad": 0, "heads": 16, "groups": 4, "head_dim": 64, "dtype": "bf16"},
        # a 480p clip of 6 chunks under the decoder's window of 4
        {"name": "attend_clip", "op": "attend", "seqs": 1, "tokens": 9360, "new": 0, "chunk": 1560,
         "window": 4, "pad": 0, "heads": 16, "groups": 4, "head_dim": 64, "dtype": "bf16"},
        # ragged sequences packed into one batch, causal, padded at its end
        {"name": "attend_packed", "op": "attend", "seqs": 5, "tokens": 8191, "new": 0, "chunk": 1,
         "window": 0, "pad": 129, "heads": 32, "groups": 8, "head_dim": 128, "dtype": "fp16"},
        # a few short sequences, three queries a group: what latency costs
        {"name": "attend_short_grad", "op": "attend_grad", "seqs": 2, "tokens": 77, "new": 0,
         "chunk": 1, "window": 0, "pad": 3, "heads": 6, "groups": 2, "head_dim": 64,
         "dtype": "fp16"},
        # the clip's gradient
        {"name": "attend_clip_grad", "op": "attend_grad", "seqs": 1, "tokens": 9360, "new": 0,
         "chunk": 1560, "window": 4, "pad": 0, "heads": 16, "groups": 4, "head_dim": 64,
         "dtype": "bf16"},
        # one long causal sequence's gradient
        {"name": "attend_long_grad", "op": "attend_grad", "seqs": 1, "tokens": 8191, "new": 0,
         "chunk": 1, "window": 0, "pad": 0, "heads": 32, "groups": 8, "head_dim": 128,
         "dtype": "bf16"},
        # between two blocks, one new token of 8 streams, each with a gate of its own
        {"name": "join_token", "op": "join", "tokens": 8, "width": 1024, "dtype": "bf16",
         "stream": "fp32", "gate_tokens": 1, "post": True, "pre": True, "codes": False},
        # between two refinement blocks of a 480p chunk in training: both inputs kept in 8 bits
        {"name": "join_chunk", "op": "join", "tokens": 6240, "width": 1024, "dtype": "bf16",
         "stream": "fp32", "gate_tokens": 6240, "post": True, "pre": True, "codes": True},
        {"name": "join_chunk_grad", "op": "join_grad", "tokens": 6240, "width": 1024,
         "dtype": "bf16", "stream": "fp32", "gate_tokens": 6240, "post": True, "pre": True,
         "codes": True},
        # a wide model's batch of ragged length, a gate for every 1000 tokens, nothing in 8 bits
        {"name": "join_wide_grad", "op": "join_grad", "tokens": 16001, "width": 4096,
         "dtype": "bf16", "stream": "bf16", "gate_tokens": 1000, "post": True, "pre": True,
         "codes": False},
        # the hidden activations of a 480p refinement block's MLP into 8 bits
        {"name": "save_hidden", "op": "save", "tokens": 6240, "width": 4096, "dtype": "bf16"},
        # a batch of ragged length back from 8 bits, transposed for a weight gradient
        {"name": "load_transposed", "op": "load", "tokens": 16001, "width": 4096, "dtype": "fp16",
         "transposed": True},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend_grad", "attend_grad", "join", "join_grad",
                     "join_grad", "save", "load"])
    dtype = rng.choice(["bf16", "fp16"])
    if op.startswith("attend"):
        groups, per = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 6, 8])
        tokens = _log(rng, 1, 8191)
        case = {"op": op, "seqs": min(tokens, rng.choice([1, 1, 2, 3, 8])), "tokens": tokens,
                "new": 0, "chunk": rng.choice([1, 1, 1, _log(rng, 2, 1560)]), "window": 0,
                "pad": rng.choice([0, 0, 1, 100]), "heads": groups * per, "groups": groups,
                "head_dim": rng.choice([64, 128]), "dtype": dtype}
        if rng.random() < 0.4:
            case["window"] = max(1, _log(rng, 1, tokens) // case["chunk"])
        if rng.random() < 0.3:  # new tokens after a past
            case["new"] = _log(rng, 1, 500)
            case["tokens"] = _log(rng, case["seqs"], 49920)
            if op == "attend_grad":
                case["tokens"] = max(case["seqs"], case["tokens"] // 4)
        # no more scores than the longest listed case's
        while case["heads"] * _queries(case) * case["tokens"] > 32 * 8191 ** 2:
            case["tokens"] = max(case["seqs"], case["tokens"] // 2)
        return case
    width = 8 * _log(rng, 8, 512) if rng.random() < 0.5 else rng.choice([64, 128, 1024, 1536, 4096])
    tokens = _log(rng, 1, 16001)
    if op.startswith("join"):
        return {"op": op, "tokens": tokens, "width": width, "dtype": dtype,
                "stream": rng.choice(["fp32", dtype]),
                "gate_tokens": rng.choice([0, 1, tokens, _log(rng, 1, tokens)]),
                "post": rng.random() < 0.8, "pre": rng.random() < 0.8,
                "codes": rng.random() < 0.5}
    case = {"op": op, "tokens": tokens, "width": width,
            "dtype": rng.choice(["bf16", "fp16", "fp32"])}
    if op == "load":
        case["transposed"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------------------ the inputs
def _lengths(case):
    """Ragged lengths of the packed sequences, the same for every seed."""
    n, seqs = case["tokens"], case["seqs"]
    cuts = sorted(random.Random(n * 64 + seqs).sample(range(1, n), seqs - 1)) if seqs > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [n])]


def _queries(case):
    """Queries in all, without the padding."""
    new = case["new"]
    return sum(min(new, n) if new else n for n in _lengths(case))


def _spans(case):
    """The span of keys that each query sees; the padding's queries see none."""
    chunk, window, at, spans = case["chunk"], case["window"], 0, []
    for n in _lengths(case):
        for p in range(n - min(case["new"], n) if case["new"] else 0, n):
            c = p // chunk
            low = max(0, (c - window + 1) * chunk) if window else 0
            spans.append((at + low, at + min(n, (c + 1) * chunk)))
        at += n
    return spans + [(0, 0)] * case["pad"]


def _gate_rows(case):
    return -(-case["tokens"] // case["gate_tokens"]) if case["gate_tokens"] else 0


def _blocks(width):
    return -(-width // BLOCK)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]

    def randn(*shape, to=dtype):
        return torch.randn(shape, generator=gen, device="cuda").to(to)

    s = {"case": case}
    op = case["op"]
    if op.startswith("attend"):
        H, G, D, pad = case["heads"], case["groups"], case["head_dim"], case["pad"]
        spans = _spans(case)
        T, S = len(spans), case["tokens"] + pad
        s["spans"] = torch.tensor(spans, dtype=torch.int32, device="cuda")
        s["q"], s["k"], s["v"] = randn(T, H, D), randn(S, G, D), randn(S, G, D)
        names = ["q", "k", "v"]
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(H, T, device="cuda")
        if op == "attend_grad":
            s["dout"] = randn(T, H, D)
            names.append("dout")
            found = _plain_attend(s)  # what the forward pass has left
            s["out"], s["lse"] = found["out"], found["lse"]
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in "qkv")
        for n in names:
            if pad:  # the padding's rows hold whatever was there
                s[n][-pad:] = math.nan
        if own:
            from paper_2607_14898_gb300 import flashdec as fdp
            s["work"] = torch.empty(
                fdp.span_attention_workspace_bytes(T, S, H, G, D, backward=op == "attend_grad"),
                dtype=torch.uint8, device="cuda")
            s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        return s
    T, W = case["tokens"], case["width"]
    if op in ("save", "load"):
        # activations: most near zero, a few channels many times larger
        x = randn(T, W, to=torch.float32) * torch.exp(1.5 * randn(W, to=torch.float32))
        s["x"] = x.to(dtype)
        s["codes"] = torch.empty(T, W, dtype=torch.int8, device="cuda")
        s["exps"] = torch.empty(T, _blocks(W), dtype=torch.uint8, device="cuda")
        if op == "load":
            s["codes"], s["exps"] = _plain_codes(s["x"])
            s["x"] = torch.empty((W, T) if case["transposed"] else (T, W), dtype=dtype,
                                 device="cuda")
        if own:
            from paper_2607_14898_gb300 import flashdec as fdp
            s["kept"] = fdp.Checkpoint8(s["codes"], s["exps"])
        return s
    stream, f32 = DTYPES[case["stream"]], torch.float32
    rows = _gate_rows(case)
    s["h"], s["b"] = randn(T, W, to=f32).mul_(3).to(stream), randn(T, W)
    s["post"] = 1 + 0.1 * randn(W, to=f32) if case["post"] else None
    s["pre"] = 1 + 0.1 * randn(W, to=f32) if case["pre"] else None
    s["gate"] = 0.5 + 0.5 * randn(rows, W, to=f32) if rows else None
    s["scale"] = 0.7
    s["r_post"] = torch.empty(T, device="cuda") if case["post"] else None
    s["r_pre"] = torch.empty(T, device="cuda") if case["pre"] else None
    if op == "join":
        s["y"] = torch.empty_like(s["h"])
        s["u"] = torch.empty_like(s["b"]) if case["pre"] else None
        if case["codes"]:
            for n in "hb":
                s[n + "_codes"] = torch.empty(T, W, dtype=torch.int8, device="cuda")
                s[n + "_exps"] = torch.empty(T, _blocks(W), dtype=torch.uint8, device="cuda")
    else:
        found = _plain_join(s)  # what the forward pass has left
        s["r_post"], s["r_pre"] = found.get("r_post"), found.get("r_pre")
        if case["codes"]:
            s["h_codes"], s["h_exps"] = _plain_codes(s["h"])
            s["b_codes"], s["b_exps"] = _plain_codes(s["b"])
            s["h"] = s["b"] = None
        s["dy"] = randn(T, W, to=stream)
        s["du"] = randn(T, W) if case["pre"] else None
        s["dh"] = torch.empty(T, W, dtype=stream, device="cuda")
        s["db"] = torch.empty(T, W, dtype=dtype, device="cuda")
        for n in ("post", "pre", "gate"):
            s["d_" + n] = None if s[n] is None else torch.empty_like(s[n])
    if own:
        from paper_2607_14898_gb300 import flashdec as fdp
        for n in "hb":
            s["kept_" + n] = fdp.Checkpoint8(s[n + "_codes"], s[n + "_exps"]) if case["codes"] \
                else None
        if op == "join_grad":
            s["work"] = torch.empty(fdp.block_join_bwd_workspace_bytes(T, W), dtype=torch.uint8,
                                    device="cuda")
    return s


# ------------------------------------------------------------------------------ the plain form
def _seen(s):
    """[T][S]: whether query t sees key j."""
    j = torch.arange(s["k"].shape[0], device="cuda", dtype=torch.int32)
    low, high = s["spans"][:, :1], s["spans"][:, 1:]
    return (j >= low) & (j < high)


def _scores(s):
    """Scores in 32 bits [H][T][S], -inf where they are hidden, and the inputs by heads [H][.][D];
    what no query sees, and queries that see nothing, count as zeros."""
    per = s["case"]["heads"] // s["case"]["groups"]
    seen = _seen(s)
    of_query, of_key = seen.any(1)[:, None, None], seen.any(0)[:, None, None]

    def heads(x, live, times):
        return torch.where(live, x.float(), 0.0).repeat_interleave(times, 1).transpose(0, 1)

    q = heads(s["q"], of_query, 1)
    k, v = heads(s["k"], of_key, per), heads(s["v"], of_key, per)
    x = (q @ k.transpose(1, 2)) * (1 / math.sqrt(s["case"]["head_dim"]))
    return x.masked_fill_(~seen, -math.inf), q, k, v, of_query, heads


def _plain_attend(s):
    x, _, _, v, _, _ = _scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total == 0, 1.0, total)
    return {"out": out.transpose(0, 1).to(s["q"].dtype).contiguous(),
            "lse": (top + total.log())[..., 0]}


def _plain_attend_grad(s):
    case = s["case"]
    G, scale = case["groups"], 1 / math.sqrt(case["head_dim"])
    x, q, k, v, of_query, heads = _scores(s)
    lse = torch.where(s["lse"] == -math.inf, 0.0, s["lse"])[..., None]
    p = x.sub_(lse).exp_()
    dout, out = heads(s["dout"], of_query, 1), heads(s["out"], of_query, 1)
    delta = (dout * out).sum(-1, keepdim=True)
    dv = p.transpose(1, 2) @ dout
    ds = (dout @ v.transpose(1, 2)).sub_(delta).mul_(p)
    dq = (ds @ k) * scale
    dk = (ds.transpose(1, 2) @ q) * scale

    def of_group(x):
        return x.unflatten(0, (G, -1)).sum(1).transpose(0, 1).to(s["q"].dtype).contiguous()

    return {"dq": dq.transpose(0, 1).to(s["q"].dtype).contiguous(), "dk": of_group(dk),
            "dv": of_group(dv)}


def _plain_codes(x):
    """(codes int8 [T][W], exponents uint8 [T][blocks]) of x: in every block of 32 elements the
    smallest power of two that lets the largest fit into 127 steps."""
    T, W = x.shape
    y = torch.zeros(T, _blocks(W) * BLOCK, device="cuda")
    y[:, :W] = x
    y = y.view(T, -1, BLOCK)
    top = y.abs().amax(-1)
    m, e = torch.frexp(top)                      # top = m 2^e, 0.5 <= m < 1
    e = (e - 7 + (m > 127 / 128).int()).clamp(min=-126)
    e = torch.where(top == 0, -126, e)
    codes = torch.round(y.double() * torch.exp2(-e.double())[..., None])
    return codes.view(T, -1)[:, :W].to(torch.int8).contiguous(), (e + 127).to(torch.uint8)


def _plain_values(codes, exps):
    """The values that codes stand for, exact in 32 bits."""
    step = torch.exp2(exps.double() - 127).float().repeat_interleave(BLOCK, 1)
    return codes.float() * step[:, :codes.shape[1]]


def _by_token(s, gate):
    """The gate of every token (1 without one)."""
    case = s["case"]
    if gate is None:
        return 1.0
    if gate.shape[0] == 1:
        return gate
    return gate.repeat_interleave(case["gate_tokens"], 0)[:case["tokens"]]


def _plain_join(s):
    case = s["case"]
    found = {}
    b = s["b"].float()
    n = b
    if case["post"]:
        found["r_post"] = (b.square().mean(-1) + EPS).rsqrt()
        n = b * found["r_post"][:, None] * s["post"]
    y = s["h"].float() + s["scale"] * _by_token(s, s["gate"]) * n
    found["y"] = y.to(s["h"].dtype)
    if case["pre"]:
        found["r_pre"] = (y.square().mean(-1) + EPS).rsqrt()
        found["u"] = (y * found["r_pre"][:, None] * s["pre"]).to(s["b"].dtype)
    if case["codes"]:
        found["h_codes"], found["h_exps"] = _plain_codes(s["h"])
        found["b_codes"], found["b_exps"] = _plain_codes(s["b"])
    return found


def _plain_join_grad(s):
    case = s["case"]
    if case["codes"]:
        h = _plain_values(s["h_codes"], s["h_exps"])
        b = _plain_values(s["b_codes"], s["b_exps"])
    else:
        h, b = s["h"].float(), s["b"].float()
    found = {}
    gate, post = _by_token(s, s["gate"]), s["post"] if case["post"] else 1.0
    r = s["r_post"][:, None] if case["post"] else 1.0
    n = b * r
    d = s["dy"].float()
    if case["pre"]:
        y = h + s["scale"] * gate * (n * post)
        m = y * s["r_pre"][:, None]
        du = s["du"].float()
        found["d_pre"] = (du * m).sum(0)
        g = du * s["pre"]
        d = d + s["r_pre"][:, None] * (g - m * (g * m).mean(-1, keepdim=True))
    found["dh"] = d.to(s["dh"].dtype)
    w = s["scale"] * d
    if s["gate"] is not None:
        each = w * n * post
        rows, of = s["gate"].shape[0], case["gate_tokens"]
        full = torch.zeros(rows * of, case["width"], device="cuda")
        full[:case["tokens"]] = each
        found["d_gate"] = full.view(rows, of, -1).sum(1)
    if case["post"]:
        found["d_post"] = (w * gate * n).sum(0)
        dn = w * gate * post
        db = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    else:
        db = w * gate
    found["db"] = db.to(s["db"].dtype)
    return found


# ------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "save":
            codes, exps = _plain_codes(s["x"])
            return {"codes": codes, "exps": exps}
        if op == "load":
            x = _plain_values(s["codes"], s["exps"]).to(s["x"].dtype)
            return {"x": x.t().contiguous() if case["transposed"] else x}
        return {"attend": _plain_attend, "attend_grad": _plain_attend_grad, "join": _plain_join,
                "join_grad": _plain_join_grad}[op](s)
    from paper_2607_14898_gb300 import flashdec as fdp
    if op == "attend":
        fdp.op_span_attention(s["q"], s["k"], s["v"], s["spans"], s["out"], s["lse"],
                              workspace=s["work"], err=s["err"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "attend_grad":
        fdp.op_span_attention_bwd(s["q"], s["k"], s["v"], s["spans"], s["out"], s["lse"],
                                  s["dout"], s["dq"], s["dk"], s["dv"], workspace=s["work"],
                                  err=s["err"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if op == "save":
        fdp.op_checkpoint_save(s["x"], s["kept"])
        return {"codes": s["codes"], "exps": s["exps"]}
    if op == "load":
        fdp.op_checkpoint_load(s["kept"], s["x"], transposed=case["transposed"])
        return {"x": s["x"]}
    if op == "join":
        fdp.op_block_join(s["h"], s["b"], s["y"], s["u"], post_gain=s["post"], pre_gain=s["pre"],
                          gate=s["gate"], gate_tokens=case["gate_tokens"], scale=s["scale"],
                          eps=EPS, r_post=s["r_post"], r_pre=s["r_pre"], h_kept=s["kept_h"],
                          b_kept=s["kept_b"])
        names = ["y", "u", "r_post", "r_pre", "h_codes", "h_exps", "b_codes", "b_exps"]
    else:
        fdp.op_block_join_bwd(
            s["dy"], s["du"], s["kept_h"] if case["codes"] else s["h"],
            s["kept_b"] if case["codes"] else s["b"], s["dh"], s["db"], post_gain=s["post"],
            pre_gain=s["pre"], gate=s["gate"], gate_tokens=case["gate_tokens"], scale=s["scale"],
            r_post=s["r_post"], r_pre=s["r_pre"], d_post=s["d_post"], d_pre=s["d_pre"],
            d_gate=s["d_gate"], workspace=s["work"])
        names = ["dh", "db", "d_post", "d_pre", "d_gate"]
    return {n: s[n] for n in names if s.get(n) is not None}


def work(case):
    esz = 4 if case["dtype"] == "fp32" else 2
    if case["op"].startswith("attend"):
        H, G, D = case["heads"], case["groups"], case["head_dim"]
        spans = _spans(case)
        pairs = sum(max(0, b - a) for a, b in spans)
        q, kv = len(spans) * H * D * 2, (case["tokens"] + case["pad"]) * G * D * 2
        small = len(spans) * (8 + 4 * H)
        if case["op"] == "attend":
            return {"bytes": 2 * q + 2 * kv + small, "flops": 4 * H * D * pairs}
        return {"bytes": 4 * q + 4 * kv + small, "flops": 10 * H * D * pairs}
    n = case["tokens"] * case["width"]
    kept = n + case["tokens"] * _blocks(case["width"])
    if case["op"] in ("save", "load"):
        return {"bytes": n * esz + kept, "flops": n}
    stream = 4 if case["stream"] == "fp32" else 2
    small = case["width"] * 4 * (_gate_rows(case) + case["post"] + case["pre"]) \
        + case["tokens"] * 4 * (case["post"] + case["pre"])
    pre = 2 if case["pre"] else 0
    if case["op"] == "join":
        return {"bytes": n * (2 * stream + 2 + pre) + small + (2 * kept if case["codes"] else 0),
                "flops": 10 * n}
    inputs = 2 * kept if case["codes"] else n * (stream + 2)
    return {"bytes": n * (2 * stream + 2 + pre) + inputs + 2 * small, "flops": 25 * n}


# ------------------------------------------------------------------------------ in 64 bits
def _exact_attend(s, case, grad):
    """Sequence by sequence and head by head: the queries of a sequence against its own keys."""
    H, per, D = case["heads"], case["heads"] // case["groups"], case["head_dim"]
    f64 = {"dtype": torch.float64, "device": "cuda"}
    T, S = s["q"].shape[0], s["k"].shape[0]
    out, lse = torch.zeros(T, H, D, **f64), torch.full((H, T), -math.inf, **f64)
    dq = torch.zeros(T, H, D, **f64)
    dk, dv = torch.zeros(S, case["groups"], D, **f64), torch.zeros(S, case["groups"], D, **f64)
    at, t0 = 0, 0
    for n in _lengths(case):
        m = min(case["new"], n) if case["new"] else n
        c = torch.arange(n - m, n, device="cuda") // case["chunk"]
        keys = torch.arange(n, device="cuda")[None] // case["chunk"]
        hide = keys > c[:, None]
        if case["window"]:
            hide |= keys <= c[:, None] - case["window"]
        for h in range(H):
            q = s["q"][t0:t0 + m, h].double()
            k, v = (s[x][at:at + n, h // per].double() for x in "kv")
            x = torch.einsum("td,jd->tj", q, k).div_(math.sqrt(D))
            x[hide] = -math.inf
            if not grad:
                lse[h, t0:t0 + m] = torch.logsumexp(x, 1)
                out[t0:t0 + m, h] = torch.softmax(x, 1) @ v
                continue
            p = torch.exp(x - s["lse"][h, t0:t0 + m].double()[:, None])
            do, o = s["dout"][t0:t0 + m, h].double(), s["out"][t0:t0 + m, h].double()
            dv[at:at + n, h // per] += torch.einsum("tj,td->jd", p, do)
            p *= torch.einsum("td,jd->tj", do, v) - torch.einsum("td,td->t", do, o)[:, None]
            dq[t0:t0 + m, h] = (p @ k) / math.sqrt(D)
            dk[at:at + n, h // per] += torch.einsum("tj,td->jd", p, q) / math.sqrt(D)
        at, t0 = at + n, t0 + m
    return {"dq": dq, "dk": dk, "dv": dv} if grad else {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("attend"):
        return _exact_attend(s, case, op == "attend_grad")
    if op == "save":
        return None  # whole numbers
    T, W = case["tokens"], case["width"]

    def values(codes, exps):
        of = torch.arange(W, device="cuda") // BLOCK
        return torch.ldexp(codes.double(), exps.long()[:, of] - 127)

    if op == "load":
        x = values(s["codes"], s["exps"])
        return {"x": x.T if case["transposed"] else x}
    if case["codes"] and op == "join_grad":
        h = values(s["h_codes"], s["h_exps"])
        b = values(s["b_codes"], s["b_exps"])
    else:
        h, b = s["h"].double(), s["b"].double()
    post = s["post"].double() if case["post"] else torch.ones(W, device="cuda").double()
    gate = torch.ones(1, W, device="cuda").double() if s["gate"] is None else s["gate"].double()
    row = torch.arange(T, device="cuda") // max(1, case["gate_tokens"]) if s["gate"] is not None \
        else torch.zeros(T, dtype=torch.long, device="cuda")
    if op == "join":
        found = {"h_codes": None, "h_exps": None, "b_codes": None, "b_exps": None} \
            if case["codes"] else {}
        z = b * gate[row] * post
        if case["post"]:
            found["r_post"] = 1 / torch.sqrt(torch.linalg.vector_norm(b, dim=1) ** 2 / W + EPS)
            z *= found["r_post"][:, None]
        found["y"] = h + s["scale"] * z
        if case["pre"]:
            y = found["y"]
            found["r_pre"] = 1 / torch.sqrt(torch.linalg.vector_norm(y, dim=1) ** 2 / W + EPS)
            found["u"] = torch.einsum("td,t,d->td", y, found["r_pre"], s["pre"].double())
        return found
    # the gradient: sums over rows as products, the norms' projections as inner products
    n = b * s["r_post"].double()[:, None] if case["post"] else b
    d = s["dy"].double()
    found = {}
    if case["pre"]:
        r, du = s["r_pre"].double(), s["du"].double()
        m = (h + s["scale"] * gate[row] * n * post) * r[:, None]
        found["d_pre"] = torch.einsum("td,td->d", du, m)
        along = torch.einsum("td,d,td->t", du, s["pre"].double(), m) / W
        d = d + r[:, None] * du * s["pre"].double() - (r * along)[:, None] * m
    found["dh"] = d
    part = torch.zeros(gate.shape[0], W, dtype=torch.float64, device="cuda")
    part.index_add_(0, row, s["scale"] * d * n)
    if s["gate"] is not None:
        found["d_gate"] = part * post
    dn = s["scale"] * d * gate[row] * post
    if case["post"]:
        found["d_post"] = (part * gate).sum(0)
        along = torch.einsum("td,td->t", dn, n) / W
        found["db"] = s["r_post"].double()[:, None] * (dn - along[:, None] * n)
    else:
        found["db"] = dn
    return found
