"""An endless stream through a cache of fixed size, which keeps the entries that are looked at.

Synthetic streams whose queries keep coming back to a few early tokens (a title card, a face) are
run through one attention layer three ways: with every token kept, with the last tokens only (a
window of the same size), and with a BoundedStream. Printed is how far the two limited ones are
from attention over everything.

    python examples/bounded_stream.py [--tokens 6000] [--capacity 512] [--chunk 1]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2607_14898_gb300 import flashdec as fdp  # noqa: E402
from paper_2607_14898_gb300.bounded import BoundedStream  # noqa: E402


def stream_of(streams, tokens, heads, groups, dim, seed):
    """Queries, keys, values: 32 tokens of the first 256 are what many later queries look for."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    k, v = randn(streams, tokens, groups, dim), randn(streams, tokens, groups, dim)
    q = 0.3 * randn(streams, tokens, heads, dim)
    marked = torch.randperm(256, generator=gen, device="cuda")[:32]
    pick = marked[torch.randint(0, 32, (streams, tokens, heads), generator=gen, device="cuda")]
    group = torch.arange(heads, device="cuda") // (heads // groups)
    # each query leans towards one of the marked keys of its group
    for s in range(streams):
        q[s] += 3 * k[s][pick[s], group]
    return q.bfloat16(), k.bfloat16(), v.bfloat16(), marked


def run(bounded, q, k, v, chunk):
    out = torch.empty_like(q)
    for t in range(0, q.shape[1], chunk):
        pos = torch.arange(t, min(t + chunk, q.shape[1]), dtype=torch.int32, device="cuda")
        pos = pos.expand(q.shape[0], -1).contiguous()
        e = t + pos.shape[1]
        out[:, t:e] = bounded.step(q[:, t:e].contiguous(), k[:, t:e].contiguous(),
                                   v[:, t:e].contiguous(), pos)
    bounded.check()
    return out


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=6000)
    ap.add_argument("--capacity", type=int, default=512)
    ap.add_argument("--chunk", type=int, default=1)
    a = ap.parse_args()
    S, H, G, D = 2, 16, 4, 64
    # a quarter of each head carries the position, the rest meets its content wherever that is
    plan = fdp.Rotary(D, rot_dim=16, layout="half", base=1e6)
    q, k, v, marked = stream_of(S, a.tokens, H, G, D, 0)

    def make(capacity, recent, decay=0.999):
        return BoundedStream(S, H, G, D, capacity, plan=plan, sinks=0, recent=recent, decay=decay)
    everything = run(make(a.tokens, 0), q, k, v, a.chunk)
    tail = slice(a.tokens * 3 // 4, None)  # long after the marked tokens
    norm = float(everything[:, tail].float().norm())
    # entries among the last capacity - chunk are kept, so that the oldest ones make room
    for name, b in (("the last %d tokens" % a.capacity, make(a.capacity, a.capacity - a.chunk)),
                    ("the %d most used" % a.capacity, make(a.capacity, a.capacity // 4))):
        got = run(b, q, k, v, a.chunk)
        off = float((got[:, tail].float() - everything[:, tail].float()).norm()) / norm
        kept = int(torch.isin(b.cache.pos, marked.int()).sum()) / (S * G)
        print(f"{name}: {off:.3f} away from all {a.tokens} tokens, "
              f"{kept:.1f} of the 32 marked tokens kept")


if __name__ == "__main__":
    main()
