"""Two residual attention blocks learn to look something up, on the library's training operators.

Packed sequences of ragged length; every token of a sequence is to end up with the first token's
content, which only attention can bring there. The blocks keep their activations in 8 bits between the
forward and the backward pass; weights and optimiser are fp32 torch tensors.

    python examples/train_residual.py [--steps 200] [--width 256]
"""
import argparse
import os
import random
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2607_14898_gb300 import ResidualAttention  # noqa: E402


def batch(tokens, width, rng, gen):
    """(content, target, spans): the first token of a sequence is marked by its first element."""
    x = torch.randn(tokens, width, generator=gen, device="cuda")
    x[:, 0] = 0
    target, spans, at = torch.empty_like(x), [], 0
    while at < tokens:
        n = min(tokens - at, rng.randint(3, 60))
        x[at, 0] = 8
        target[at:at + n] = x[at]
        spans += [(at, at + p + 1) for p in range(n)]
        at += n
    return x, target, torch.tensor(spans, dtype=torch.int32, device="cuda")


def make_blocks(tokens, width, heads, groups, head_dim, seed=0):
    """(blocks, their parameters by name)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    blocks, params = [], []
    for _ in range(2):
        def randn(*shape):
            return torch.randn(shape, generator=gen, device="cuda")
        p = {"w_qkv": randn((heads + 2 * groups) * head_dim, width) * width ** -0.5,
             "w_out": randn(width, heads * head_dim) * (heads * head_dim) ** -0.5,
             "post_gain": torch.ones(width, device="cuda"), "pre_gain": torch.ones(width, device="cuda"),
             "gate": torch.full((1, width), 0.5, device="cuda")}
        blocks.append(ResidualAttention(tokens, width, heads, groups, head_dim, p["w_qkv"], p["w_out"],
                                        p["post_gain"], p["pre_gain"], p["gate"], tokens))
        params.append(p)
    return blocks, params


def train_step(blocks, params, x, target, spans):
    """The loss, and every parameter's gradient in its .grad."""
    h, u = x, (x / x.square().mean(1, keepdim=True).sqrt()).bfloat16()
    for b in blocks:
        h, u = b.forward(h, u, spans)
    off = h - target
    dh, du = off * (2 / off.numel()), torch.zeros_like(u)
    for b, p in reversed(list(zip(blocks, params))):
        dh, du, grads = b.backward(dh, du)
        for name, g in grads.items():
            p[name].grad = g
    return off.square().mean()


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=2048)
    a = ap.parse_args(argv)
    heads, groups, head_dim = 8, 2, 64
    blocks, params = make_blocks(a.tokens, a.width, heads, groups, head_dim)
    every = [t for p in params for t in p.values()]
    optimiser = torch.optim.Adam(every, lr=2e-3)
    rng, gen = random.Random(0), torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for step in range(a.steps):
        loss = train_step(blocks, params, *batch(a.tokens, a.width, rng, gen))
        optimiser.step()
        for b, p in zip(blocks, params):
            b.load(p["w_qkv"], p["w_out"])
        losses.append(float(loss))
        if step % 20 == 0 or step == a.steps - 1:
            print(f"step {step}: mean squared error {losses[-1]:.4f}")
    for b in blocks:
        b.check()
    return losses


if __name__ == "__main__":
    main()
