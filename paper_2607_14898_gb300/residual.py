"""A residual attention block in training, on the library's kernels.

    q, k, v = u W_qkv^T;  a = attention in spans of keys;  b = a W_out^T
    y = h + scale gate norm(b) post_gain;  u_next = norm(y) pre_gain

One forward call is the projections (fd_op_linear), the attention (fd_op_span_attention) and the join
with the next block's norm (fd_op_block_join); backward their gradients. What the backward pass needs of
the wide activations, u, h and b, is kept in 8 bits (fd_op_checkpoint_save and the join itself).
"""
from __future__ import annotations

import torch

from . import flashdec as fdp


class ResidualAttention:
    """One block for `tokens` packed tokens (a multiple of 8) of `width`, `heads` query heads in `groups` KV
    groups of head_dim 64 or 128, bfloat16, residual stream float32.

    w_qkv float32 or bfloat16 [(heads + 2 groups) head_dim][width], w_out [width][heads head_dim];
    post_gain, pre_gain float32 [width]; gate float32 [ceil(tokens / gate_tokens)][width] or None.
    load() takes the weights after they have changed. Buffers are allocated once; a block holds what one
    forward call leaves for one backward call. The calls run on the current stream."""

    def __init__(self, tokens, width, heads, groups, head_dim, w_qkv, w_out, post_gain, pre_gain, gate=None,
                 gate_tokens=0, scale=1.0, eps=1e-6):
        if tokens < 8 or tokens % 8 or not 32 <= width <= 8192 or width % 32:
            raise ValueError("tokens in multiples of 8 and a width of 32 to 8192 in multiples of 32 are required")
        if head_dim not in (64, 128) or not 1 <= groups <= heads or heads % groups or heads > 128 * groups:
            raise ValueError("head_dim 64 or 128 and heads in equal groups of 128 at most are required")
        self.tokens, self.width, self.heads, self.groups, self.head_dim = tokens, width, heads, groups, head_dim
        self.post_gain, self.pre_gain, self.gate, self.gate_tokens = post_gain, pre_gain, gate, gate_tokens
        self.scale, self.eps = scale, eps
        dev, bf16, f32 = post_gain.device, torch.bfloat16, torch.float32
        H, G, D, T, W = heads, groups, head_dim, tokens, width
        self.inner, self.mixed = H * D, (H + 2 * G) * D

        def new(*shape, dtype=bf16):
            return torch.empty(shape, dtype=dtype, device=dev)

        self.w_qkv, self.w_out = new(self.mixed, W), new(W, self.inner)
        self.w_qkv_t, self.w_out_t = new(W, self.mixed), new(self.inner, W)
        self.load(w_qkv, w_out)
        self.zeros = torch.zeros(max(self.mixed, W, self.inner), device=dev)
        self.qkv, self.out, self.b = new(T, self.mixed), new(T, H, D), new(T, W)
        self.lse, self.r_post, self.r_pre = new(H, T, dtype=f32), new(T, dtype=f32), new(T, dtype=f32)
        self.dqkv, self.dout, self.db = new(T, self.mixed), new(T, H, D), new(T, W)
        self.u_kept, self.h_kept, self.b_kept = (fdp.Checkpoint8.empty(T, W, dev) for _ in range(3))
        self.u_t = new(W, T)
        self.wide = new(T, max(self.mixed, W, self.inner), dtype=f32)  # a product before it is rounded
        self.work = [torch.empty(fdp.span_attention_workspace_bytes(T, T, H, G, D, backward=back),
                                 dtype=torch.uint8, device=dev) for back in (False, True)]
        self.join_work = torch.empty(fdp.block_join_bwd_workspace_bytes(T, W), dtype=torch.uint8, device=dev)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)
        self.spans = None

    def load(self, w_qkv, w_out) -> None:
        """The weights, rounded to bfloat16, as they are and transposed."""
        for w, to, to_t in ((w_qkv, self.w_qkv, self.w_qkv_t), (w_out, self.w_out, self.w_out_t)):
            to.copy_(w)
            to_t.copy_(to.t())

    def _linear(self, A, W, to):
        """A W^T into `to` (fp32 sums; rounded once where `to` is narrower)."""
        rows, cols = A.shape[0], W.shape[0]
        wide = to if to.dtype == torch.float32 else self.wide.view(-1)[:rows * cols].view(rows, cols)
        fdp.op_linear(fdp.EPI_F32, A, W, self.zeros[:cols], wide, err=self.err)
        if wide is not to:
            to.copy_(wide)

    def _heads(self, x):
        """Queries, keys and values (or their gradients) as parts of one matrix."""
        H, G, D = self.heads, self.groups, self.head_dim
        return (x[:, :H * D].unflatten(1, (H, D)), x[:, H * D:(H + G) * D].unflatten(1, (G, D)),
                x[:, (H + G) * D:].unflatten(1, (G, D)))

    def forward(self, h, u, spans):
        """(y, u_next) of the residual stream h float32 [tokens][width] and the block's normed input u bfloat16;
        spans int32 [tokens][2]: the keys that each token sees."""
        if u.dtype != torch.bfloat16 or not u.is_contiguous():
            raise TypeError("u: a contiguous bfloat16 tensor is required")  # (the products read it as it lies)
        self.spans = spans
        fdp.op_checkpoint_save(u, self.u_kept)
        self._linear(u, self.w_qkv, self.qkv)
        q, k, v = self._heads(self.qkv)
        fdp.op_span_attention(q, k, v, spans, self.out, self.lse, workspace=self.work[0], err=self.err)
        self._linear(self.out.view(self.tokens, self.inner), self.w_out, self.b)
        y, u_next = torch.empty_like(h), torch.empty_like(u)
        fdp.op_block_join(h, self.b, y, u_next, post_gain=self.post_gain, pre_gain=self.pre_gain,
                          gate=self.gate, gate_tokens=self.gate_tokens, scale=self.scale, eps=self.eps,
                          r_post=self.r_post, r_pre=self.r_pre, h_kept=self.h_kept, b_kept=self.b_kept)
        return y, u_next

    def backward(self, dy, du_next):
        """(dh, du, gradients) from those of forward's results: dh float32 and du bfloat16 [tokens][width];
        gradients float32 by name: w_qkv, w_out, post_gain, pre_gain and gate."""
        f32 = torch.float32
        dh, du = torch.empty_like(dy), torch.empty_like(du_next)
        g = {"post_gain": torch.empty_like(self.post_gain), "pre_gain": torch.empty_like(self.pre_gain),
             "gate": None if self.gate is None else torch.empty_like(self.gate),
             "w_qkv": torch.empty(self.w_qkv.shape, dtype=f32, device=dy.device),
             "w_out": torch.empty(self.w_out.shape, dtype=f32, device=dy.device)}
        fdp.op_block_join_bwd(dy, du_next, self.h_kept, self.b_kept, dh, self.db, post_gain=self.post_gain,
                              pre_gain=self.pre_gain, gate=self.gate, gate_tokens=self.gate_tokens,
                              scale=self.scale, r_post=self.r_post, r_pre=self.r_pre,
                              d_post=g["post_gain"], d_pre=g["pre_gain"], d_gate=g["gate"],
                              workspace=self.join_work)
        out = self.out.view(self.tokens, self.inner)
        self._linear(self.db, self.w_out_t, self.dout.view(self.tokens, self.inner))
        self._linear(self.db.t().contiguous(), out.t().contiguous(), g["w_out"])
        fdp.op_span_attention_bwd(*self._heads(self.qkv), self.spans, self.out, self.lse, self.dout,
                                  *self._heads(self.dqkv), workspace=self.work[1], err=self.err)
        self._linear(self.dqkv, self.w_qkv_t, du)
        fdp.op_checkpoint_load(self.u_kept, self.u_t, transposed=True)
        self._linear(self.dqkv.t().contiguous(), self.u_t, g["w_qkv"])
        return dh, du, g

    def check(self) -> None:
        """Raises if a kernel of an earlier call gave up a wait (synchronises)."""
        code = int(self.err)
        if code:
            raise RuntimeError(f"residual attention: status word {code}")
