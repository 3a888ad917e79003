"""One attention layer's cache of bounded size for streams that never end.

The decoder's own caches keep the last W chunks. A BoundedStream keeps, in the same memory for
any length of stream, the entries that attention has used most: each step turns the new queries
and keys by their positions, puts the new keys and values into the slots of the entries with the
least accumulated weight, and attends over the slots, adding to their weights. A step is three
library calls (fd_op_rotary, fd_op_cache_insert, fd_op_cache_attention) on buffers that are
allocated when a step size first comes up, so that once the cache is full steps can be captured in
a CUDA graph. The buffers of the last few step sizes are kept, and those of captured steps.
"""
from __future__ import annotations

import torch

from . import flashdec as fdp


class BoundedStream:
    """Caches of `streams` streams with `capacity` slots for each KV group.

    plan: the Rotary that turns queries and keys (None: they come turned). sinks, recent: entries at
    positions below `sinks` or among the last `recent` before the step's first token are given up last;
    recent is half of the capacity by default. (With none of the newest protected, totals that only
    grow give up the entries that came last first, and the cache stays as it was when it filled up.)
    decay: the weights gathered so far are multiplied by it before a step's are added.

    The calls run on the current stream; the tensors that they are given have to be ready on it."""

    KEPT_SIZES = 4  # step sizes whose buffers are kept, besides those of captured steps

    def __init__(self, streams, heads, groups, head_dim, capacity, dtype=torch.bfloat16, plan=None,
                 sinks=4, recent=None, decay=1.0, device="cuda"):
        self.heads, self.plan = heads, plan
        self._recent_given = recent is not None
        self.recent = recent if self._recent_given else capacity // 2
        self.sinks, self.decay = sinks, decay
        shape = (streams, groups, capacity)
        k = torch.zeros(*shape, head_dim, dtype=dtype, device=device)
        self.cache = fdp.Cache(k, torch.zeros_like(k),
                               torch.full(shape, -1, dtype=torch.int32, device=device),
                               torch.zeros(shape, device=device))
        self.filled = 0  # slots that may hold something: new tokens take empty slots in order
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self._buffers: dict = {}
        self._streams: dict = {}      # the streams that have used each buffer
        self._sizes: dict = {}        # the buffers of each step size, the one used last at the end
        self._latest = self._marked = None
        self._captured: set = set()   # step sizes that graphs hold

    def _begin(self, n):
        """A step of n tokens begins: lets go of the buffers of the size that was used least recently
        when there are more than KEPT_SIZES. A captured step's stay: its graph holds their addresses."""
        self._here = here = fdp._stream_on(self.cache.device, None)
        capturing = torch.cuda.is_current_stream_capturing()
        if capturing:
            self._captured.add(n)
        # the buffers of the last step that came to its end know the stream that it ran on
        self._moved = self._marked != (n, here) and not capturing
        self._marked = None
        if n == self._latest:
            return
        self._latest = n
        self._sizes[n] = self._sizes.pop(n, set())
        if len(self._sizes) > self.KEPT_SIZES:
            for m in [m for m in self._sizes if m not in self._captured][:-self.KEPT_SIZES]:
                for key in self._sizes.pop(m):
                    del self._buffers[key], self._streams[key]

    def _new(self, key, shape, dtype):
        self._sizes[self._latest].add(key)
        self._streams[key] = {self._here}
        t = self._buffers[key] = torch.empty(shape, dtype=dtype, device=self.err.device)
        return t

    def _mark(self, key, t):
        """The current stream uses the buffer: its memory, once it is let go of, is not given to anyone
        else before the stream is through with it."""
        if self._here not in self._streams[key]:
            t.record_stream(torch.cuda.current_stream(t.device))
            self._streams[key].add(self._here)

    def _buffer(self, name, shape, dtype):
        """A buffer of the step, allocated when its size first comes up."""
        key = (name, tuple(shape))
        t = self._buffers.get(key)
        if t is None:
            return self._new(key, shape, dtype)
        if self._moved:
            self._mark(key, t)
        return t

    def step(self, q, k, v, pos, axes_pos=None, whole_chunk=False):
        """Attention of q [streams][n][heads][head_dim] over the cache with the new k, v
        [streams][n][groups][head_dim] in it; returns out like q (a buffer that the next step of
        n tokens overwrites). pos int32 [streams][n]: ascending positions, those of the rotary
        embedding too unless axes_pos int32 [streams][n][axes] gives its own. whole_chunk: every
        token sees all n new tokens, as in the decoder's chunks; else a token sees no later one."""
        S, n, H, D = q.shape
        if n == 0:
            return torch.empty_like(q)
        c = self.cache
        G = c.groups
        self._begin(n)
        if self.plan is not None:
            turn = (pos if axes_pos is None else axes_pos).reshape(S * n, -1)
            q_t, k_t = (self._buffer("q", q.shape, q.dtype), self._buffer("k", k.shape, k.dtype))
            fdp.op_rotary(self.plan, turn, q.reshape(S * n, H, D), q_t.view(S * n, H, D),
                          k.reshape(S * n, G, D), k_t.view(S * n, G, D))
            q, k = q_t, k_t
        if k.stride() != v.stride() and not fdp._same_steps(k.stride(), v.stride(), k.shape):
            # (the insert takes one set of strides: what comes out of the rotation is contiguous, values
            # that are a part of a fused projection are not)
            k, v = (self._buffer(name, x.shape, x.dtype).copy_(x)
                    if x.get_device() == c.device and not x.is_contiguous() else x
                    for name, x in (("k", k), ("v", v)))
        slots = self._buffer("slots", (S, G, n), torch.int32)
        fdp.op_cache_insert(c, k, v, pos, slots, sinks=self.sinks, recent=self.recent)
        self.filled = min(c.capacity, self.filled + n)
        out = self._buffer("out", (S, n, H, D), c.dtype)
        # What a call needs does not only grow with the slots: take the larger of now and full. (One
        # workspace for each step size: a captured step keeps its own.)
        need = c.workspace_bytes(self.filled, H, n)
        if self.filled < c.capacity:
            need = max(need, c.workspace_bytes(c.capacity, H, n))
        work = self._buffers.get(("work", n))
        if work is None or work.numel() < need:
            work = self._new(("work", n), (need,), torch.uint8)
        elif self._moved:
            self._mark(("work", n), work)
        q_pos = pos[:, -1:].expand(S, n).contiguous() if whole_chunk else pos
        fdp.op_cache_attention(c, q, q_pos, out, weight_out=c.weight, used=self.filled,
                               decay=self.decay, workspace=work, err=self.err)
        self._marked = None if n in self._captured else (n, self._here)
        return out

    def compact(self, capacity, now):
        """A BoundedStream of fewer slots that holds this one's most used entries; now int32
        [streams]: the next token's position (recency counts from it, and is the new stream's: half of
        its capacity unless this stream was given another)."""
        c = self.cache
        used = self.filled
        new = BoundedStream(c.streams, self.heads, c.groups, c.head_dim, capacity, c.dtype,
                            self.plan, self.sinks, self.recent if self._recent_given else None,
                            self.decay, self.err.device)
        came = torch.empty(c.streams, c.groups, capacity, dtype=torch.int32,
                           device=self.err.device)
        # slots past the filled ones are empty, so they may count where they are needed
        fdp.op_cache_compact(c, new.cache, now, came, used=max(used, capacity), sinks=self.sinks,
                             recent=new.recent)
        new.filled = min(capacity, used)
        return new

    def check(self) -> None:
        """Raises if a kernel of an earlier step gave up a wait (synchronises)."""
        code = int(self.err)
        if code:
            raise RuntimeError(f"bounded cache: status word {code}")
