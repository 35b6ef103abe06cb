"""A hybrid schedule's stack through the library alone (Section 3.3: the
sparse backbone with a few layers replaced by standard multi-head attention).

The schedule is a list whose entries are sparse layer codes (hypercube layers
or hcmix.LAYER_NEAR) or "attn".  Runs of sparse layers are one hcmix stack
each; an attention layer is the library's linear map (query/key/value
projection), attention core and linear map (output projection); windows past
the fixed ones (256 positions, a multiple of 32, head dimension 64), fewer
key/value heads than query heads (kv_heads) and stacks that are not causal,
whose attention is not either, take the attention of any length.  Backward:
each sparse run's dX chain (hcmix_stack_backward_data), each attention
layer's three backward products, and at the end the weight gradients of all
sparse layers in one hcmix_stack_weight_gradients call.  No arithmetic is
done here: every step is a library call on device tensors.

    h = HybridStack(schedule, w_self, w_off, attn_w, heads)
    y = h.forward(x)             # x [batch, n, width] bf16
    dx = h.backward(dy)          # then h.dw_self, h.dw_off, h.dw_attn (fp32)

An attention layer's weights are (wqkv [(heads + 2 kv_heads) * head_dim, width],
wout [width, heads * head_dim]).  rotary: a dict of hcmix.rotary's arguments
(freqs, and layout and scale where they differ from its own), applied to queries
and keys.  Position by position, over caches of the sparse layers' inputs and
of keys and values in 8 bits (causal stacks):

    d = h.decoder(batch, n)
    y = d.step(x, pos)           # x [batch, width], pos = 0, 1, ...
"""
from __future__ import annotations

import torch

from . import hcmix


class HybridStack:
    def __init__(self, schedule, w_self, w_off, attn_w, heads, causal=True, kv_heads=None,
                 rotary=None):
        self.schedule = list(schedule)
        self.w_self, self.w_off = list(w_self), list(w_off)
        self.attn_w = [tuple(p) for p in attn_w]
        self.heads = heads
        self.kv_heads = heads if kv_heads is None else kv_heads
        self.rotary = rotary
        self.causal = causal
        self.segments = []
        cur, ns, na = [], 0, 0
        for e in self.schedule:
            if e == "attn":
                if cur:
                    self.segments.append(("sparse", cur))
                self.segments.append(("attn", na))
                cur, na = [], na + 1
            else:
                cur.append((ns, e))
                ns += 1
        if cur:
            self.segments.append(("sparse", cur))
        if na != len(self.attn_w) or ns > len(self.w_self):
            raise ValueError("schedule does not match the weights given")
        self.num_sparse = ns
        self._saved = []
        self._dw_in = []
        self.dw_self = self.dw_off = self.dw_attn = None

    # ---- an attention layer's parts ----

    def head_dim(self, layer):
        return self.attn_w[layer][0].shape[0] // (self.heads + 2 * self.kv_heads)

    def _split(self, packed):
        """Queries, keys and values of packed [batch, n, heads + 2 kv_heads, hd]."""
        return packed.split([self.heads, self.kv_heads, self.kv_heads], 2)

    def _rotate(self, packed, positions=None, inverse=False):
        """Queries and keys turned in place."""
        qk = packed[:, :, :self.heads + self.kv_heads]
        hcmix.rotary(qk, positions=positions, inverse=inverse, out=qk, **self.rotary)

    def _fixed_window(self, n, hd):
        return (self.causal and self.kv_heads == self.heads and hd == 64 and n % 32 == 0
                and n <= 256)

    # ---- one segment at a time (so that a caller can time each) ----

    def forward_segment(self, k, x):
        kind, arg = self.segments[k]
        if kind == "sparse":
            xs = hcmix.stack_forward(x, [self.w_self[j] for j, _ in arg],
                                     [self.w_off[j] for j, _ in arg], [c for _, c in arg],
                                     self.causal)
            self._saved.append(xs)
            return xs[-1]
        wqkv, wout = self.attn_w[arg]
        batch, n, width = x.shape
        hd = self.head_dim(arg)
        qkv = hcmix.linear_forward(x.view(batch * n, width), wqkv)
        packed = qkv.view(batch, n, -1, hd)
        if self.rotary is not None:
            self._rotate(packed)
        if self._fixed_window(n, hd):
            o, lse = hcmix.attention_forward(qkv.view(batch, n, 3, self.heads, hd))
        else:
            o, lse = hcmix.grouped_attention_forward(*self._split(packed), causal=self.causal)
        y = hcmix.linear_forward(o.view(batch * n, self.heads * hd), wout)
        self._saved.append((x, qkv, o, lse))
        return y.view(batch, n, -1)

    def backward_segment(self, k, g):
        kind, arg = self.segments[k]
        sv = self._saved[k]
        if kind == "sparse":
            g_out = g
            g, grads = hcmix.stack_backward_data([self.w_self[j] for j, _ in arg],
                                                 [self.w_off[j] for j, _ in arg],
                                                 [c for _, c in arg], g_out, self.causal)
            self._dw_in.append((arg, sv[:len(arg)], [*grads, g_out]))
            return g
        x, qkv, o, lse = sv
        wqkv, wout = self.attn_w[arg]
        batch, n, width = x.shape
        hd = self.head_dim(arg)
        rows = batch * n
        d_o, d_wout = hcmix.linear_backward(o.view(rows, -1), wout, g.reshape(rows, -1))
        d_o = d_o.view(batch, n, self.heads, hd)
        if self._fixed_window(n, hd):
            dqkv = hcmix.attention_backward(qkv.view(batch, n, 3, self.heads, hd), o, lse, d_o)
        else:
            dqkv = torch.empty_like(qkv)
            dq, dk, dv = self._split(dqkv.view(batch, n, -1, hd))
            hcmix.grouped_attention_backward(*self._split(qkv.view(batch, n, -1, hd)), o, lse, d_o,
                                             causal=self.causal, dq=dq, dk=dk, dv=dv)
        if self.rotary is not None:
            self._rotate(dqkv.view(batch, n, -1, hd), inverse=True)
        dx, d_wqkv = hcmix.linear_backward(x.view(rows, width), wqkv, dqkv.view(rows, -1))
        self.dw_attn[arg] = (d_wqkv, d_wout)
        return dx.view(batch, n, width)

    def sparse_weight_gradients(self):
        """All sparse layers' weight gradients in one library call (fp32)."""
        xs, gs, codes, order = [], [], [], []
        for arg, xin, gout in self._dw_in:
            xs += xin
            gs += gout
            codes += [c for _, c in arg]
            order += [j for j, _ in arg]
        dws, dwo = hcmix.stack_weight_gradients(xs, gs, codes, self.causal) if xs else ([], [])
        self.dw_self = [None] * self.num_sparse
        self.dw_off = [None] * self.num_sparse
        for k, j in enumerate(order):
            self.dw_self[j], self.dw_off[j] = dws[k], dwo[k]

    # ---- whole step ----

    def forward(self, x):
        self._saved = []
        for k in range(len(self.segments)):
            x = self.forward_segment(k, x)
        return x

    def backward(self, dy):
        self._dw_in = []
        self.dw_attn = [None] * len(self.attn_w)
        g = dy
        for k in reversed(range(len(self.segments))):
            g = self.backward_segment(k, g)
        self.sparse_weight_gradients()
        return g

    # ---- position by position ----

    def decoder(self, batch, n, device="cuda"):
        """The stack over windows of n positions, one position at a time."""
        return HybridDecoder(self, batch, n, device)


class HybridDecoder:
    """Caches and buffers of a causal hybrid stack for `batch` windows of n.

    The linear maps take an even number of rows: an odd batch has one row more in
    the attention layers' buffers, which nothing reads."""

    def __init__(self, stack, batch, n, device):
        if not stack.causal:
            raise ValueError("decoder: the stack is not causal")
        self.stack, self.batch, self.n = stack, batch, n
        bf, rows = torch.bfloat16, batch + batch % 2
        # row p: p for every window, the positions of a step and (p + 1) its lengths
        self._at = torch.arange(n + 1, dtype=torch.int32, device=device)[:, None].repeat(1, batch)
        self._parts = []
        for kind, arg in stack.segments:
            if kind == "sparse":
                codes = [c for _, c in arg]
                ws, wo = ([w[j] for j, _ in arg] for w in (stack.w_self, stack.w_off))
                cache = hcmix.alloc_decode_cache(batch, n, ws[0].shape[0], codes, bf, device)
                self._parts.append((ws, wo, codes, cache))
                continue
            wqkv, wout = stack.attn_w[arg]
            hd = stack.head_dim(arg)
            cache = hcmix.alloc_kv_cache(batch, n, stack.kv_heads, hd, device)
            bufs = [torch.zeros((rows, w), dtype=bf, device=device)
                    for w in (wqkv.shape[1], wqkv.shape[0], wout.shape[1])]
            self._parts.append((wqkv, wout, hd, cache, *bufs))

    def step(self, x, pos):
        """Position pos of every window (in order 0, 1, ...): x and the result are
        [batch, width]."""
        if not 0 <= pos < self.n:
            raise ValueError(f"pos: {pos}, expected 0 .. {self.n - 1}")
        s, batch = self.stack, self.batch
        at, lengths = self._at[pos], self._at[pos + 1]
        for (kind, _), part in zip(s.segments, self._parts):
            if kind == "sparse":
                ws, wo, codes, cache = part
                x = hcmix.decode_step(x, ws, wo, codes, self.n, pos, cache)
                continue
            wqkv, wout, hd, cache, xin, qkv, o = part
            if batch % 2:
                own = xin[:batch]
                if x.shape != own.shape or x.dtype != own.dtype:     # copy_ would make it fit
                    raise ValueError(f"x: shape {tuple(x.shape)} and dtype {x.dtype}, expected "
                                     f"{tuple(own.shape)} and {own.dtype}")
                own.copy_(x)
                x = xin
            hcmix.linear_forward(x, wqkv, out=qkv)
            packed = qkv[:batch].view(batch, 1, -1, hd)
            if s.rotary is not None:
                s._rotate(packed, positions=at.view(batch, 1))
            q, k, v = s._split(packed)
            hcmix.kv_cache_append(k, v, at, cache, self.n)
            hcmix.kv_cache_attention(q, lengths, cache, self.n, s.kv_heads, max_length=pos + 1,
                                     out=o[:batch].view(batch, 1, s.heads, hd))
            x = hcmix.linear_forward(o, wout)[:batch]
        return x
