"""Attention blocks over a convolution's feature map: the operators of
``attention.py`` and ``linear_attention.py`` together, as a network with a
convolution backbone uses them.

    features = plan.conv2d(x, wspec, bias)            # [n, c, h, w], fp32
    block = AttentionBlock(n, c, h, w, heads=8, heads_k=4, dim=32)
    y, saved = block.forward(features, save=True)
    dx, grads = block.backward(dy, features, saved)

The map becomes bf16 tokens in the layer norm (its layout and type change on
the way), queries and keys are rotated by their row and column, every token
attends to all others by differential attention, and the result is added to
the map.  The projections are plain matrix products.

``LinearAttentionBlock`` goes over the frames of a video instead, each pixel
after those before it, with a state of fixed size for all the frames so far:

    block = LinearAttentionBlock(n, c, h, w, heads=8, heads_k=4, dim=32, dim_v=64)
    y0, state = block.forward(frame0)
    y1, state = block.forward(frame1, state, frame=1)
"""
from __future__ import annotations

from . import (DiffAttention, LinearAttention, head_norm_rotary, head_norm_rotary_backward, layer_norm, layer_norm_backward,
               rotary)


class AttentionBlock:
    def __init__(self, batch, channels, height, width, heads, heads_k, dim, base=100.0, device=None, seed=0):
        import torch
        if dim % 4:
            raise ValueError("dim must be a multiple of 4: half of its pairs follow the row, half the column")
        dev = torch.device("cuda", torch.cuda.current_device() if device is None else int(device))
        self.shape = (batch, channels, height, width)
        self.heads, self.heads_k, self.dim = heads, heads_k, dim
        tokens, dim_v = height * width, 2 * dim
        self.attention = DiffAttention(batch, tokens, tokens, heads, heads_k, dim, dim_v, dtype=torch.bfloat16,
                                       device=dev.index)
        self.widths = [heads * 2 * dim, heads_k * 2 * dim, heads_k * dim_v]
        gen = torch.Generator(device=dev).manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=gen, device=dev) * cols ** -0.5).bfloat16()

        self.params = {"norm_weight": torch.ones(channels, device=dev), "norm_bias": torch.zeros(channels, device=dev),
                       "project": matrix(sum(self.widths), channels), "merge": matrix(channels, heads * dim_v),
                       "lam": torch.full((heads,), 0.5, device=dev)}
        rows = torch.arange(height, dtype=torch.int32, device=dev)
        cols = torch.arange(width, dtype=torch.int32, device=dev)
        self.positions = torch.stack(torch.meshgrid(rows, cols, indexing="ij"), -1).view(tokens, 2).contiguous()
        self.sections = (dim // 4, dim // 4)
        self.freqs = torch.cat([base ** (-torch.arange(p, device=dev, dtype=torch.float32) / p) for p in self.sections])

    def _split(self, qkv):
        n, s, _ = qkv.shape
        q, k, v = qkv.split(self.widths, -1)
        return (q.view(n, s, self.heads, 2, self.dim), k.view(n, s, self.heads_k, 2, self.dim),
                v.view(n, s, self.heads_k, 2 * self.dim))

    def forward(self, x, save=False, workspace=None):
        """x [n, c, h, w] (fp32) -> x + attention(norm(x)), and with save=True
        what backward needs.  `workspace`: as the attention's; by default each
        call allocates its own, so that calls on several streams stay apart."""
        import torch
        p = self.params
        tokens, mean, rstd = layer_norm(x, p["norm_weight"], p["norm_bias"], layout="first", out_layout="last",
                                        out_dtype=torch.bfloat16, return_stats=True)
        q, k, v = self._split(tokens @ p["project"].t())
        q, k = rotary(q, self.positions, self.freqs, self.sections, other=k)
        args = (q, k, v, p["lam"])
        if save:
            o, kept = self.attention.forward(*args, workspace=workspace, save=True)
        else:
            o, kept = self.attention.forward(*args, workspace=workspace), None
        y = (o.flatten(2) @ p["merge"].t()).transpose(1, 2).reshape(x.shape).float() + x
        return (y, (tokens, mean, rstd, args, o, kept)) if save else y

    def backward(self, dy, x, saved, workspace=None):
        """dx and the gradients of the parameters (a dict like `params`)."""
        import torch
        p = self.params
        tokens, mean, rstd, args, o, kept = saved
        n, s, c = tokens.shape
        dout = dy.flatten(2).transpose(1, 2).to(torch.bfloat16).reshape(n * s, c)
        grads = {"merge": dout.t() @ o.view(n * s, -1)}
        do = (dout @ p["merge"]).view(o.shape)
        dq, dk, dv, grads["lam"] = self.attention.backward(do, *args, kept, workspace=workspace)
        dqkv = torch.empty((n, s, sum(self.widths)), dtype=torch.bfloat16, device=x.device)
        q, k, v = self._split(dqkv)
        rotary(dq, self.positions, self.freqs, self.sections, other=dk, inverse=True, out=q, out_other=k)
        v.copy_(dv)
        dqkv = dqkv.view(n * s, -1)
        grads["project"] = dqkv.t() @ tokens.view(n * s, c)
        dtokens = (dqkv @ p["project"]).view(n, s, c)
        dx, grads["norm_weight"], grads["norm_bias"] = layer_norm_backward(
            dtokens, x, mean, rstd, p["norm_weight"], layout="first", out_layout="last")
        return dx + dy, grads


class LinearAttentionBlock:
    """y = x + linear attention(norm(x)) over the frames of a stream of feature
    maps.  The pixels of a frame follow one another row by row; queries and keys
    are normed by head and rotated by their frame, row and column, and the state
    [n, heads_k, dim, dim_v] (fp32) that a call returns is what the next frame's
    begins with."""

    def __init__(self, batch, channels, height, width, heads, heads_k, dim, dim_v, base=100.0, device=None, seed=0):
        import torch
        if dim % 2 or dim < 6:
            raise ValueError("dim must be even and at least 6: its pairs follow the frame, the row and the column")
        dev = torch.device("cuda", torch.cuda.current_device() if device is None else int(device))
        self.shape = (batch, channels, height, width)
        self.heads, self.heads_k, self.dim, self.dim_v = heads, heads_k, dim, dim_v
        tokens = height * width
        self.frame, self.pixel = (LinearAttention(batch, s, heads, heads_k, dim, dim_v, dtype=torch.bfloat16,
                                                  device=dev.index) for s in (tokens, 1))
        self.widths = [heads * dim, heads_k * dim, heads_k * dim_v]
        gen = torch.Generator(device=dev).manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=gen, device=dev) * cols ** -0.5).bfloat16()

        self.params = {"norm_weight": torch.ones(channels, device=dev), "norm_bias": torch.zeros(channels, device=dev),
                       "project": matrix(sum(self.widths), channels), "merge": matrix(channels, heads * dim_v),
                       "q_weight": torch.ones(dim, device=dev), "k_weight": torch.ones(dim, device=dev)}
        # heads that remember from 8 pixels to 8 frames' worth of them
        spread = torch.arange(heads_k, device=dev, dtype=torch.float32) / max(heads_k - 1, 1)
        self.log_decay = -1 / (8 * float(max(tokens, 1)) ** spread)
        rows = torch.arange(height, dtype=torch.int32, device=dev)
        cols = torch.arange(width, dtype=torch.int32, device=dev)
        grid = torch.stack(torch.meshgrid(rows, cols, indexing="ij"), -1).view(tokens, 2)
        self.positions = torch.cat([torch.zeros_like(grid[:, :1]), grid], -1)
        third = dim // 6
        self.sections = (dim // 2 - 2 * third, third, third)
        self.freqs = torch.cat([base ** (-torch.arange(p, device=dev, dtype=torch.float32) / p) for p in self.sections])

    def new_state(self):
        """The state before the first frame."""
        import torch
        return torch.zeros(self.frame.state_shape, dtype=torch.float32, device=self.log_decay.device)

    def _positions(self, frame):
        if not frame:
            return self.positions
        positions = self.positions.clone()
        positions[:, 0] = frame
        return positions

    def _split(self, qkv):
        n, s, _ = qkv.shape
        q, k, v = qkv.split(self.widths, -1)
        return (q.view(n, s, self.heads, self.dim), k.view(n, s, self.heads_k, self.dim),
                v.view(n, s, self.heads_k, self.dim_v))

    def _turned(self, qkv, positions):
        q, k, v = self._split(qkv)
        p = self.params
        q, k = head_norm_rotary(q, p["q_weight"], positions, self.freqs, self.sections, other=k, other_weight=p["k_weight"])
        return q, k, v

    def forward(self, x, state=None, frame=0, save=False, workspace=None):
        """(y, state behind this frame) of x [n, c, h, w] (fp32), the stream's
        `frame`-th, from the state before it (None: zero, of a first frame); with
        save=True also what backward needs (with a copy of `state`, as step writes
        states in place).  `workspace`: as the attention's; by default each call
        allocates its own."""
        import torch
        p = self.params
        if save and state is not None:
            state = state.clone()
        tokens, mean, rstd = layer_norm(x, p["norm_weight"], p["norm_bias"], layout="first", out_layout="last",
                                        out_dtype=torch.bfloat16, return_stats=True)
        positions = self._positions(frame)
        qkv = tokens @ p["project"].t()
        args = self._turned(qkv, positions)
        o, last = self.frame.forward(*args, self.log_decay, state=state, return_state=True, workspace=workspace)
        y = (o.flatten(2) @ p["merge"].t()).transpose(1, 2).reshape(x.shape).float() + x
        return (y, last, (tokens, mean, rstd, positions, qkv, args, state, o)) if save else (y, last)

    def step(self, x, state, at):
        """y [n, c] of one pixel x [n, c] (fp32) at (frame, row, column), an int32
        tensor of three on the device, from the pixels before it; `state` is
        updated in place."""
        import torch
        p = self.params
        tokens = layer_norm(x.unsqueeze(1), p["norm_weight"], p["norm_bias"], out_dtype=torch.bfloat16)
        q, k, v = self._turned(tokens @ p["project"].t(), at.view(1, 3))
        o, _ = self.pixel.forward(q, k, v, self.log_decay, state=state, out_state=state)
        return (o.flatten(1) @ p["merge"].t()).float() + x

    def backward(self, dy, x, saved, dstate=None, workspace=None):
        """dx, the gradients of the parameters (a dict like `params`) and that of
        the state that forward was given (None without one), from dy and, where
        the state it returned was used, `dstate`, that state's gradient."""
        import torch
        p = self.params
        tokens, mean, rstd, positions, qkv, args, state, o = saved
        n, s, c = tokens.shape
        dout = dy.flatten(2).transpose(1, 2).to(torch.bfloat16).reshape(n * s, c)
        grads = {"merge": dout.t() @ o.view(n * s, -1)}
        do = (dout @ p["merge"]).view(o.shape)
        dq, dk, dv, first = self.frame.backward(do, *args, self.log_decay, state=state, dstate=dstate, workspace=workspace)
        dqkv = torch.empty((n, s, sum(self.widths)), dtype=torch.bfloat16, device=x.device)
        q, k, _ = self._split(qkv)
        to_q, to_k, to_v = self._split(dqkv)
        _, grads["q_weight"], _, grads["k_weight"] = head_norm_rotary_backward(
            dq, q, p["q_weight"], positions, self.freqs, self.sections, dy_other=dk, other=k, other_weight=p["k_weight"],
            out=to_q, out_other=to_k)
        to_v.copy_(dv)
        dqkv = dqkv.view(n * s, -1)
        grads["project"] = dqkv.t() @ tokens.view(n * s, c)
        dtokens = (dqkv @ p["project"]).view(n, s, c)
        dx, grads["norm_weight"], grads["norm_bias"] = layer_norm_backward(
            dtokens, x, mean, rstd, p["norm_weight"], layout="first", out_layout="last")
        return dx + dy, grads, first
