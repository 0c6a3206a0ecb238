"""An attention block over a convolution's feature map: the operators of
``attention.py`` together, as a network with a convolution backbone uses them.

    features = plan.conv2d(x, wspec, bias)            # [n, c, h, w], fp32
    block = AttentionBlock(n, c, h, w, heads=8, heads_k=4, dim=32)
    y, saved = block.forward(features, save=True)
    dx, grads = block.backward(dy, features, saved)

The map becomes bf16 tokens in the layer norm (its layout and type change on
the way), queries and keys are rotated by their row and column, every token
attends to all others by differential attention, and the result is added to
the map.  The projections are plain matrix products.
"""
from __future__ import annotations

from . import DiffAttention, layer_norm, layer_norm_backward, rotary


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
