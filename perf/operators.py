"""The calls of the attention block that follows a convolution backbone: layer
norm, rotary positions over several axes, and differential attention, over the
range of sizes that they are called with.

Each case is one pass through one operator.  A training pass returns the
output and every gradient.  Where `own` is false the operators are computed
in their plain form, elementary torch operations in 32 bits; where it is true,
by the library.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def _norm(name, n, c, s, layout, dtype, out_layout=None, out_dtype=None, train=False):
    return {"name": name, "op": "norm", "n": n, "c": c, "s": s, "layout": layout, "dtype": dtype,
            "out_layout": out_layout or layout, "out_dtype": out_dtype or dtype, "train": train}


def _rotary(name, n, grid, hq, hk, d, sections, dtype, interleaved=False, inverse=False):
    """`grid`: the extents of the axes, as a text ("16x24x24"); `sections`:
    rotated pairs per axis, as a text."""
    return {"name": name, "op": "rotary", "n": n, "grid": grid, "hq": hq, "hk": hk, "d": d, "sections": sections,
            "dtype": dtype, "interleaved": interleaved, "inverse": inverse}


def _attn(name, n, sq, sk, hq, hk, d, dv, dtype, causal=False, lengths="full", packed=False, train=False):
    """`lengths`: "full" (no key lengths given), "cache" (each sequence has
    filled between half of the cache and all of it) or "ragged" (any length,
    one sequence empty)."""
    return {"name": name, "op": "attn", "n": n, "sq": sq, "sk": sk, "hq": hq, "hk": hk, "d": d, "dv": dv,
            "dtype": dtype, "causal": causal, "lengths": lengths, "packed": packed, "train": train}


def listed():
    return [
        # One image's last feature map (512 channels of 14 x 14) into tokens:
        # a few microseconds, all latency.
        _norm("norm_tokens_512x14", 1, 512, 14 * 14, "first", "fp32", out_layout="last", out_dtype="bf16"),
        # A batch of the 256-channel 56 x 56 feature maps, kept as maps, as
        # between two convolutions.
        _norm("norm_map_256x56", 32, 256, 56 * 56, "first", "fp32"),
        # Training step of a norm over tokens, the width of an attention block.
        _norm("norm_train_tokens_1024", 32, 1024, 28 * 28, "last", "bf16", train=True),
        # Training step on feature maps of odd sizes.
        _norm("norm_train_map_ragged", 5, 77, 57 * 75, "first", "fp32", train=True),
        # Rows and columns of one image's tokens: latency.
        _rotary("rotary_image_14x14", 1, "14x14", 16, 16, 32, "8,8", "fp32"),
        # Time, rows and columns of a batch of clips, shared key heads.
        _rotary("rotary_video_16x32x32", 4, "16x32x32", 32, 8, 64, "8,12,12", "bf16"),
        # One new token per sequence over a long cache: serving.
        _attn("attn_decode_8k", 16, 1, 8192, 16, 4, 64, 128, "bf16", causal=True, lengths="cache"),
        # The tokens of a 28 x 28 map, every one seeing every other, from one
        # packed projection.
        _attn("attn_image_28x28", 8, 784, 784, 8, 8, 64, 128, "bf16", packed=True),
        # A long causal sequence with shared key heads.
        _attn("attn_causal_8k", 1, 8192, 8192, 16, 4, 64, 128, "bf16", causal=True),
        # Small heads in fp32, as the convolutions give them, sequences of
        # every length in one batch.
        _attn("attn_train_fp32_ragged", 6, 301, 301, 6, 3, 32, 64, "fp32", lengths="ragged", train=True),
        # Training on the tokens of 56 x 56 maps: the largest.
        _attn("attn_train_56x56", 4, 56 * 56, 56 * 56, 8, 8, 64, 128, "bf16", packed=True, train=True),
        # Training with wide heads, causal, odd length.
        _attn("attn_train_causal_wide", 2, 1999, 1999, 8, 4, 128, 256, "bf16", causal=True, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_norm(rng):
    layout = rng.choice(["first", "last"])
    dtype = rng.choice(["fp32", "bf16"])
    c = _log_int(rng, 16, 2048)
    s = _log_int(rng, 49, 112 * 112)
    n = max(1, min(64, _log_int(rng, 1 << 17, 1 << 25) // (c * s)))
    train = rng.random() < 0.5
    to_tokens = layout == "first" and not train and rng.random() < 0.5
    return _norm("", n, c, s, layout, dtype, out_layout="last" if to_tokens else layout,
                 out_dtype="bf16" if to_tokens else dtype, train=train)


def _draw_rotary(rng):
    d = rng.choice([32, 64, 128])
    axes = rng.choice([1, 2, 3])
    if axes == 1:
        grid, sections = [_log_int(rng, 1, 1024)], [d // 2]
    elif axes == 2:
        grid, sections = [_log_int(rng, 2, 64) for _ in range(2)], [d // 4, d // 4]
    else:
        grid = [_log_int(rng, 1, 16)] + [_log_int(rng, 2, 32) for _ in range(2)]
        sections = [d // 8, 3 * d // 16, 3 * d // 16]
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4])
    tokens = math.prod(grid)
    n = max(1, min(16, (1 << 26) // (tokens * (hq + hk) * d)))
    return _rotary("", rng.randint(1, n), "x".join(map(str, grid)), hq, hk, d, ",".join(map(str, sections)),
                   rng.choice(["fp32", "bf16"]), interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5)


def _draw_attn(rng):
    d = rng.choice([32, 64, 64, 128])
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4])
    kind = rng.choice(["decode", "forward", "train"])
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    if kind == "decode":
        sk = _log_int(rng, 256, 16384)
        n = max(1, min(32, _log_int(rng, 1 << 14, 1 << 18) // sk))
        return _attn("", n, rng.choice([1, 1, 2, 5]), sk, hq, hk, d, 2 * d, dtype, causal=True, lengths="cache")
    # products a head's width deep, below the largest listed case's
    most = 2e10 if dtype == "bf16" else 4e9
    s = _log_int(rng, 17, min(4096, math.sqrt(most / (hq * d))))
    n = _log_int(rng, 1, max(1, min(16, most / (s * s * hq * d))))
    return _attn("", n, s, s, hq, hk, d, 2 * d, dtype, causal=rng.random() < 0.5,
                 lengths=rng.choice(["full", "ragged"]), packed=rng.random() < 0.5, train=kind == "train")


def draw(rng):
    kind = rng.choice(["norm", "rotary", "attn", "attn"])
    return {"norm": _draw_norm, "rotary": _draw_rotary, "attn": _draw_attn}[kind](rng)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _randn(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _norm_inputs(case, seed):
    gen, n, c, s = _generator(seed), case["n"], case["c"], case["s"]
    shape = (n, c, s) if case["layout"] == "first" else (n, s, c)
    # activations after a ReLU: nonnegative, mean well away from zero
    x = torch.relu(_randn(gen, shape) + 0.5).to(DTYPES[case["dtype"]])
    weight = 1.0 + 0.2 * _randn(gen, (c,))
    bias = 0.1 * _randn(gen, (c,))
    out = (n, c, s) if case["out_layout"] == "first" else (n, s, c)
    dy = _randn(gen, out, DTYPES[case["out_dtype"]]) if case["train"] else None
    return {"x": x, "weight": weight, "bias": bias, "dy": dy}


def _grid(case):
    return [int(v) for v in case["grid"].split("x")]


def _sections(case):
    return tuple(int(v) for v in case["sections"].split(","))


def _rotary_inputs(case, seed):
    gen, grid, sections = _generator(seed), _grid(case), _sections(case)
    tokens, dtype = math.prod(grid), DTYPES[case["dtype"]]
    q = _randn(gen, (case["n"], tokens, case["hq"], case["d"]), dtype)
    k = _randn(gen, (case["n"], tokens, case["hk"], case["d"]), dtype)
    ranges = [torch.arange(g, device="cuda", dtype=torch.int32) for g in grid]
    positions = torch.stack([m.reshape(-1) for m in torch.meshgrid(*ranges, indexing="ij")], dim=-1).contiguous()
    freqs = torch.cat([100.0 ** (-torch.arange(p, device="cuda", dtype=torch.float32) / p) for p in sections])
    return {"q": q, "k": k, "positions": positions, "freqs": freqs, "sections": sections}


def _attn_inputs(case, seed):
    gen, dtype = _generator(seed), DTYPES[case["dtype"]]
    n, sq, sk, hq, hk, d, dv = (case[i] for i in ("n", "sq", "sk", "hq", "hk", "d", "dv"))
    if case["packed"]:
        # q, k and v are slices of one projection's output
        wq, wk, wv = hq * 2 * d, hk * 2 * d, hk * dv
        qkv = _randn(gen, (n, sq, wq + wk + wv), dtype)
        q, k, v = qkv.split([wq, wk, wv], dim=-1)
        q, k, v = q.view(n, sq, hq, 2, d), k.view(n, sk, hk, 2, d), v.view(n, sk, hk, dv)
    else:
        q = _randn(gen, (n, sq, hq, 2, d), dtype)
        k = _randn(gen, (n, sk, hk, 2, d), dtype)
        v = _randn(gen, (n, sk, hk, dv), dtype)
    lam = (0.2 + 0.6 * torch.rand((hq,), generator=gen, device="cuda")).to(dtype)
    lengths = None
    if case["lengths"] == "cache":
        lengths = torch.randint((sk + 1) // 2, sk + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    elif case["lengths"] == "ragged":
        lengths = torch.randint(1, sk + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
        if n > 1:
            lengths[n // 2] = 0
    do = _randn(gen, (n, sq, hq, dv), dtype) if case["train"] else None
    return {"q": q, "k": k, "v": v, "lam": lam, "lengths": lengths, "do": do}


_INPUTS = {"norm": _norm_inputs, "rotary": _rotary_inputs, "attn": _attn_inputs}


def prepare(case, seed):
    state = dict(_INPUTS[case["op"]](case, seed), case=case)
    if own and case["op"] == "attn":
        import paper_2003_12621_amd as fs
        plan = fs.DiffAttention(case["n"], case["sq"], case["sk"], case["hq"], case["hk"], case["d"], case["dv"],
                                dtype=DTYPES[case["dtype"]], causal=case["causal"])
        state["plan"] = plan
        state["workspace"] = plan.new_workspace(backward=case["train"])
    return state


# ---------------------------------------------------------------- plain form

def _plain_norm(st):
    case = st["case"]
    x = st["x"].float()
    if case["layout"] == "first":
        x = x.transpose(1, 2)
    mean = x.mean(-1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(-1, keepdim=True) + EPS)
    xhat = xc * rstd
    y = xhat * st["weight"] + st["bias"]

    def laid_out(t, layout, dtype):
        return (t.transpose(1, 2) if layout == "first" else t).to(dtype).contiguous()

    out = {"y": laid_out(y, case["out_layout"], DTYPES[case["out_dtype"]])}
    if case["train"]:
        dy = st["dy"].float()
        if case["out_layout"] == "first":
            dy = dy.transpose(1, 2)
        g = dy * st["weight"]
        dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
        out["dx"] = laid_out(dx, case["layout"], DTYPES[case["dtype"]])
        out["dweight"] = (dy * xhat).sum((0, 1))
        out["dbias"] = dy.sum((0, 1))
    return out


def _turn(x, cos, sin, interleaved):
    r = cos.shape[-1]
    if interleaved:
        a, b = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        rotated = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :r], x[..., r:2 * r]
        rotated = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([rotated, x[..., 2 * r:]], dim=-1)


def _plain_rotary(st):
    case = st["case"]
    pairs = torch.cat([st["positions"][:, a:a + 1].float().expand(-1, p) for a, p in enumerate(st["sections"])], dim=1)
    angle = (pairs * st["freqs"])[:, None, :]
    cos, sin = torch.cos(angle), torch.sin(angle)
    if case["inverse"]:
        sin = -sin
    return tuple(_turn(st[i].float(), cos, sin, case["interleaved"]).to(st[i].dtype) for i in ("q", "k"))


def _visible(case, lengths, device):
    """[n or 1, 1, 1, sq, sk] truth values, or None where every key is visible."""
    if lengths is None and not case["causal"]:
        return None
    sq, sk = case["sq"], case["sk"]
    length = torch.full((1,), sk, device=device) if lengths is None else lengths
    length = length.view(-1, 1, 1).long()
    j = torch.arange(sk, device=device)
    seen = (j < length).expand(-1, sq, -1)
    if case["causal"]:
        i = torch.arange(sq, device=device)[:, None]
        seen = seen & (j <= i + length - sq)
    return seen[:, None, None]


def _plain_attn(st):
    case = st["case"]
    n, sq, sk, hq, hk, d, dv = (case[i] for i in ("n", "sq", "sk", "hq", "hk", "d", "dv"))
    g, scale = hq // hk, 1.0 / math.sqrt(d)
    dtype = st["q"].dtype
    q = st["q"].float().permute(0, 2, 3, 1, 4)                                   # n hq 2 sq d
    k = st["k"].float().permute(0, 2, 3, 1, 4).repeat_interleave(g, dim=1)        # n hq 2 sk d
    v = st["v"].float().permute(0, 2, 1, 3).repeat_interleave(g, dim=1)           # n hq sk dv
    lam = st["lam"].float().view(1, hq, 1, 1)
    s = (q @ k.transpose(-1, -2)) * scale
    seen = _visible(case, st["lengths"], q.device)
    if seen is not None:
        s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    del s
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    both = p[:, :, 0] - lam * p[:, :, 1]
    o = both @ v
    out = {"o": o.permute(0, 2, 1, 3).to(dtype).contiguous()}
    if case["train"]:
        do = st["do"].float().permute(0, 2, 1, 3)                                 # n hq sq dv
        t = do @ v.transpose(-1, -2)
        gv = both.transpose(-1, -2) @ do
        gp = torch.stack([t, -lam * t], dim=2)
        ds = p * (gp - (gp * p).sum(-1, keepdim=True)) * scale
        gq = ds @ k
        gk = ds.transpose(-1, -2) @ q
        gk = gk.view(n, hk, g, 2, sk, d).sum(2)
        gv = gv.view(n, hk, g, sk, dv).sum(2)
        out["dq"] = gq.permute(0, 3, 1, 2, 4).to(dtype).contiguous()
        out["dk"] = gk.permute(0, 3, 1, 2, 4).to(dtype).contiguous()
        out["dv"] = gv.permute(0, 2, 1, 3).to(dtype).contiguous()
        out["dlam"] = -(p[:, :, 1] * t).sum((0, 2, 3)).to(st["lam"].dtype)
    return out


# ---------------------------------------------------------------- the library

def _own_norm(st):
    import paper_2003_12621_amd as fs
    case = st["case"]
    kw = {"layout": case["layout"], "out_layout": case["out_layout"]}
    if not case["train"]:
        return {"y": fs.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS,
                                   out_dtype=DTYPES[case["out_dtype"]], **kw)}
    y, mean, rstd = fs.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS, out_dtype=DTYPES[case["out_dtype"]],
                                  return_stats=True, **kw)
    dx, dweight, dbias = fs.layer_norm_backward(st["dy"], st["x"], mean, rstd, st["weight"], **kw)
    return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}


def _own_rotary(st):
    import paper_2003_12621_amd as fs
    case = st["case"]
    return fs.rotary(st["q"], st["positions"], st["freqs"], st["sections"], other=st["k"],
                     interleaved=case["interleaved"], inverse=case["inverse"])


def _own_attn(st):
    plan, train = st["plan"], st["case"]["train"]
    args = (st["q"], st["k"], st["v"], st["lam"])
    if not train:
        return {"o": plan.forward(*args, key_lengths=st["lengths"], workspace=st["workspace"])}
    o, saved = plan.forward(*args, key_lengths=st["lengths"], workspace=st["workspace"], save=True)
    dq, dk, dv, dlam = plan.backward(st["do"], *args, saved, key_lengths=st["lengths"],
                                     workspace=st["workspace"])
    return {"o": o, "dq": dq, "dk": dk, "dv": dv, "dlam": dlam}


_PLAIN = {"norm": _plain_norm, "rotary": _plain_rotary, "attn": _plain_attn}
_OWN = {"norm": _own_norm, "rotary": _own_rotary, "attn": _own_attn}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------- work

def _pairs(case):
    """Visible (query, key) pairs per head, with key lengths at their mean."""
    sq, sk = case["sq"], case["sk"]
    length = {"full": sk, "cache": 0.75 * sk, "ragged": 0.5 * sk}[case["lengths"]]
    pairs = sq * length
    if case["causal"]:
        pairs -= sq * (sq - 1) / 2 if length >= sq else sq * length - length * (length + 1) / 2
    return case["n"] * pairs, case["n"] * length


def work(case):
    b = BYTES[case["dtype"]]
    if case["op"] == "norm":
        e, ob = case["n"] * case["c"] * case["s"], BYTES[case["out_dtype"]]
        nbytes, flops = e * (b + ob) + 8 * case["c"], 8 * e
        if case["train"]:
            nbytes, flops = nbytes + e * (ob + b) + 12 * case["c"], flops + 14 * e
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "rotary":
        grid, sections = _grid(case), _sections(case)
        tokens = math.prod(grid)
        e = case["n"] * tokens * (case["hq"] + case["hk"]) * case["d"]
        return {"bytes": 2 * b * e + 4 * len(grid) * tokens + 4 * sum(sections), "flops": 3 * e}
    n, sq, hq, hk, d, dv = (case[i] for i in ("n", "sq", "hq", "hk", "d", "dv"))
    pairs, keys = _pairs(case)
    qo = n * sq * hq * (2 * d + dv)
    kv = keys * hk * (2 * d + dv)
    nbytes, flops = b * (qo + kv), hq * pairs * (4 * d + 2 * dv)
    if case["train"]:
        # dO, dq; dk and dv over the whole key range; the output, q, k and v count once
        nbytes += b * (qo + n * case["sk"] * hk * (2 * d + dv))
        flops += hq * pairs * (12 * d + 4 * dv)
    return {"bytes": int(nbytes), "flops": int(flops)}


# ---------------------------------------------------------------- in 64 bits

def _exact_norm(case, inp):
    # the definition, and its gradient by differentiation of it
    axis = 1 if case["layout"] == "first" else 2
    x, w, b = (inp[i].double().requires_grad_(case["train"]) for i in ("x", "weight", "bias"))
    shape = [1, 1, 1]
    shape[axis] = -1
    xhat = (x - x.mean(axis, keepdim=True)) / torch.sqrt(x.var(axis, unbiased=False, keepdim=True) + EPS)
    y = xhat * w.view(shape) + b.view(shape)
    if case["out_layout"] != case["layout"]:
        y = y.transpose(1, 2).contiguous()
    out = {"y": y.detach()}
    if case["train"]:
        out["dx"], out["dweight"], out["dbias"] = torch.autograd.grad(y, (x, w, b), inp["dy"].double())
    return out


def _exact_rotary(case, inp):
    pair_axis = [a for a, p in enumerate(inp["sections"]) for _ in range(p)]
    angle = inp["positions"].double()[:, pair_axis] * inp["freqs"].double()
    if case["inverse"]:
        angle = -angle
    turn = torch.complex(torch.cos(angle), torch.sin(angle))[None, :, None, :]
    outs = []
    for name in ("q", "k"):
        x = inp[name].double()
        r = turn.shape[-1]
        first, second = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if case["interleaved"] else (x[..., :r], x[..., r:2 * r])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        y = x.clone()
        if case["interleaved"]:
            y[..., 0:2 * r:2], y[..., 1:2 * r:2] = z.real, z.imag
        else:
            y[..., :r], y[..., r:2 * r] = z.real, z.imag
        outs.append(y)
    return tuple(outs)


def _exact_attn(case, inp):
    n, sq, sk, hq, hk, d, dv = (case[i] for i in ("n", "sq", "sk", "hq", "hk", "d", "dv"))
    if n * hq * sq * sk * (4 * d + 2 * dv) * (4 if case["train"] else 1) > 1.5e13:
        return None
    scale, dev = d ** -0.5, inp["q"].device
    o = torch.zeros((n, sq, hq, dv), dtype=torch.float64, device=dev)
    grads = {i: torch.zeros(inp[i].shape, dtype=torch.float64, device=dev) for i in ("q", "k", "v", "lam")}
    for b in range(n):
        length = sk if inp["lengths"] is None else int(inp["lengths"][b])
        first = 0       # the first row that sees a key
        if case["causal"]:
            first = min(sq, max(0, sq - length))
        if length == 0 or first == sq:
            continue
        hidden = None
        if case["causal"]:
            rows = torch.arange(first, sq, device=dev)[:, None]
            hidden = torch.arange(length, device=dev)[None, :] > rows + (length - sq)
        for h in range(hq):
            kv = h * hk // hq
            qs, ks, vs, lam = (t.double().requires_grad_(case["train"]) for t in (
                inp["q"][b, first:, h], inp["k"][b, :length, kv], inp["v"][b, :length, kv], inp["lam"][h]))
            maps = []
            for m in range(2):
                s = scale * (qs[:, m] @ ks[:, m].T.contiguous())
                if hidden is not None:
                    s = s.masked_fill(hidden, -math.inf)
                maps.append(torch.softmax(s, dim=-1))
            oh = (maps[0] - lam * maps[1]) @ vs
            o[b, first:, h] = oh.detach()
            if case["train"]:
                gq, gk, gv, gl = torch.autograd.grad(oh, (qs, ks, vs, lam), inp["do"][b, first:, h].double())
                grads["q"][b, first:, h] = gq
                grads["k"][b, :length, kv] += gk
                grads["v"][b, :length, kv] += gv
                grads["lam"][h] += gl
    out = {"o": o}
    if case["train"]:
        out.update({"d" + i: grads[i] for i in ("q", "k", "v", "lam")})
    return out


def exact(case, seed):
    inp = _INPUTS[case["op"]](case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "attn": _exact_attn}[case["op"]](case, inp)
