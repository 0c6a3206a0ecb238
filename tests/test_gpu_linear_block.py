"""The linear attention block over a stream of frames: a run of its operators
together, forward, backward through the state, and pixel by pixel, against the
same formulas in 64 bits."""
import numpy as np
import pytest

from workloads import small_layer

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")
from paper_2003_12621_amd.block import LinearAttentionBlock  # noqa: E402

pytestmark = pytest.mark.gpu


def _reference(block, frames, dys, first=0):
    """On the CPU in float64, parameters as the block holds them: the outputs of
    the frames, one after the other, and the gradients of their sum with dys."""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in block.params.items()}
    xs = [x.double().cpu().requires_grad_() for x in frames]
    decay = block.log_decay.double().cpu().exp()
    n, c, h, w = xs[0].shape
    g = block.heads // block.heads_k
    state = torch.zeros(n, block.heads_k, block.dim, block.dim_v, dtype=torch.float64)
    pairs = block.dim // 2
    axis = [i for i, s in enumerate(block.sections) for _ in range(s)]
    ys = []
    for f, x in enumerate(xs):
        t = x.flatten(2).transpose(1, 2)
        t = (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + 1e-5)
        t = t * p["norm_weight"] + p["norm_bias"]
        q, k, v = block._split(t @ p["project"].t())
        positions = block.positions.double().cpu().clone()
        positions[:, 0] = first + f
        angle = (positions[:, axis] * block.freqs.double().cpu())[:, None]
        cos, sin = torch.cos(angle), torch.sin(angle)

        def turn(z, weight):
            z = z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-6) * weight
            return torch.cat([z[..., :pairs] * cos - z[..., pairs:] * sin, z[..., pairs:] * cos + z[..., :pairs] * sin], -1)

        q, k = turn(q, p["q_weight"]), turn(k, p["k_weight"])
        o = []
        for i in range(h * w):
            state = decay.view(-1, 1, 1) * state + k[:, i].unsqueeze(-1) * v[:, i].unsqueeze(-2)
            o.append((q[:, i].unsqueeze(-1) * state.repeat_interleave(g, 1)).sum(-2) * block.dim ** -0.5)
        o = torch.stack(o, 1)
        ys.append((o.flatten(2) @ p["merge"].t()).transpose(1, 2).reshape(x.shape) + x)
    names = list(p)
    loss = sum((y * dy.double().cpu()).sum() for y, dy in zip(ys, dys))
    grads = torch.autograd.grad(loss, xs + [p[i] for i in names])
    return [y.detach() for y in ys], state.detach(), grads[:len(xs)], dict(zip(names, grads[len(xs):]))


def _rel(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


def _frames(n, c, h, w, count):
    x, wt = small_layer(count * n, 12, h, w, c, 3, seed=23)
    plan = fs.Plan(count * n, 12, h, w, c, 3)
    y = plan.conv2d(torch.from_numpy(x).cuda(), plan.transform_weights(torch.from_numpy(wt).cuda()))
    return [t.contiguous() for t in y.split(n)]


@pytest.mark.parametrize("heads,heads_k,dim,dim_v", [(4, 2, 32, 64), (3, 3, 20, 24)])
def test_block_over_frames(heads, heads_k, dim, dim_v):
    """Two frames, the second from the first one's state, and back through it."""
    n, c, h, w = 2, 48, 14, 10
    frames = _frames(n, c, h, w, 2)
    block = LinearAttentionBlock(n, c, h, w, heads, heads_k, dim, dim_v, seed=3)
    rng = np.random.default_rng(5)
    for name in ("q_weight", "k_weight"):
        block.params[name] = torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda()
    dys = [torch.from_numpy(rng.standard_normal((n, c, h, w)).astype(np.float32)).cuda() for _ in range(2)]
    y0, s0, saved0 = block.forward(frames[0], save=True)
    y1, s1, saved1 = block.forward(frames[1], s0, frame=1, save=True)
    dx1, g1, ds = block.backward(dys[1], frames[1], saved1)
    dx0, g0, none = block.backward(dys[0], frames[0], saved0, dstate=ds)
    again, _ = block.forward(frames[1], s0, frame=1)
    torch.cuda.synchronize()
    assert none is None and torch.equal(again, y1)
    ys, last, dxs, want = _reference(block, frames, dys)
    # bf16 tokens, projections, normed heads, scores or states, outputs and their
    # gradients: a chain of about twelve roundings of 2^-8 / sqrt(3), 8e-3 in all,
    # on the way to the first matrix's gradient; the residual path carries y and dx
    # past most of them
    for got, ref in ((y0, ys[0]), (y1, ys[1]), (s1, last), (dx0, dxs[0]), (dx1, dxs[1])):
        assert _rel(got, ref) <= 1e-2
    for name in want:
        assert _rel(g0[name].double() + g1[name].double(), want[name]) <= 2e-2, name


def test_pixels_continue_a_frame():
    """A frame, then the next one pixel by pixel, also as a captured graph that is
    replayed, as the frames one after the other."""
    n, c, h, w = 3, 48, 6, 5
    frames = _frames(n, c, h, w, 2)
    block = LinearAttentionBlock(n, c, h, w, 4, 2, 24, 40, seed=4)
    zeros = torch.zeros_like(frames[0])
    ys, last, _, _ = _reference(block, frames, [zeros, zeros])
    at = torch.zeros(3, dtype=torch.int32, device="cuda")
    _, state = block.forward(frames[0])
    kept = state.clone()
    pixels = frames[1].flatten(2)

    def place(i):
        at.copy_(torch.tensor([1, i // w, i % w], dtype=torch.int32))

    y = torch.empty_like(pixels)
    for i in range(h * w):
        place(i)
        y[:, :, i] = block.step(pixels[:, :, i].contiguous(), state, at)
    torch.cuda.synchronize()
    assert _rel(y.view_as(frames[1]), ys[1]) <= 1e-2 and _rel(state, last) <= 1e-2

    x, state2 = pixels[:, :, 0].contiguous(), kept.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.step(x, state2, at)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.step(x, state2, at)
    state2.copy_(kept)
    for i in range(h * w):
        place(i)
        x.copy_(pixels[:, :, i])
        graph.replay()
        assert torch.equal(out, y[:, :, i]), i
    torch.cuda.synchronize()
    assert torch.equal(state2, state)


def test_refusals():
    with pytest.raises(ValueError):
        LinearAttentionBlock(1, 8, 4, 4, 2, 1, 7, 8)
    with pytest.raises(ValueError):
        LinearAttentionBlock(1, 8, 4, 4, 2, 1, 4, 8)
