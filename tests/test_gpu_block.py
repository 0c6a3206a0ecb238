"""The attention block over a split convolution's feature map, forward and
backward, against the same formula differentiated in 64 bits."""
import numpy as np
import pytest

from workloads import small_layer

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")
from paper_2003_12621_amd.block import AttentionBlock  # noqa: E402

pytestmark = pytest.mark.gpu


def _reference(block, x, dy):
    """On the CPU in float64, parameters as the block holds them."""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in block.params.items()}
    x = x.double().cpu().requires_grad_()
    n, c, h, w = x.shape
    t = x.flatten(2).transpose(1, 2)
    t = (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + 1e-5)
    t = t * p["norm_weight"] + p["norm_bias"]
    q, k, v = block._split(t @ p["project"].t())
    r = block.dim // 2
    angle = (block.positions.double().cpu()[:, [0] * (r // 2) + [1] * (r // 2)] * block.freqs.double().cpu())[:, None, None]
    cos, sin = torch.cos(angle), torch.sin(angle)
    turn = lambda z: torch.cat([z[..., :r] * cos - z[..., r:] * sin, z[..., r:] * cos + z[..., :r] * sin], -1)
    g = block.heads // block.heads_k
    q, k, v = turn(q), turn(k).repeat_interleave(g, 2), v.repeat_interleave(g, 2)
    m = torch.einsum("bihmd,bjhmd->bhmij", q, k).mul(block.dim ** -0.5).softmax(-1)
    o = torch.einsum("bhij,bjhe->bihe", m[:, :, 0] - p["lam"].view(-1, 1, 1) * m[:, :, 1], v)
    y = (o.flatten(2) @ p["merge"].t()).transpose(1, 2).reshape(x.shape) + x
    names = list(p)
    grads = torch.autograd.grad(y, [x] + [p[i] for i in names], dy.double().cpu())
    return y.detach(), grads[0], dict(zip(names, grads[1:]))


def _rel(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


def test_block_over_a_convolution():
    n, c, h, w = 2, 48, 14, 10
    x, wt = small_layer(n, 12, h, w, c, 3, seed=21)
    plan = fs.Plan(n, 12, h, w, c, 3)
    features = plan.conv2d(torch.from_numpy(x).cuda(), plan.transform_weights(torch.from_numpy(wt).cuda()))
    block = AttentionBlock(n, c, h, w, heads=4, heads_k=2, dim=32, seed=3)
    y, saved = block.forward(features, save=True)
    dy = torch.from_numpy(np.random.default_rng(5).standard_normal(y.shape).astype(np.float32)).cuda()
    dx, grads = block.backward(dy, features, saved)
    plain = block.forward(features)
    torch.cuda.synchronize()
    assert torch.equal(plain, y)
    want_y, want_dx, want = _reference(block, features, dy)
    # bf16 tokens, projections, terms and outputs: a chain of about ten roundings
    # of 2^-9 / sqrt(3) each on the way to the first matrix's gradient, 4e-3 in
    # all; the residual path carries y and dx past most of them
    assert _rel(y, want_y) <= 1e-2
    assert _rel(dx, want_dx) <= 1e-2
    for name, g in grads.items():
        assert _rel(g, want[name]) <= 2e-2, name
