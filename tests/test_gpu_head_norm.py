"""Norms of heads with their rotation, and the gradients of both, on the GPU
against the definition in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32.  y: the sum of a head's squares is
a chain of at most 22 roundings in a lane and 6 between lanes, half of whose
relative error goes into rstd; division and root add 2 u, the two products 2 u,
the sines and the turn 5 u: 23 u = 1.4e-6 of the largest element.  dx: g = w u
carries 6 u, the mean of g z the 28 roundings of its sum and 10 u of its factors,
times a z of at most 5 here: 6 + 5 * 38 u of the gradient's size, below 1.2e-5 of
the largest element.  bf16 adds the rounding of the result, 2^-8 of an element.
dweight: terms good to 40 u, summed in chains that are no longer than the rows
and the parts: (rows + 1200 + 40) u of the sum of the terms' magnitudes.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
TOL = {"fp32": 1.4e-6, "bf16": 2.0 ** -8 + 1.4e-6}
TOL_DX = {"fp32": 1.2e-5, "bf16": 2.0 ** -8 + 1.2e-5}
EPS = 1e-6


def _np(t):
    return t.detach().double().cpu().numpy()


def _turn(x, positions, freqs, sections, interleaved, back=False):
    r = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = (positions[..., axis] * freqs)[:, :, None, :] * (-1 if back else 1)
    c, s = np.cos(angle), np.sin(angle)
    y = x.copy()
    ia, ib = (np.arange(0, 2 * r, 2), np.arange(1, 2 * r, 2)) if interleaved else (np.arange(r), np.arange(r, 2 * r))
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def reference(x, w, positions, freqs, sections, interleaved=False, eps=EPS, dy=None):
    """x [n, s, h, d], positions [n or 1, s, axes], float64: y, or (y, dx, dw,
    the sum of the magnitudes of dw's terms) where dy is given."""
    rstd = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    z = x * rstd
    w = np.ones(x.shape[-1]) if w is None else w
    y = _turn(z * w, positions, freqs, sections, interleaved)
    if dy is None:
        return y
    u = _turn(dy, positions, freqs, sections, interleaved, back=True)
    g = w * u
    dx = rstd * (g - z * (g * z).mean(-1, keepdims=True))
    return y, dx, (u * z).sum((0, 1, 2)), np.abs(u * z).sum((0, 1, 2))


def make(seed, n, s, h, d, sections, dtype, per_batch=False):
    rng = np.random.default_rng(seed)
    f = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32))
    x, dy = (f(n, s, h, d) * 0.7).to(DTYPE[dtype]).cuda(), f(n, s, h, d).to(DTYPE[dtype]).cuda()
    pos = torch.from_numpy(rng.integers(-200, 200, (n, s, len(sections)) if per_batch else (s, len(sections))).astype(np.int32))
    freqs = np.concatenate([100.0 ** (-np.arange(p) / max(p, 1)) for p in sections]).astype(np.float32)
    return x, dy, (1 + 0.2 * f(d)).cuda(), pos.cuda(), torch.from_numpy(freqs).cuda()


def wanted(x, w, pos, freqs, sections, dy=None, **kw):
    p = _np(pos)
    flat = lambda t: _np(t).reshape(*t.shape[:2], -1, t.shape[-1])
    return reference(flat(x), None if w is None else _np(w), p if p.ndim == 3 else p[None], _np(freqs), sections,
                     dy=None if dy is None else flat(dy), **kw)


def err(got, want):
    return float(np.abs(_np(got).reshape(want.shape) - want).max() / np.abs(want).max())


def check(x, dy, w, pos, freqs, sections, dtype, **kw):
    y = fs.head_norm_rotary(x, w, pos, freqs, sections, eps=EPS, **kw)
    dx, dw = fs.head_norm_rotary_backward(dy, x, w, pos, freqs, sections, eps=EPS, **kw)
    torch.cuda.synchronize()
    want_y, want_dx, want_dw, size = wanted(x, w, pos, freqs, sections, dy=dy, **kw)
    assert y.dtype == x.dtype and dx.dtype == x.dtype and dw.dtype == torch.float32
    assert err(y, want_y) <= TOL[dtype]
    assert err(dx, want_dx) <= TOL_DX[dtype]
    rows = x[..., 0].numel()
    assert (np.abs(_np(dw) - want_dw) <= (rows + 1240) * U * size).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,sections", [(32, (8, 8)), (64, (8, 12, 12)), (64, (32,)), (128, (10, 6, 0, 16)), (6, (1, 2)),
                                        (5, (1, 1)), (2, (1,)), (40, (8, 8)), (40, (20,)), (40, (5, 5, 5)), (96, (24, 24)),
                                        (72, (4,)), (250, (100, 25)), (1024, (512,)), (1024, (100,)), (1022, (255, 256))])
def test_widths_and_sections(d, sections, interleaved, dtype):
    x, dy, w, pos, freqs = make(d, 2, 19, 3, d, sections, dtype)
    print(f"[case] head norm d {d} sections {sections} {dtype} interleaved {interleaved}", flush=True)
    check(x, dy, w, pos, freqs, sections, dtype, interleaved=interleaved)


@pytest.mark.parametrize("n,s,h", [(1, 1, 1), (3, 700, 2), (1, 5000, 5), (2, 16, 40), (16, 1, 20), (1, 9001, 1)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sizes(n, s, h, dtype):
    x, dy, w, pos, freqs = make(1, n, s, h, 64, (16, 16), dtype, per_batch=True)
    check(x, dy, w, pos, freqs, (16, 16), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_tensors_strides_and_in_place(dtype):
    """Queries and keys as slices of one projection, heads in two dimensions."""
    n, s, hq, hk, d, sec = 2, 33, 4, 2, 32, (8, 8)
    x, dy, wq, pos, freqs = make(3, n, s, 1, (hq + 2 * hk) * 2 * d + 8, sec, dtype)
    wq, wk = wq[:d].contiguous(), wq[d:2 * d].contiguous()
    part = lambda t: (t[:, :, 0, :hq * 2 * d].unflatten(-1, (hq, 2, d)),
                      t[:, :, 0, hq * 2 * d:(hq + hk) * 2 * d].unflatten(-1, (hk, 2, d)))
    (q, k), (gq, gk) = part(x), part(dy)
    want = [wanted(t, w, pos, freqs, sec, dy=g) for t, w, g in ((q, wq, gq), (k, wk, gk))]
    a, b = fs.head_norm_rotary(q, wq, pos, freqs, sec, other=k, other_weight=wk)
    back = fs.head_norm_rotary_backward(gq, q, wq, pos, freqs, sec, dy_other=gk, other=k, other_weight=wk)
    torch.cuda.synchronize()
    assert a.shape == q.shape and back[2].shape == k.shape
    for got, grad, dw, w in ((a, back[0], back[1], want[0]), (b, back[2], back[3], want[1])):
        assert err(got, w[0]) <= TOL[dtype] and err(grad, w[1]) <= TOL_DX[dtype]
        assert (np.abs(_np(dw) - w[2]) <= (n * s * 8 + 1240) * U * w[3]).all()
    # in place, and nothing else of the tensors changes
    before = x.clone(), dy.clone()
    a2, b2 = fs.head_norm_rotary(q, wq, pos, freqs, sec, other=k, other_weight=wk, out=q, out_other=k)
    rest = slice((hq + hk) * 2 * d, None)
    assert a2 is q and torch.equal(q, a) and torch.equal(k, b)
    x.copy_(before[0])
    again = fs.head_norm_rotary_backward(gq, q, wq, pos, freqs, sec, dy_other=gk, other=k, other_weight=wk, out=gq,
                                         out_other=gk)
    torch.cuda.synchronize()
    assert again[0] is gq and torch.equal(gq, back[0]) and torch.equal(gk, back[2])
    assert torch.equal(again[1], back[1]) and torch.equal(again[3], back[3])
    assert torch.equal(x, before[0]) and torch.equal(dy[..., rest], before[1][..., rest])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,s,h,h1,d", [(1, 9001, 9, 5, 64), (2, 3, 100, 37, 128), (3, 5, 1, 70, 32)])
def test_in_place_rounds_of_heads(n, s, h, h1, d, dtype):
    """More heads than a workgroup takes at once, of two slices of one tensor:
    rows are read while the ones before them are written, forwards and back."""
    sections = (d // 4, d // 4)
    x, dy, w, pos, freqs = make(15, n, s, h + h1, d, sections, dtype)
    w1 = w.flip(0).contiguous()
    both, grads = x.clone(), dy.clone()
    fs.head_norm_rotary(both[:, :, :h], w, pos, freqs, sections, other=both[:, :, h:], other_weight=w1, eps=EPS,
                        out=both[:, :, :h], out_other=both[:, :, h:])
    _, dw, _, dw1 = fs.head_norm_rotary_backward(
        grads[:, :, :h], x[:, :, :h], w, pos, freqs, sections, dy_other=grads[:, :, h:], other=x[:, :, h:], other_weight=w1,
        eps=EPS, out=grads[:, :, :h], out_other=grads[:, :, h:])
    torch.cuda.synchronize()
    for part, weight, got in ((slice(0, h), w, dw), (slice(h, None), w1, dw1)):
        y, dx, want, size = wanted(x[:, :, part], weight, pos, freqs, sections, dy=dy[:, :, part])
        assert err(both[:, :, part], y) <= TOL[dtype] and err(grads[:, :, part], dx) <= TOL_DX[dtype]
        rows = n * s * x[:, :, part].shape[2]
        assert (np.abs(_np(got) - want) <= (rows + 1240) * U * size).all()


@pytest.mark.parametrize("d", [64, 1024])
def test_in_place_wide(d):
    """Heads that 64 lanes take in several pieces, too, may be written in place."""
    x, dy, w, pos, freqs = make(11, 2, 9, 3, d, (d // 4,), "fp32")
    args = (w, pos, freqs, (d // 4,))
    want = fs.head_norm_rotary(x, *args), *fs.head_norm_rotary_backward(dy, x, *args)
    keep = x.clone()
    assert torch.equal(fs.head_norm_rotary(x, *args, out=x), want[0])
    dx, dw = fs.head_norm_rotary_backward(dy, keep, *args, out=dy)
    assert torch.equal(dx, want[1]) and torch.equal(dw, want[2])


@pytest.mark.parametrize("offset,pad", [(1, 0), (2, 1), (4, 4)])
def test_alignment(offset, pad):
    """Bases and strides that allow accesses of 1, 2 and 4 elements only."""
    n, s, h, d, sec = 2, 21, 3, 32, (16,)
    x, dy, w, pos, freqs = make(5, n, s, h, d, sec, "bf16")
    shift = lambda t: torch.cat([torch.zeros(offset, dtype=t.dtype, device="cuda"),
                                 torch.nn.functional.pad(t, (0, pad)).flatten()])[offset:].view(n, s, h, d + pad)[..., :d]
    check(shift(x), shift(dy), w, pos, freqs, sec, "bf16")


def test_expanded_gradient_and_no_weight():
    """The gradient of a sum over tokens is one row for all; a weight of None is 1."""
    x, dy, _, pos, freqs = make(6, 2, 40, 3, 64, (16, 16), "bf16")
    check(x, dy[:, :1].expand(-1, 40, -1, -1), None, pos, freqs, (16, 16), "bf16")


def test_rows_of_zeros():
    """A padded batch's rows: zero, with the finite gradient of the formula."""
    x, dy, w, pos, freqs = make(7, 2, 20, 2, 32, (16,), "fp32")
    x[1, 12:] = 0
    y = fs.head_norm_rotary(x, w, pos, freqs, (16,), eps=EPS)
    dx, _ = fs.head_norm_rotary_backward(dy, x, w, pos, freqs, (16,), eps=EPS)
    torch.cuda.synchronize()
    want = wanted(x, w, pos, freqs, (16,), dy=dy)
    assert (y[1, 12:] == 0).all()
    there = _np(dx)[1, 12:]
    assert np.abs(there - want[1][1, 12:]).max() <= TOL_DX["fp32"] * np.abs(want[1][1, 12:]).max()


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    """<dx, e> and <dw, f> against central differences of <dy, y> in 64 bits."""
    x, dy, w, pos, freqs = make(8, 1, 6, 2, 20, (4, 3), "fp32")
    dx, dw = fs.head_norm_rotary_backward(dy, x, w, pos, freqs, (4, 3), eps=EPS, interleaved=interleaved)
    torch.cuda.synchronize()
    rng = np.random.default_rng(9)
    e, f = rng.standard_normal(tuple(x.shape)), rng.standard_normal(20)
    value = lambda a, b: (_np(dy) * reference(a, b, _np(pos)[None], _np(freqs), (4, 3), interleaved)).sum()
    h = 1e-5
    for got, step in (((_np(dx) * e).sum(), (h * e, 0)), ((_np(dw) * f).sum(), (0, h * f))):
        slope = (value(_np(x) + step[0], _np(w) + step[1]) - value(_np(x) - step[0], _np(w) - step[1])) / (2 * h)
        # 240 terms of size about 1 good to 1.2e-5 each, differences to h^2
        assert abs(got - slope) <= 240 * 1.2e-5 * 3


def test_two_streams_and_repeated_calls():
    """Calls on two streams with workspaces of their own give what one gives."""
    x, dy, w, pos, freqs = make(10, 2, 3000, 4, 64, (32,), "bf16")
    want = fs.head_norm_rotary_backward(dy, x, w, pos, freqs, (32,))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            got.append(fs.head_norm_rotary_backward(dy, x, w, pos, freqs, (32,)))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_graph():
    q, k = torch.empty(2, 60, 4, 32, device="cuda"), torch.empty(2, 60, 2, 32, device="cuda")
    gq, gk = torch.empty_like(q), torch.empty_like(k)
    pos = torch.randint(0, 50, (60, 2), device="cuda", dtype=torch.int32)
    freqs, wq, wk = torch.rand(16, device="cuda"), torch.rand(32, device="cuda"), torch.rand(32, device="cuda")

    def make_calls():
        kw = dict(other=k, other_weight=wk)
        return [*fs.head_norm_rotary(q, wq, pos, freqs, (8, 8), **kw),
                *fs.head_norm_rotary_backward(gq, q, wq, pos, freqs, (8, 8), dy_other=gk, **kw)]

    def fill(i):
        gen = torch.Generator(device="cuda").manual_seed(i)
        for t in (q, k, gq, gk):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        make_calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = make_calls()
    for i in range(1, 5):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = make_calls()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want)), i
