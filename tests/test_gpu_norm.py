"""Layer norm on the GPU, forward and backward, against its definition in 64 bits.

Tolerances (relative L2 norm).  fp32: sums of up to 8192 terms in fp32 with
independent roundings, below sqrt(8192) 2^-24 = 6e-6 of a term's size in the
worst ordering and far less in pieces: 1e-5.  The gradients of the parameters
sum over rows as well: the same bound.  dx is a difference of terms (with two
channels, all but eps / var of it cancels): its error is relative to its first
term, rstd dy w.  bf16 outputs: one rounding of 8 bits,
2^-9 / sqrt(3) = 1.2e-3 on average, at most 2^-8: 3e-3.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
TOL = {"fp32": 1e-5, "bf16": 3e-3}
EPS = 1e-5


def _np(t):
    return t.double().cpu().numpy()


def _rel(got, want):
    return float(np.linalg.norm(_np(got).reshape(want.shape) - want) / max(np.linalg.norm(want), 1e-30))


def _tokens(a, first):
    """[n, c, s] or [n, s, c] -> [n, s, c]."""
    return a.transpose(0, 2, 1) if first else a


def reference(x, w, b, dy):
    """x, dy [n, s, c] in float64."""
    mean = x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + EPS)
    xhat = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(-1, keepdims=True) - xhat * (g * xhat).mean(-1, keepdims=True))
    return xhat * w + b, (dx, np.linalg.norm(rstd * g)), (dy * xhat).sum((0, 1)), dy.sum((0, 1)), mean.ravel(), rstd.ravel()


def check(n, s, c, layout, dtype, out_layout=None, out_dtype=None, offset=0.5, params=True):
    print(f"[case] norm {n}x{s}x{c} {layout}->{out_layout} {dtype}->{out_dtype}", flush=True)
    out_layout, out_dtype = out_layout or layout, out_dtype or dtype
    rng = np.random.default_rng(n * 7 + s * 3 + c)
    first, out_first = layout == "first", out_layout == "first"
    x = torch.from_numpy(rng.standard_normal((n, c, s) if first else (n, s, c)).astype(np.float32) + np.float32(offset))
    dy = torch.from_numpy(rng.standard_normal((n, c, s) if out_first else (n, s, c)).astype(np.float32))
    w = torch.from_numpy(rng.uniform(0.5, 1.5, c).astype(np.float32)) if params else None
    b = torch.from_numpy(rng.standard_normal(c).astype(np.float32)) if params else None
    x, dy = x.to(DTYPE[dtype]).cuda(), dy.to(DTYPE[out_dtype]).cuda()
    wd, bd = (w.cuda(), b.cuda()) if params else (None, None)
    y, mean, rstd = fs.layer_norm(x, wd, bd, eps=EPS, layout=layout, out_layout=out_layout,
                                  out_dtype=DTYPE[out_dtype], return_stats=True)
    dx, dw, db = fs.layer_norm_backward(dy, x, mean, rstd, wd, layout=layout, out_layout=out_layout)
    plain = fs.layer_norm(x, wd, bd, eps=EPS, layout=layout, out_layout=out_layout, out_dtype=DTYPE[out_dtype])
    torch.cuda.synchronize()
    assert torch.equal(plain, y)
    assert y.shape == dy.shape and dx.shape == x.shape and y.dtype == DTYPE[out_dtype] and dx.dtype == x.dtype
    want = reference(_tokens(_np(x), first), _np(w) if params else 1.0, _np(b) if params else 0.0,
                     _tokens(_np(dy), out_first))
    if out_first:
        assert _rel(y, want[0].transpose(0, 2, 1)) <= TOL[out_dtype]
    else:
        assert _rel(y, want[0]) <= TOL[out_dtype]
    dx_want, dx_terms = want[1]
    assert np.linalg.norm(_tokens(_np(dx), first) - dx_want) <= TOL[dtype] * dx_terms
    assert _rel(dw, want[2]) <= 1e-5
    assert _rel(db, want[3]) <= 1e-5
    assert _rel(mean, want[4]) <= 1e-5 and _rel(rstd, want[5]) <= 1e-5


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("c", [1, 2, 7, 8, 64, 77, 128, 136, 257, 512, 768, 1024, 1032, 1500, 4096, 4104, 8191, 8192])
def test_channels_last(c, dtype):
    # one channel has no variance: only the finite output is checked there
    if c == 1:
        y = fs.layer_norm(torch.randn(5, 1, device="cuda").to(DTYPE[dtype]))
        assert not y.any()
        return
    check(2, 37, c, "last", dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("c", [2, 16, 33, 64, 77, 256, 257, 512, 600, 1024, 1025, 2047, 2048])
@pytest.mark.parametrize("s", [49, 64, 132])
def test_channels_first(c, s, dtype):
    check(2, s, c, "first", dtype)


@pytest.mark.parametrize("dtype,out_dtype", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("c,s", [(3, 5), (64, 64), (77, 49), (256, 100), (300, 196), (512, 196), (1000, 52), (2048, 49)])
def test_map_to_tokens(c, s, dtype, out_dtype):
    check(3, s, c, "first", dtype, out_layout="last", out_dtype=out_dtype)


@pytest.mark.parametrize("layout", ["first", "last"])
def test_fp32_to_bf16(layout):
    check(2, 60, 96, layout, "fp32", out_dtype="bf16")


@pytest.mark.parametrize("n,s", [(1, 1), (1, 4), (1, 8000), (3000, 1), (40, 300)])
@pytest.mark.parametrize("layout", ["first", "last"])
def test_row_counts(n, s, layout):
    check(n, s, 48, layout, "fp32")


@pytest.mark.parametrize("layout", ["first", "last"])
def test_without_parameters(layout):
    check(2, 30, 40, layout, "fp32", params=False)


@pytest.mark.parametrize("layout", ["first", "last"])
def test_large_mean(layout):
    """A mean of 1000 standard deviations: the deviations are taken from the
    mean, not as a difference of squares.  fp32 inputs of size 1000 carry
    2^-24 * 1000 = 6e-5 of the deviations' size in the mean's rounding."""
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((2, 200, 56)) + 1000).astype(np.float32)
    y = fs.layer_norm(torch.from_numpy(x).cuda(), layout=layout)
    torch.cuda.synchronize()
    x64 = x.astype(np.float64)
    axis = 1 if layout == "first" else 2
    want = (x64 - x64.mean(axis, keepdims=True)) / np.sqrt(x64.var(axis, keepdims=True) + EPS)
    assert _rel(y, want) <= 3e-4


def test_gradient_by_differences():
    rng = np.random.default_rng(4)
    x, dy = rng.standard_normal((1, 6, 10)), rng.standard_normal((1, 6, 10))
    w, b = rng.uniform(0.5, 1.5, 10), rng.standard_normal(10)
    dev = [torch.from_numpy(a.astype(np.float32)).cuda() for a in (x, w, b, dy)]
    x, w, b, dy = (_np(a) for a in dev)
    _, mean, rstd = fs.layer_norm(*dev[:3], eps=EPS, return_stats=True)
    grads = fs.layer_norm_backward(dev[3], dev[0], mean, rstd, dev[1])
    torch.cuda.synchronize()
    for i, g in enumerate(grads):
        step = rng.standard_normal((x, w, b)[i].shape)
        f = []
        for sign in (1, -1):
            a = [x, w, b]
            a[i] = a[i] + sign * 1e-5 * step
            f.append((reference(*a, dy)[0] * dy).sum())
        want = (f[0] - f[1]) / 2e-5
        # fp32 gradients: 1e-6 of the norms' product; the difference adds 1e-9
        assert abs((_np(g) * step).sum() - want) <= 1e-5 * np.linalg.norm(_np(g)) * np.linalg.norm(step)


def test_not_finite_stays_in_its_row():
    x = torch.randn(6, 64, device="cuda")
    good = fs.layer_norm(x)
    x[2, 5], x[4, 7] = float("nan"), float("inf")
    y = fs.layer_norm(x)
    assert torch.isnan(y[2]).all() and torch.isnan(y[4]).any()
    for r in (0, 1, 3, 5):
        assert torch.equal(y[r], good[r])
    m = torch.randn(1, 64, 49, device="cuda")
    good = fs.layer_norm(m, layout="first")
    m[0, 3, 10] = float("nan")
    y = fs.layer_norm(m, layout="first")
    assert torch.isnan(y[0, :, 10]).all()
    keep = [i for i in range(49) if i != 10]
    assert torch.equal(y[..., keep], good[..., keep])


def test_repeatable_and_on_another_stream():
    x = torch.randn(300, 96, 49, device="cuda")
    dy = torch.randn_like(x)
    w = torch.rand(96, device="cuda")
    _, mean, rstd = fs.layer_norm(x, w, layout="first", return_stats=True)
    a = fs.layer_norm_backward(dy, x, mean, rstd, w, layout="first")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b = fs.layer_norm_backward(dy, x, mean, rstd, w, layout="first")
    stream.synchronize()
    for u, v in zip(a, b):
        assert torch.equal(u, v)
