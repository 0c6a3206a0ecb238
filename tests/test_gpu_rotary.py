"""Rotary positions on the GPU against the definition in 64 bits.

Tolerances (largest error over the largest element of a pair's size).  fp32:
the turned pair is two products and a sum (1.5 * 2^-24 each, below 1.8e-7) of
sines good to 2^-23: 5e-7.  bf16: one rounding to 8 significant bits, at most
2^-8 = 3.9e-3 of the element, besides the fp32 errors: 4e-3.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
TOL = {"fp32": 5e-7, "bf16": 4e-3}


def _np(t):
    return t.double().cpu().numpy()


def reference(x, positions, freqs, sections, interleaved=False, inverse=False):
    """x [n, s, h, d], positions [n or 1, s, axes], all float64."""
    r = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = (positions[..., axis] * freqs)[:, :, None, :]
    if inverse:
        angle = -angle
    c, s = np.cos(angle), np.sin(angle)
    y = x.copy()
    ia, ib = (np.arange(0, 2 * r, 2), np.arange(1, 2 * r, 2)) if interleaved else (np.arange(r), np.arange(r, 2 * r))
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def make(seed, n, s, h, d, sections, dtype, top=200, per_batch=False):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((n, s, h, d)).astype(np.float32)).to(DTYPE[dtype]).cuda()
    shape = (n, s, len(sections)) if per_batch else (s, len(sections))
    pos = torch.from_numpy(rng.integers(-top, top, shape).astype(np.int32)).cuda()
    freqs = torch.from_numpy(np.concatenate([100.0 ** (-np.arange(p) / max(p, 1)) for p in sections]).astype(np.float32)).cuda()
    return x, pos, freqs


def err(got, want):
    return float(np.abs(_np(got) - want).max() / np.abs(want).max())


def wanted(x, pos, freqs, sections, **kw):
    p = _np(pos)
    return reference(_np(x), p if p.ndim == 3 else p[None], _np(freqs), sections, **kw)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("d,sections", [(32, (8, 8)), (64, (8, 12, 12)), (64, (32,)), (128, (10, 6, 0, 16)), (6, (1, 2)),
                                        (5, (1, 1)), (2, (1,)), (80, (20, 12)), (1024, (512,))])
def test_widths_and_sections(d, sections, interleaved, inverse, dtype):
    x, pos, freqs = make(d, 2, 19, 3, d, sections, dtype)
    print(f"[case] rotary d {d} sections {sections} {dtype}", flush=True)
    y = fs.rotary(x, pos, freqs, sections, interleaved=interleaved, inverse=inverse)
    torch.cuda.synchronize()
    assert err(y, wanted(x, pos, freqs, sections, interleaved=interleaved, inverse=inverse)) <= TOL[dtype]


@pytest.mark.parametrize("n,s,h", [(1, 1, 1), (3, 700, 2), (1, 5000, 5), (2, 16, 40)])
def test_sizes(n, s, h):
    x, pos, freqs = make(1, n, s, h, 64, (16, 16), "bf16", per_batch=True)
    y = fs.rotary(x, pos, freqs, (16, 16))
    torch.cuda.synchronize()
    assert err(y, wanted(x, pos, freqs, (16, 16))) <= TOL["bf16"]


def test_large_positions():
    """Angles of a million turns keep their precision."""
    x, pos, freqs = make(2, 1, 300, 2, 32, (16,), "fp32", top=2 ** 31 - 1)
    freqs = freqs * 0.731
    y = fs.rotary(x, pos, freqs, (16,))
    torch.cuda.synchronize()
    assert err(y, wanted(x, pos, freqs, (16,))) <= TOL["fp32"]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_two_tensors_strides_and_in_place(dtype):
    n, s, hq, hk, d, sec = 2, 33, 4, 2, 32, (8, 8)
    x, pos, freqs = make(3, n, s, 1, (hq + 2 * hk) * 2 * d + 8, sec, dtype)
    packed = x[:, :, 0, :-8]
    q = packed[..., :hq * 2 * d].unflatten(-1, (hq, 2, d))
    k = packed[..., hq * 2 * d:(hq + hk) * 2 * d].unflatten(-1, (hk, 2, d))
    want = [wanted(t.flatten(2, 3), pos, freqs, sec).reshape(t.shape) for t in (q, k)]
    a, b = fs.rotary(q, pos, freqs, sec, other=k)
    torch.cuda.synchronize()
    assert a.shape == q.shape and err(a, want[0]) <= TOL[dtype] and err(b, want[1]) <= TOL[dtype]
    before = x.clone()
    a2, b2 = fs.rotary(q, pos, freqs, sec, other=k, out=q, out_other=k)
    torch.cuda.synchronize()
    assert a2 is q and torch.equal(q, a) and torch.equal(k, b)
    rest = slice((hq + hk) * 2 * d, None)
    assert torch.equal(x[..., rest], before[..., rest])
    # an odd offset: element accesses
    odd = torch.zeros(n, s, 3, d + 1, dtype=x.dtype, device="cuda")
    odd[..., 1:] = torch.randn(n, s, 3, d, device="cuda")
    y = fs.rotary(odd[..., 1:], pos, freqs, sec)
    torch.cuda.synchronize()
    assert err(y, wanted(odd[..., 1:], pos, freqs, sec)) <= TOL[dtype]


def test_inverse_is_the_gradient():
    """<dy, R x> = <R^T dy, x>."""
    x, pos, freqs = make(5, 2, 50, 3, 64, (10, 10), "fp32")
    dy = torch.randn_like(x)
    y = fs.rotary(x, pos, freqs, (10, 10))
    dx = fs.rotary(dy, pos, freqs, (10, 10), inverse=True)
    torch.cuda.synchronize()
    a, b = (_np(dy) * _np(y)).sum(), (_np(dx) * _np(x)).sum()
    # 19 200 products, each side rounded to 5e-7
    assert abs(a - b) <= 5e-7 * np.linalg.norm(_np(dy)) * np.linalg.norm(_np(x))
