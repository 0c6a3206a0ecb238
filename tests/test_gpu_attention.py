"""Differential attention on the GPU against its definition in 64 bits.

Tolerances (relative L2 norm).  fp32: products of fp32 numbers summed in fp32
over at most a few hundred terms, an error below 2^-24 sqrt(terms) of a term's
size each; softmax terms by an exp2 good to 2^-22: 1e-5 leaves a factor of
ten.  bf16: inputs are given in bf16 to both sides; the terms of the softmax,
the score gradients, and the outputs are rounded to 8 bits, an error of
2^-9 / sqrt(3) relative to each, independent of one another, and o and o2
enter the gradients rounded once more: sqrt(4) * 2^-9 / sqrt(3) = 2.3e-3, and
5e-3 allows for a cancelling difference of the maps.
"""
import numpy as np
import pytest

from attention_reference import make_inputs, reference

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

TOL = {"fp32": 1e-5, "bf16": 5e-3}
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def _np(t):
    return t.double().cpu().numpy()


def _err(got, want):
    norm = np.linalg.norm(want)
    return float(np.linalg.norm(_np(got) - want) / norm) if norm else float(np.abs(_np(got)).max(initial=0.0))


def check(n, sq, sk, hq, hk, d, dv, dtype, causal=False, lengths=None, lam_count=None, lam_dtype=None, scale=None,
          train=True, seed=0, place=None):
    """`place`: a function that puts a dense tensor into another layout."""
    print(f"[case] {n}x{sq}x{sk} heads {hq}/{hk} d {d} dv {dv} {dtype} causal={causal} lengths={lengths}", flush=True)
    dt = DTYPE[dtype]
    arrays = make_inputs(seed, n, sq, sk, hq, hk, d, dv, lam_count)
    q, k, v, lam, do = (_dev(a, dt) for a in arrays)
    lam = lam.to(lam_dtype or dt)
    want = reference(*(_np(t) for t in (q, k, v, lam)), lengths=lengths, causal=causal, scale=scale,
                     do=_np(do) if train else None)
    if place:
        q, k, v, do = (place(t) for t in (q, k, v, do))
    kl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    plan = fs.DiffAttention(n, sq, sk, hq, hk, d, dv, dtype=dt, causal=causal, scale=scale)
    if not train:
        o = plan.forward(q, k, v, lam, key_lengths=kl)
        torch.cuda.synchronize()
        assert _err(o, want) <= TOL[dtype]
        return o
    o, saved = plan.forward(q, k, v, lam, key_lengths=kl, save=True)
    grads = plan.backward(do, q, k, v, lam, saved, key_lengths=kl)
    torch.cuda.synchronize()
    errors = {name: _err(t, w) for name, t, w in zip(("o", "dq", "dk", "dv", "dlam"), (o, *grads), want)}
    print(errors)
    for name, e in errors.items():
        # dlam: a sum with cancellation over rows, of which each term carries the
        # error of the rounded o2; its own rounding is as any other output's
        assert e <= TOL[dtype] * (4 if name == "dlam" else 1), (name, errors)
    return (o, *grads)


WIDTHS = [(32, 64), (64, 128), (128, 256)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("causal", [False, True])
def test_widths(d, dv, causal, dtype):
    check(2, 70, 70, 2, 2, d, dv, dtype, causal=causal)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", [(1, 1), (3, 5), (20, 40), (40, 24), (72, 130), (8, 256), (128, 8)])
def test_odd_widths(d, dv, dtype):
    check(1, 37, 45, 2, 1, d, dv, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sq,sk", [(1, 1), (1, 200), (31, 33), (33, 31), (129, 64), (5, 300), (260, 7), (128, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(sq, sk, causal, dtype):
    check(2, sq, sk, 2, 1, 32, 64, dtype, causal=causal)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_key_lengths(causal, dtype):
    """Sequences of no key, one, some and all; lengths out of range are clamped."""
    check(6, 50, 90, 2, 2, 32, 64, dtype, causal=causal, lengths=[0, 1, 33, 90, 120, -3])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("hq,hk", [(8, 1), (6, 3), (5, 5)])
def test_shared_key_heads(hq, hk, dtype):
    check(2, 40, 61, hq, hk, 64, 128, dtype, causal=True)


@pytest.mark.parametrize("lam_count,lam_dtype", [(1, torch.float32), (4, torch.float32), (1, torch.bfloat16)])
def test_one_lam_for_all_heads(lam_count, lam_dtype):
    check(2, 40, 40, 4, 2, 32, 64, "bf16", lam_count=lam_count, lam_dtype=lam_dtype)


def test_scale():
    check(1, 40, 50, 2, 2, 64, 128, "fp32", scale=0.3)


def _padded(t):
    """Rows in a wider buffer: strides of other multiples, 16-byte aligned."""
    big = torch.full(t.shape[:-1] + (t.shape[-1] + 16,), float("nan"), dtype=t.dtype, device=t.device)
    big[..., 8:8 + t.shape[-1]] = t
    return big[..., 8:8 + t.shape[-1]]


def _unaligned(t):
    big = torch.full(t.shape[:-1] + (t.shape[-1] + 3,), float("nan"), dtype=t.dtype, device=t.device)
    big[..., 1:1 + t.shape[-1]] = t
    return big[..., 1:1 + t.shape[-1]]


def _heads_first(t):
    return t.transpose(1, 2).contiguous().transpose(1, 2)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("place", [_padded, _unaligned, _heads_first])
def test_strides(place, dtype):
    a = check(2, 45, 45, 4, 2, 32, 64, dtype, causal=True, place=place)
    b = check(2, 45, 45, 4, 2, 32, 64, dtype, causal=True)
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_nothing_is_read_past_the_key_lengths(dtype):
    """NaN and infinities behind each sequence's keys change nothing."""
    n, s, h, d, dv = 3, 64, 2, 32, 64
    q, k, v, lam, do = (_dev(a, DTYPE[dtype]) for a in make_inputs(3, n, s, s, h, h, d, dv))
    lengths = [40, 0, 64]
    kl = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    plan = fs.DiffAttention(n, s, s, h, h, d, dv, dtype=DTYPE[dtype])
    outs = []
    for fill in (0.0, float("nan"), float("inf")):
        for b, l in enumerate(lengths):
            k[b, l:], v[b, l:] = fill, fill
        o, saved = plan.forward(q, k, v, lam, key_lengths=kl, save=True)
        outs.append((o, *plan.backward(do, q, k, v, lam, saved, key_lengths=kl)))
    torch.cuda.synchronize()
    for other in outs[1:]:
        for x, y in zip(outs[0], other):
            assert torch.equal(x, y)
    dk, dv_ = outs[0][2], outs[0][3]
    for b, l in enumerate(lengths):
        assert not dk[b, l:].any() and not dv_[b, l:].any()
    assert not outs[0][0][1].any() and not outs[0][1][1].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_large_scores(dtype):
    """Scores of some hundreds: each row's weight sits on one key, and the
    running maximum moves far."""
    n, s, h, d, dv = 1, 200, 2, 64, 128
    q, k, v, lam, do = make_inputs(5, n, s, s, h, h, d, dv)
    q, k = q * 12, k * 12
    dt = DTYPE[dtype]
    q, k, v, lam, do = (_dev(a, dt) for a in (q, k, v, lam, do))
    want = reference(*(_np(t) for t in (q, k, v, lam)))
    got = fs.DiffAttention(n, s, s, h, h, d, dv, dtype=dt).forward(q, k, v, lam)
    torch.cuda.synchronize()
    # a score of size 1e3 carries 2^-24 * 1e3 of rounding (fp32 sums of 64 products)
    assert _err(got, want) <= {"fp32": 1e-3, "bf16": 5e-3}[dtype]


def test_gradient_by_differences():
    """Directional differences of the 64-bit reference's loss agree with the
    operator's fp32 gradients."""
    n, sq, sk, hq, hk, d, dv = 1, 9, 13, 2, 1, 8, 12
    arrays = make_inputs(7, n, sq, sk, hq, hk, d, dv)
    do = arrays[4].astype(np.float64)
    dev = [_dev(a, torch.float32) for a in arrays]
    plan = fs.DiffAttention(n, sq, sk, hq, hk, d, dv, causal=True)
    o, saved = plan.forward(*dev[:4], save=True)
    grads = plan.backward(dev[4], *dev[:4], saved)
    torch.cuda.synchronize()
    rng = np.random.default_rng(8)
    for i in range(4):
        step = rng.standard_normal(arrays[i].shape)
        eps = 1e-5
        moved = []
        for sign in (1, -1):
            x = [a.astype(np.float64) for a in arrays[:4]]
            x[i] = x[i] + sign * eps * step
            moved.append((reference(*x, causal=True) * do).sum())
        want = (moved[0] - moved[1]) / (2 * eps)
        got = float((_np(grads[i]) * step).sum())
        # the difference's own error is eps^2 of third derivatives of order one;
        # fp32 gradients sum to 1e-6 of the norms
        assert abs(got - want) <= 1e-4 * (1 + np.linalg.norm(_np(grads[i])) * np.linalg.norm(step) * 1e-2)


def test_repeatable():
    """The same bits on every run: nothing depends on the order of workgroups."""
    q, k, v, lam, do = (_dev(a, torch.bfloat16) for a in make_inputs(9, 2, 300, 300, 4, 2, 64, 128))
    plan = fs.DiffAttention(2, 300, 300, 4, 2, 64, 128, dtype=torch.bfloat16, causal=True)
    runs = []
    for _ in range(3):
        o, saved = plan.forward(q, k, v, lam, save=True)
        runs.append((o, *plan.backward(do, q, k, v, lam, saved)))
    torch.cuda.synchronize()
    for r in runs[1:]:
        for x, y in zip(runs[0], r):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("sq,causal", [(1, True), (7, True), (40, False)])
def test_few_rows_over_many_keys(d, dv, sq, causal, dtype):
    """The kernel whose workgroups share the keys, with lengths that leave
    workgroups and waves without any."""
    n, sk, hq, hk = 5, 900, 4, 2
    lengths = [900, 1, 0, 470, 33]
    assert fs.DiffAttention(n, sq, sk, hq, hk, d, dv, dtype=DTYPE[dtype], causal=causal).info.key_splits > 1
    check(n, sq, sk, hq, hk, d, dv, dtype, causal=causal, lengths=lengths, train=sq == 7)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("causal", [False, True])
def test_many_tiles(d, dv, causal, dtype):
    """The kernels that go over all keys or rows in one workgroup (no shared
    steps), several stages long."""
    n, s, hq, hk = 40, 150, 16, 16
    info = fs.DiffAttention(n, s, s, hq, hk, d, dv, dtype=DTYPE[dtype], causal=causal).info
    assert info.key_splits == 0
    # most sequences empty, so that the reference stays small
    check(n, s, s, hq, hk, d, dv, dtype, causal=causal, lengths=[150 if b == 3 else 0 for b in range(n)])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_shared_backward_steps(dtype):
    """Few tiles of many steps: workgroups share them and their parts are added
    up; with strides that leave no 16-byte accesses, too."""
    a = check(1, 310, 290, 4, 2, 32, 64, dtype, causal=True)
    b = check(1, 310, 290, 4, 2, 32, 64, dtype, causal=True, place=_unaligned)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    check(1, 300, 280, 2, 1, 30, 50, dtype)


def test_offsets_beyond_32_bits():
    """Tokens 2^22 elements apart: the last keys lie 9 GB from the first."""
    n, sq, sk, h, d, dv = 1, 3, 1100, 1, 32, 64
    dt = torch.bfloat16
    q, k, v, lam, do = (_dev(a, dt) for a in make_inputs(11, n, sq, sk, h, h, d, dv))
    stride = 1 << 22
    big = torch.empty(sk * stride, dtype=dt, device="cuda")
    kv = big.as_strided((n, sk, h, 2 * d + dv), (0, stride, 2 * d + dv, 1))
    kv[..., :2 * d] = k.flatten(3)
    kv[..., 2 * d:] = v
    kf, vf = kv[..., :2 * d].unflatten(-1, (2, d)), kv[..., 2 * d:]
    assert kf.stride(1) == stride
    plan = fs.DiffAttention(n, sq, sk, h, h, d, dv, dtype=dt)
    near, far = [], []
    for out, kk, vv in ((near, k, v), (far, kf, vf)):
        o, saved = plan.forward(q, kk, vv, lam, save=True)
        out += [o, *plan.backward(do, q, kk, vv, lam, saved)]
    torch.cuda.synchronize()
    for x, y in zip(near, far):
        assert torch.equal(x, y)
    too_far = big.as_strided((n, 2, h, 2, d), (0, (1 << 22) + 8, 2 * d, d, 1))
    small = fs.DiffAttention(n, sq, 2, h, h, d, dv, dtype=dt)
    with pytest.raises(fs.FftsplitError) as e:
        small.forward(q, too_far, v[:, :2], lam)
    assert e.value.status == fs.ERROR_NOT_SUPPORTED


def test_refusals():
    dt = torch.float32
    q, k, v, lam, do = (_dev(a, dt) for a in make_inputs(2, 2, 8, 300, 4, 2, 16, 32))
    plan = fs.DiffAttention(2, 8, 300, 4, 2, 16, 32)
    with pytest.raises(ValueError):
        plan.forward(q[:, :7], k, v, lam)
    with pytest.raises(TypeError):
        plan.forward(q.bfloat16(), k, v, lam)
    with pytest.raises(TypeError):
        plan.forward(q.cpu(), k, v, lam)
    with pytest.raises(ValueError):
        plan.forward(q, k, v, lam[:3])
    with pytest.raises(TypeError):
        plan.forward(q, k, v, lam.double())
    with pytest.raises(TypeError):
        plan.forward(q, k, v, lam, key_lengths=torch.ones(2, device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError):
        plan.forward(q, k, v, lam, key_lengths=torch.ones(3, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        plan.forward(q.transpose(-1, -2).contiguous().transpose(-1, -2), k, v, lam)
    with pytest.raises(ValueError):
        plan.forward(q, k, v, lam, out=torch.empty(3, device="cuda"))
    assert plan.info.forward_workspace_bytes > 0
    with pytest.raises(fs.FftsplitError) as e:
        plan.forward(q, k, v, lam, workspace=torch.empty(16, device="cuda", dtype=torch.uint8))
    assert e.value.status == fs.ERROR_INSUFFICIENT_WORKSPACE
    with pytest.raises(fs.FftsplitError) as e:
        plan.forward(q, k, v, lam, out=v.view(-1)[:8 * 2 * 4 * 32].view(2, 8, 4, 32))
    assert "overlaps" in str(e.value)
    # and a sound call still works
    assert torch.isfinite(plan.forward(q, k, v, lam)).all()


def test_another_stream():
    """Enqueued on the current stream, in its order: the inputs are produced
    there behind work that takes a while."""
    n, s, h, d, dv = 2, 128, 4, 64, 128
    q, k, v, lam, do = (_dev(a, torch.bfloat16) for a in make_inputs(4, n, s, s, h, h, d, dv))
    plan = fs.DiffAttention(n, s, s, h, h, d, dv, dtype=torch.bfloat16)
    want = plan.forward(q, k, v, lam)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    q2 = torch.zeros_like(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        w = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            w = w @ w * 1e-3
        q2.copy_(q)
        got = plan.forward(q2, k, v, lam)
    side.synchronize()
    assert torch.equal(got, want)
