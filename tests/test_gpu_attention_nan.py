"""What is not finite in differential attention: a NaN that a row sees makes
that row NaN, and one that belongs to no visible pair reaches nothing."""
import pytest

from attention_reference import make_inputs

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

from test_gpu_attention import DTYPE, WIDTHS, _dev  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("filled,at", [(513, 512), (513, 3), (600, 599), (8192, 8191), (33, 32), (1, 0), (8192, 0)])
@pytest.mark.parametrize("map", [0, 1])
def test_nan_in_a_visible_key_of_a_long_cache(map, filled, at, d, dv, dtype):
    """Workgroups share the keys; the NaN's share may hold nothing else.  Its
    sequence's rows of that key head are NaN, all others stay as they are."""
    n, sk, hq, hk, dt = 3, 8192, 4, 2, DTYPE[dtype]
    print(f"[case] {filled} keys, NaN at {at}, map {map}, {d}/{dv} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(filled)
    f = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    q, k, v, lam = f(n, 1, hq, 2, d), f(n, sk, hk, 2, d), f(n, sk, hk, dv), torch.rand(hq, device="cuda").to(dt)
    lengths = torch.tensor([700, filled, 8192], dtype=torch.int32, device="cuda")
    plan = fs.DiffAttention(n, 1, sk, hq, hk, d, dv, dtype=dt, causal=True)
    assert plan.info.key_splits > 1
    want, kept = plan.forward(q, k, v, lam, key_lengths=lengths, save=True)
    k[1, at, 1, map, 5] = float("nan")
    o, saved = plan.forward(q, k, v, lam, key_lengths=lengths, save=True)
    torch.cuda.synchronize()
    assert torch.isfinite(want).all()
    assert torch.isnan(o[1, 0, 2:]).all()
    assert torch.isnan(saved[map][1, 0, 2:]).all() and torch.equal(saved[1 - map], kept[1 - map])
    lse, before = (x[2].view(n, hq, 2) for x in (saved, kept))
    assert torch.isnan(lse[1, 2:, map]).all() and torch.equal(lse[:, :, 1 - map], before[:, :, 1 - map])
    o[1, 0, 2:] = want[1, 0, 2:]
    assert torch.equal(o, want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
def test_nan_in_a_visible_key_of_many_rows(d, dv, dtype):
    n, s, h, dt = 3, 150, 16, DTYPE[dtype]
    q, k, v, lam, _ = (_dev(a, dt) for a in make_inputs(4, n, s, s, h, h, d, dv))
    plan = fs.DiffAttention(n, s, s, h, h, d, dv, dtype=dt, causal=True)
    assert plan.info.key_splits == 0
    want = plan.forward(q, k, v, lam)
    k[1, 70, 3, 0, 0] = float("nan")
    o = plan.forward(q, k, v, lam)
    torch.cuda.synchronize()
    assert torch.isnan(o[1, 70:, 3]).all()
    o[1, 70:, 3] = want[1, 70:, 3]
    assert torch.equal(o, want)


def _all(plan, q, k, v, lam, do, lengths):
    o, saved = plan.forward(q, k, v, lam, key_lengths=lengths, save=True)
    return (o, *plan.backward(do, q, k, v, lam, saved, key_lengths=lengths))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("sq,sk,filled", [(90, 60, [60, 20, 0, 33, 1]), (5, 900, [2, 900, 0, 4, 1]), (300, 290, [290, 7, 0, 64, 129])])
def test_rows_that_see_no_key_reach_nothing(sq, sk, filled, d, dv, dtype):
    """Whatever q and dout hold there: zero output, zero gradient of the row, and
    no part in any other."""
    n, hq, hk, dt = len(filled), 4, 2, DTYPE[dtype]
    print(f"[case] {sq}x{sk} {filled} {d}/{dv} {dtype}", flush=True)
    q, k, v, lam, do = (_dev(a, dt) for a in make_inputs(6, n, sq, sk, hq, hk, d, dv))
    lengths = torch.tensor(filled, dtype=torch.int32, device="cuda")
    plan = fs.DiffAttention(n, sq, sk, hq, hk, d, dv, dtype=dt, causal=True)
    outs = []
    for fill in (0.0, float("nan"), float("inf")):
        for b, l in enumerate(filled):
            q[b, :max(0, sq - l)], do[b, :max(0, sq - l)] = fill, fill
        outs.append(_all(plan, q, k, v, lam, do, lengths))
    torch.cuda.synchronize()
    for other in outs:
        for name, x, y in zip(("o", "dq", "dk", "dv", "dlam"), outs[0], other):
            assert torch.isfinite(x).all() and torch.equal(x, y), name
        for b, l in enumerate(filled):
            assert not other[0][b, :max(0, sq - l)].any() and not other[1][b, :max(0, sq - l)].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("sq,sk", [(90, 60), (5, 900)])
def test_rows_that_see_no_key_stay_zero_beside_a_nan(sq, sk, d, dv, dtype):
    """Next to rows that see one: NaN in the first value, and in a row's q."""
    n, h, length, dt = 2, 2, 3, DTYPE[dtype]
    q, k, v, lam, do = (_dev(a, dt) for a in make_inputs(7, n, sq, sk, h, h, d, dv))
    lengths = torch.tensor([length, 0], dtype=torch.int32, device="cuda")
    v[0, 0], q[0, sq - 1] = float("nan"), float("nan")
    plan = fs.DiffAttention(n, sq, sk, h, h, d, dv, dtype=dt, causal=True)
    o, saved = plan.forward(q, k, v, lam, key_lengths=lengths, save=True)
    dq, dk, dval, _ = plan.backward(do, q, k, v, lam, saved, key_lengths=lengths)
    torch.cuda.synchronize()
    assert torch.isnan(o[0, sq - length:]).all() and torch.isnan(dk[0, :length]).all()
    for t in (o, dq, *saved[:2]):
        assert not t[0, :sq - length].any() and not t[1].any()
    assert not dk[0, length:].any() and not dval[0, length:].any() and not dk[1].any() and not dval[1].any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sq,sk", [(90, 60), (5, 900)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_rows_that_see_no_key_do_not_depend_on_lam(value, sq, sk, dtype):
    n, h, d, dv, length, dt = 2, 2, 32, 64, 3, DTYPE[dtype]
    q, k, v, lam, do = (_dev(a, dt) for a in make_inputs(8, n, sq, sk, h, h, d, dv))
    lam[1] = value
    lengths = torch.tensor([length, 0], dtype=torch.int32, device="cuda")
    plan = fs.DiffAttention(n, sq, sk, h, h, d, dv, dtype=dt, causal=True)
    o, *grads = _all(plan, q, k, v, lam, do, lengths)
    torch.cuda.synchronize()
    assert torch.isfinite(o[:, :, 0]).all() and not torch.isfinite(o[0, sq - length:, 1]).any()
    for t in (o, grads[0]):
        assert not t[0, :sq - length].any() and not t[1].any()
    for t in grads[1:3]:
        assert not t[0, length:].any() and not t[1].any()
