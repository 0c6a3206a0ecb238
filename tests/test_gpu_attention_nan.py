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
