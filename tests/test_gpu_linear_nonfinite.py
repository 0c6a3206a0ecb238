"""What an infinity or a NaN in a linear attention call reaches: the state's column
from its token on and the outputs that take it, and nothing else, whether tokens go
one by one, as one segment or in several."""
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

TILE = 32


def _run(plan, q, k, v, do, log_decay, state, returned):
    if returned:
        o, last = plan.forward(q, k, v, log_decay, state=state, return_state=True)
        grads = plan.backward(do, q, k, v, log_decay, state=state, dstate=state)
    else:
        o, last = plan.forward(q, k, v, log_decay), None
        grads = plan.backward(do, q, k, v, log_decay)
    torch.cuda.synchronize()
    return o, last, *grads


def _make(s, dtype):
    gen = torch.Generator(device="cuda").manual_seed(s)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    n, hq, hk, d, dv = 2, 4, 2, 40, 72
    x = [rand(n, s, h, w).to(dtype) for h, w in ((hq, d), (hk, d), (hk, dv), (hq, dv))]
    return (*x, torch.tensor([-0.01, -0.3], device="cuda"), rand(n, hk, d, dv)), fs.LinearAttention(n, s, hq, hk, d, dv,
                                                                                                   dtype=dtype)


def _same(got, want, but):
    """Equal bit for bit but where `but` is true, and not finite nowhere else."""
    return torch.equal(torch.where(but, torch.zeros_like(got), got), torch.where(but, torch.zeros_like(want), want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("s,returned", [(6, True), (9, True), (150, False), (150, True), (700, True)])
def test_value(s, returned, value, dtype):
    x, plan = _make(s, dtype)
    want = _run(plan, *x, returned)
    b, t, g, c = 1, (2 * s) // 3, 0, 5
    v = x[2].clone()
    v[b, t, g, c] = value
    o, last, dq, dk, dv, dstate = _run(plan, *x[:2], v, *x[3:], returned)
    heads = slice(2 * g, 2 * g + 2)
    first = t if plan.info.recurrent else t // TILE * TILE      # of the rows that multiply it, if only by zero
    tile = t // TILE * TILE                                     # (the backward pass goes by tiles always)
    reached = torch.zeros_like(o, dtype=torch.bool)
    reached[b, first:, heads, c] = True
    assert _same(o, want[0], reached) and not torch.isfinite(o[b, t:, heads, c]).any()
    if returned:
        reached = torch.zeros_like(last, dtype=torch.bool)
        reached[b, g, :, c] = True
        assert _same(last, want[1], reached) and not torch.isfinite(last[b, g, :, c]).any()
        assert torch.equal(dstate, want[5])
    reached = torch.zeros_like(dq, dtype=torch.bool)
    reached[b, tile:, heads] = True
    assert _same(dq, want[2], reached) and not torch.isfinite(dq[b, t:, heads]).any()
    reached = torch.zeros_like(dk, dtype=torch.bool)
    reached[b, t, g] = True
    assert _same(dk, want[3], reached) and not torch.isfinite(dk[b, t, g]).any()
    assert torch.equal(dv, want[4])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("s,returned", [(6, True), (150, False), (700, True)])
def test_query(s, returned, dtype):
    """A query reaches its own output, no state, and the gradients of the keys and
    values up to its tile's end."""
    x, plan = _make(s, dtype)
    want = _run(plan, *x, returned)
    b, t, h = 0, s // 3, 3
    q = x[0].clone()
    q[b, t, h, 7] = float("nan")
    o, last, dq, dk, dv, dstate = _run(plan, q, *x[1:], returned)
    reached = torch.zeros_like(o, dtype=torch.bool)
    reached[b, t, h] = True
    assert _same(o, want[0], reached) and torch.isnan(o[b, t, h]).all()
    assert torch.equal(dq, want[2]) and (not returned or torch.equal(last, want[1]))
    end = (t // TILE + 1) * TILE
    for got, i in ((dk, 3), (dv, 4)):
        reached = torch.zeros_like(got, dtype=torch.bool)
        reached[b, :end, h // 2] = True
        assert _same(got, want[i], reached) and not torch.isfinite(got[b, :t + 1, h // 2]).all()
    if returned:
        assert torch.isnan(dstate[b, h // 2, 7]).all()
