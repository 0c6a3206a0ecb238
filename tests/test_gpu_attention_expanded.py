"""Differential attention on tensors whose rows lie closer together than they
are wide: expanded over the tokens (stride 0, as the gradient of a sum over
tokens is), overlapping windows, and one token with any stride.

Where a tensor lies does not change what is computed, so every result equals
that of a dense copy bit for bit.
"""
import pytest

from attention_reference import make_inputs

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

from test_gpu_attention import DTYPE, WIDTHS, _dev, check  # noqa: E402

pytestmark = pytest.mark.gpu


def _rows(shape, dtype, seed, step, lead):
    """A tensor of this [batch, tokens, ...] shape whose tokens start `step`
    elements apart, `lead` elements into its memory."""
    width = 1
    for s in shape[2:]:
        width *= s
    gen = torch.Generator(device="cuda").manual_seed(seed)
    batch = (step * (shape[1] - 1) + width + 7) // 8 * 8
    memory = torch.randn(lead + shape[0] * batch, generator=gen, device="cuda").to(dtype)
    inner, size = [], width
    for s in shape[2:]:
        size //= s
        inner.append(size)
    return memory.as_strided(shape, (batch, step, *inner), lead)


def _run(plan, q, k, v, lam, do):
    o, saved = plan.forward(q, k, v, lam, save=True)
    return (o, *plan.backward(do, q, k, v, lam, saved))


def _compare(n, sq, sk, hq, hk, d, dv, dtype, causal, step, lead=0, names=("q", "k", "v", "do")):
    print(f"[case] {n}x{sq}x{sk} {hq}/{hk} {d}/{dv} {dtype} causal={causal} step={step} lead={lead} {names}", flush=True)
    dt = DTYPE[dtype]
    shapes = {"q": (n, sq, hq, 2, d), "k": (n, sk, hk, 2, d), "v": (n, sk, hk, dv), "do": (n, sq, hq, dv)}
    t = {}
    for i, (name, shape) in enumerate(shapes.items()):
        width = shape[-1] * (shape[2] if len(shape) == 4 else 2 * shape[2])
        t[name] = _rows(shape, dt, i, step if name in names else width, lead if name in names else 0)
    lam = torch.rand(hq, device="cuda").to(dt)
    plan = fs.DiffAttention(n, sq, sk, hq, hk, d, dv, dtype=dt, causal=causal)
    got = _run(plan, t["q"], t["k"], t["v"], lam, t["do"])
    want = _run(plan, *(t[i].contiguous() for i in ("q", "k", "v")), lam, t["do"].contiguous())
    torch.cuda.synchronize()
    for name, x, y in zip(("o", "dq", "dk", "dv", "dlam"), got, want):
        assert torch.isfinite(x).all() and torch.equal(x, y), name


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("s", [45, 196, 310])
def test_expanded_over_tokens(s, lead, causal, dtype):
    """One row for all tokens; from memory with and without 16-byte alignment."""
    _compare(1, s, s, 4, 2, 32, 64, dtype, causal, 0, lead)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
def test_each_tensor_at_each_width(name, d, dv, dtype):
    _compare(2, 70, 75, 2, 1, d, dv, dtype, False, 0, names=(name,))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("step", [8, 3])
def test_overlapping_windows(step, dtype):
    """Rows that share elements with the next ones."""
    _compare(2, 77, 90, 2, 2, 32, 64, dtype, True, step)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sk", [1, 40])
def test_one_token_with_any_stride(sk, dtype):
    """The stride of a dimension of one token has no meaning, whatever it is:
    2^28 of 4 or 2^29 of 8 bytes wrap round in 32 bits."""
    n, h, d, dv, dt = 2, 2, 32, 64, DTYPE[dtype]
    q, k, v, lam, do = (_dev(a, dt) for a in make_inputs(1, n, 1, sk, h, h, d, dv))
    plan = fs.DiffAttention(n, 1, sk, h, h, d, dv, dtype=dt)
    want = _run(plan, q, k, v, lam, do)
    for stride in (0, 1, 1 << 26, 1 << 28, 1 << 30, (1 << 40) + 8):
        far = lambda t: t.as_strided(t.shape, (t.stride(0), stride, *t.stride()[2:])) if t.shape[1] == 1 else t
        got = _run(plan, far(q), far(k), far(v), lam, far(do))
        torch.cuda.synchronize()
        for name, x, y in zip(("o", "dq", "dk", "dv", "dlam"), got, want):
            assert torch.equal(x, y), (name, stride)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_of_a_sum_over_tokens(dtype, monkeypatch):
    """Against the definition in 64 bits, at the tolerances of test_gpu_attention.py."""
    def equal_rows(*args):
        q, k, v, lam, do = make_inputs(*args)
        do[:] = do[:, :1]
        return q, k, v, lam, do

    def place(t):
        return t[:, :1].expand_as(t) if t.dim() == 4 and t.shape[1] == 50 else t

    monkeypatch.setattr("test_gpu_attention.make_inputs", equal_rows)
    check(2, 50, 61, 4, 2, 32, 64, dtype, place=place)
