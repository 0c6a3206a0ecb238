"""Gradients of bf16 differential attention where sums cancel: keys and values
around a common one (dS sums to zero over a row's keys, so an error of D stays
whole where the result does not), or rows of q and dout.

Tolerance (relative L2 norm).  One rounding to bf16 is 1.7e-3 of a normally
distributed array (measured: 1.66e-3).  A gradient is rounded, and so are the
terms it is summed of, which the common part of the other factor magnifies: keys
0.5 + N(0, 1) by sqrt(1.25), to 1.9e-3.  D is a sum over o1, whose terms are
rounded as well, over values of 2 + N(0, 1) and with the mean key 0.5: 1.66e-3 *
sqrt(5) * 0.5 = 1.9e-3.  Together 3.1e-3; 4e-3 leaves room for short rows.
dlam, in fp32 and from unrounded terms: fp32's 2^-24 times its cancelling sum
over some thousand rows, below 1e-4.
"""
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

TOL = {"dq": 4e-3, "dk": 4e-3, "dv": 4e-3, "dlam": 1e-4}
WIDTHS = [(32, 64), (64, 128), (128, 256)]


def _exact(q, k, v, lam, do, seen):
    """In 64 bits, by automatic differentiation.  `seen` [n, sq, sk]."""
    q, k, v, lam = (t.detach().double().requires_grad_() for t in (q, k, v, lam))
    g = q.shape[2] // k.shape[2]
    qh = q.permute(0, 2, 3, 1, 4)
    kh = k.permute(0, 2, 3, 4, 1).repeat_interleave(g, 1)
    vh = v.permute(0, 2, 1, 3).repeat_interleave(g, 1)
    s = qh.contiguous() @ kh.contiguous() * q.shape[-1] ** -0.5
    p = s.masked_fill(~seen[:, None, None], -1e300).softmax(-1) * seen.any(-1)[:, None, None, :, None]
    o = ((p[:, :, 0] - lam.view(1, -1, 1, 1) * p[:, :, 1]) @ vh).permute(0, 2, 1, 3)
    return torch.autograd.grad(o, (q, k, v, lam), do.double())


@pytest.mark.parametrize("kind", ["keys and values", "rows"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,dv", WIDTHS)
@pytest.mark.parametrize("n,s,lengths", [(2, 333, None), (3, 200, [200, 77, 0])])
def test_gradients_around_a_common_part(n, s, lengths, d, dv, causal, kind):
    hq, hk = 4, 2
    print(f"[case] {kind} {n}x{s} {d}/{dv} causal={causal} {lengths}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(s)
    f = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    q, k, v, do = f(n, s, hq, 2, d), f(n, s, hk, 2, d), f(n, s, hk, dv), f(n, s, hq, dv)
    if kind == "rows":
        q, do = q + 0.5, do + 1
    else:
        k, v = k + 0.5, v + 2
    q, k, v, do = (t.bfloat16() for t in (q, k, v, do))
    lam = 0.2 + 0.6 * torch.rand(hq, generator=gen, device="cuda")
    kl = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    length = (torch.full((n,), s, device="cuda") if kl is None else kl).view(-1, 1, 1)
    i, j = torch.arange(s, device="cuda")[None, :, None], torch.arange(s, device="cuda")
    seen = (j < length).expand(n, s, s)
    if causal:
        seen = seen & (j <= i + length - s)
    plan = fs.DiffAttention(n, s, s, hq, hk, d, dv, dtype=torch.bfloat16, causal=causal)
    _, saved = plan.forward(q, k, v, lam, key_lengths=kl, save=True)
    got = plan.backward(do, q, k, v, lam, saved, key_lengths=kl)
    want = _exact(q, k, v, lam, do, seen)
    errors = {name: float((a.double() - b).norm() / b.norm()) for name, a, b in zip(TOL, got, want)}
    print(errors)
    for name, e in errors.items():
        assert e <= TOL[name], (name, errors)
