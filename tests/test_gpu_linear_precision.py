"""What bf16 calls of linear attention lose against 64 bits beyond the rounding of
their outputs, also where the terms of a sum cancel.

Tolerances.  A bf16 output is rounded to 2^-8 of itself at most, 1.66e-3 in the
mean square.  Operands of later products (the state before a segment, the scores)
are sums of two bf16 numbers, the first cut off and the second rounded: 2^-15 of a
value at most, 2^-16.8 in the mean square, and as much again for the terms of a
state, 2^-16.3 together.  Of a state that has a common part, which the product
cancels, that is 2^-16.3 of the common part against the rest as the signal: here the
state's common part is up to 4 * 150 (values' mean, terms that a memory of 300 tokens
holds) next to a sum of 150 terms that are independent, 12: 50 times as large, 2^-16.3
* 50 = 6.2e-4 of the output in the mean square.  With the output's own that is
1.77e-3, tested as 2e-3.
"""
import numpy as np
import pytest

from linear_reference import reference

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu

NAMES = ("o", "state", "dq", "dk", "dv")


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().cuda()


def common_parts(seed, n, s, hq, hk, d, dv, mean):
    """Keys and values with a common part, queries and gradients that add up to
    zero along it, as behind a norm; every head remembers some 300 tokens."""
    rng = np.random.default_rng(seed)
    q, k, v, do = (rng.standard_normal((n, s, h, w)) for h, w in ((hq, d), (hk, d), (hk, dv), (hq, dv)))
    k[..., :8] += 1
    q[..., :8] -= q[..., :8].mean(-1, keepdims=True)
    v += mean
    do -= do.mean(-1, keepdims=True)
    return (*(_bf16(x) for x in (q, k, v, do)), torch.full((hk,), -1 / 300, device="cuda"))


def errors(q, k, v, do, log_decay, return_state):
    n, s, hq, d = q.shape
    plan = fs.LinearAttention(n, s, hq, k.shape[2], d, v.shape[3], dtype=q.dtype)
    got = plan.forward(q, k, v, log_decay, return_state=return_state)
    o, state = got if return_state else (got, None)
    got = (o, state, *plan.backward(do, q, k, v, log_decay)[:3])
    torch.cuda.synchronize()
    want = reference(*(_np(x) for x in (q, k, v, log_decay)), do=_np(do))
    return plan, {name: np.linalg.norm(_np(g) - w) / np.linalg.norm(w) for name, g, w in zip(NAMES, got, want)
                  if g is not None}


@pytest.mark.parametrize("mean", [0, 1, 4])
@pytest.mark.parametrize("d,dv", [(64, 128), (32, 64), (40, 24), (128, 256)])
def test_states_with_a_common_part(d, dv, mean):
    """The state before a segment keeps what a product with it does not cancel.
    (The scores, rounded or not, are within 3e-3: 2.35e-3 where rounded once.)"""
    plan, off = errors(*common_parts(d, 1, 1000, 4, 2, d, dv, mean), return_state=True)
    assert plan.info.segments > 1
    for name in ("o", "dq", "dk", "dv"):
        assert off[name] <= 3e-3, (name, off)


@pytest.mark.parametrize("mean", [0, 4])
@pytest.mark.parametrize("s,state", [(300, False), (784, False), (300, True), (1000, True)])
@pytest.mark.parametrize("d,dv", [(64, 128), (40, 24)])
def test_only_the_outputs_are_rounded(d, dv, s, state, mean):
    """In sequences of one segment, and of several with a state returned."""
    plan, off = errors(*common_parts(s, 1, s, 2, 2, d, dv, mean), return_state=state)
    for name in ("o", "dq", "dk", "dv"):
        assert off[name] <= 2e-3, (name, off)


@pytest.mark.parametrize("s", [9, 128, 1000])
def test_returned_states(s):
    """A returned state's terms are bf16 numbers times fp32 weights, as three bf16
    operands that leave out nothing.  Their sums are fp32: in the mean square a
    rounding of 2^-24 / sqrt(3) for each part of the 128 terms of a segment,
    sqrt(384) of them 11 * 2^-24, and the weights (three factors and an exponent up
    to 8) 10 * 2^-24: 15 * 2^-24 = 9e-7 together, tested as 1e-6.  (Two operands
    would leave out 2.8e-6.)"""
    _, off = errors(*common_parts(s, 2, s, 2, 2, 64, 64, 0), return_state=True)
    assert off["state"] <= 1e-6, off
