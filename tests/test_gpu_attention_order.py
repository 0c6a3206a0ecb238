"""Differential attention where the order of workgroups and the sharing of their
steps can go wrong: numbers of heads and tiles that do not divide by the eight
L2 domains or a round of compute units, and parts of odd widths.

Tolerances and their derivation: test_gpu_attention.py.
"""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2003_12621_amd")

from test_gpu_attention import WIDTHS, check  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,hq,hk,s", [(1, 19, 19, 150), (2, 12, 4, 97), (5, 5, 5, 200), (1, 33, 3, 65), (3, 16, 16, 130)])
def test_causal_heads_and_tiles(n, hq, hk, s, dtype):
    """Bands of heads that end in a smaller one, and rounds that end inside a band."""
    check(n, s, s, hq, hk, 32, 64, dtype, causal=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_wide_heads_with_shared_steps(causal, dtype):
    """Gradients of the widest heads, by workgroups for either map and the
    values, each sharing its steps, with lengths that leave some without any."""
    check(3, 280, 300, 6, 3, 128, 256, dtype, causal=causal, lengths=[300, 17, 255])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("d,dv", [(21, 43), (22, 44), (10, 20), (65, 131)])
def test_parts_of_odd_widths(d, dv, dtype):
    """Parts whose rows do and do not divide into four values."""
    check(1, 310, 290, 2, 1, d, dv, dtype)


@pytest.mark.parametrize("d,dv", WIDTHS)
def test_more_workgroups_than_run_at_once(d, dv):
    """Several rounds of causal tiles on every compute unit."""
    check(9, 260, 260, 16, 16, d, dv, "bf16", causal=True, train=d < 128)
