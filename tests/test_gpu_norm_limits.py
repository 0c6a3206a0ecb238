"""Layer norm at the numbers of positions that its limits admit, where the
workgroups of a launch hold 2^32 threads and more: a small input repeated, whose
output has to repeat bit for bit."""
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu


def _check(base, times, c, **kw):
    w, b = torch.rand(c, device="cuda"), torch.rand(c, device="cuda")
    want = fs.layer_norm(base, w, b, **kw)
    x = base.expand(times, *base.shape).reshape(times * base.shape[0], *base.shape[1:])
    print(f"[case] {tuple(x.shape)}", flush=True)
    y, mean, rstd = fs.layer_norm(x, w, b, return_stats=True, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(part, want) for part in y.split(base.shape[0]))
    mean, rstd = mean.view(times, -1), rstd.view(times, -1)
    assert (mean == mean[0]).all() and (rstd == rstd[0]).all()
    del x, y
    torch.cuda.empty_cache()


def test_rows_of_256_threads():
    """2^24 + 2^14 rows of 257 channels, 256 threads a row."""
    _check(torch.randn(1 << 14, 257, device="cuda").bfloat16(), (1 << 10) + 1, 257)


def test_positions_of_128_threads():
    """2^21 - 2^13 maps of 9 positions: two workgroups of 1024 threads for each."""
    _check(torch.randn(1 << 13, 513, 9, device="cuda").bfloat16(), (1 << 8) - 1, 513, layout="first")
