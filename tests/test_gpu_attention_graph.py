"""The attention block's operators captured in a HIP graph on the caller's
stream: every replay on new inputs equals an eager call, bit for bit."""
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")

pytestmark = pytest.mark.gpu


def _replay(make, fill):
    """make() enqueues the calls and returns their outputs; fill(i) puts new
    values into the inputs."""
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        make()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = make()
    for i in range(1, 5):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = make()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w), i


def _refill(*tensors):
    def fill(i):
        gen = torch.Generator(device="cuda").manual_seed(i)
        for t in tensors:
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    return fill


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,sq,sk", [(2, 200, 200), (3, 1, 2000)])
def test_attention(n, sq, sk, dtype):
    hq, hk, d, dv = 4, 2, 64, 128
    e = lambda *s: torch.empty(s, dtype=dtype, device="cuda")
    q, k, v, do = e(n, sq, hq, 2, d), e(n, sk, hk, 2, d), e(n, sk, hk, dv), e(n, sq, hq, dv)
    lam = torch.rand(hq, device="cuda").to(dtype)
    lengths = torch.tensor([sk - 3 * b for b in range(n)], dtype=torch.int32, device="cuda")
    plan = fs.DiffAttention(n, sq, sk, hq, hk, d, dv, dtype=dtype, causal=True)
    ws = plan.new_workspace(backward=True)

    def make():
        o, saved = plan.forward(q, k, v, lam, key_lengths=lengths, workspace=ws, save=True)
        return [o, *plan.backward(do, q, k, v, lam, saved, key_lengths=lengths, workspace=ws)]

    _replay(make, _refill(q, k, v, do))


@pytest.mark.parametrize("layout", ["first", "last"])
def test_layer_norm(layout):
    x = torch.empty((3, 40, 77) if layout == "first" else (3, 77, 40), device="cuda")
    dy, w, b = torch.empty_like(x), torch.rand(40, device="cuda"), torch.rand(40, device="cuda")

    def make():
        y, mean, rstd = fs.layer_norm(x, w, b, layout=layout, return_stats=True)
        return [y, *fs.layer_norm_backward(dy, x, mean, rstd, w, layout=layout)]

    _replay(make, _refill(x, dy))


def test_rotary():
    q, k = torch.empty(2, 60, 4, 32, device="cuda"), torch.empty(2, 60, 2, 32, device="cuda")
    pos = torch.randint(0, 50, (60, 2), device="cuda", dtype=torch.int32)
    freqs = torch.rand(16, device="cuda")
    _replay(lambda: list(fs.rotary(q, pos, freqs, (8, 8), other=k)), _refill(q, k))
