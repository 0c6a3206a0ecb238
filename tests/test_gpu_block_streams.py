"""One attention block used on two streams at once, and in a graph that is
replayed beside eager calls."""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2003_12621_amd")
from paper_2003_12621_amd.block import AttentionBlock  # noqa: E402

pytestmark = pytest.mark.gpu


def _step(block, x, dy):
    y, saved = block.forward(x, save=True)
    dx, grads = block.backward(dy, x, saved)
    return [y, dx, *grads.values()]


def _inputs(shape, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda"), torch.randn(shape, generator=gen, device="cuda")


def test_two_streams():
    shape = (4, 64, 28, 28)
    block = AttentionBlock(*shape, heads=4, heads_k=2, dim=32, seed=1)
    inputs = [_inputs(shape, i) for i in range(2)]
    want = [[t.clone() for t in _step(block, *i)] for i in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for _ in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                results.append((i, _step(block, *inputs[i])))
    torch.cuda.synchronize()
    for i, got in results:
        for a, b in zip(got, want[i]):
            assert torch.equal(a, b)


def test_graph_beside_eager_calls():
    shape = (2, 64, 14, 14)
    block = AttentionBlock(*shape, heads=4, heads_k=2, dim=32, seed=2)
    (x, dy), other = _inputs(shape, 3), _inputs(shape, 4)
    want, beside = (_step(block, *i) for i in ((x, dy), other))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(block, x, dy)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _step(block, x, dy)
    for _ in range(4):
        with torch.cuda.stream(side):
            graph.replay()
        got = _step(block, *other)
        torch.cuda.synchronize()
        for a, b in zip([*outs, *got], [*want, *beside]):
            assert torch.equal(a, b)
