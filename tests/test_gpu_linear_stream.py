"""The linear attention block where a stream's state goes on while a frame's
gradients are still to come."""
import pytest

torch = pytest.importorskip("torch")
fs = pytest.importorskip("paper_2003_12621_amd")
from paper_2003_12621_amd.block import LinearAttentionBlock  # noqa: E402

pytestmark = pytest.mark.gpu


def test_saved_state_is_the_one_that_forward_was_given():
    """step() writes its state in place; gradients of a frame that began with the
    same tensor are those of what it held then."""
    n, c, h, w = 2, 32, 6, 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    block = LinearAttentionBlock(n, c, h, w, 4, 2, 24, 40, seed=2)
    x, dy, pixel = rand(n, c, h, w), rand(n, c, h, w), rand(n, c)
    state, ds = rand(*block.frame.state_shape), rand(*block.frame.state_shape)
    _, _, saved = block.forward(x, state, frame=1, save=True)
    dx, grads, first = block.backward(dy, x, saved, dstate=ds)
    _, _, saved = block.forward(x, state, frame=1, save=True)
    before = state.clone()
    block.step(pixel, state, torch.tensor([1, 0, 0], dtype=torch.int32, device="cuda"))
    assert not torch.equal(state, before)
    dx2, grads2, first2 = block.backward(dy, x, saved, dstate=ds)
    torch.cuda.synchronize()
    assert torch.equal(dx2, dx) and torch.equal(first2, first)
    assert all(torch.equal(grads2[i], grads[i]) for i in grads)
