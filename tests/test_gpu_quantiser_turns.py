"""The order of a quantiser's calls: the library keeps the state of the last one, so an earlier one's backward pass is refused."""
import pytest
import torch

from layer_cases import draw
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu


def setup(group):
    shape = (24, 128) if group else (24 * 128, 1)
    q = autograd.SoftKMeansQuantize(0.3, binding.DIST_SQL2, tol=1e-7, group=group)
    W = draw((24, 128), torch.float32, 1).view(shape).cuda()
    return q, W, draw((24, 128), torch.float32, 2).view(shape).cuda(), torch.linspace(-2, 2, 4, device="cuda").view(4, 1)


@pytest.mark.parametrize("tracked", [True, False])
@pytest.mark.parametrize("group", [0, 64])
def test_backward_of_an_earlier_call_is_refused(group, tracked):
    q, W, G, C0 = setup(group)
    w = W.clone().requires_grad_()
    first = q(w, C0)[0]
    other = (W * 1.5).requires_grad_()
    with torch.set_grad_enabled(tracked):
        second = q(other, C0)[0]
    with pytest.raises(RuntimeError, match="quantised again"):
        first.backward(G)
    assert w.grad is None
    if tracked:
        second.backward(G)
        alone, x = setup(group)[0], (W * 1.5).requires_grad_()
        alone(x, C0)[0].backward(G)
        assert torch.equal(other.grad, x.grad)
        alone.close()
    q.close()


@pytest.mark.parametrize("group", [0, 64])
def test_backward_of_the_last_call_as_often_as_asked(group):
    q, W, G, C0 = setup(group)
    w = W.clone().requires_grad_()
    out = q(w, C0)[0]
    out.backward(G, retain_graph=True)
    once = w.grad.clone()
    out.backward(G)
    assert torch.equal(w.grad, 2 * once)
    q.close()
