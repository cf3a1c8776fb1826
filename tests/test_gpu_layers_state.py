"""What the differentiable front ends keep between calls, and what they do not."""
import copy

import pytest
import torch

from layer_cases import Layer, draw
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codebook_changed_behind_autograd(dtype):
    """A change through .data moves no version counter; the next call has to see it, and a gradient to use what its forward used."""
    m = autograd.CodesLinear(Layer(48, 192, 16, 2, 64, dtype, seed=1).on_gpu(binding))
    X = draw((5, 192), dtype, 1).cuda()
    with torch.no_grad():
        Y = m(X)
        m.C.data.mul_(2.0)
        assert torch.equal(m(X), Y * 2)
        m.S.data.mul_(0.5)
        assert torch.equal(m(X), Y)
        m.C.data.copy_(torch.zeros_like(m.C))
        assert not m(X).any()


def test_module_has_its_own_parameters_and_copies():
    layer = Layer(48, 192, 16, 2, 64, torch.float32, seed=1).on_gpu(binding)
    before = layer.C.clone(), layer.S.clone()
    m = autograd.CodesLinear(layer)
    X = draw((5, 192), torch.float32, 1).cuda()
    Y = m(X).detach()
    twin = copy.deepcopy(m)
    with torch.no_grad():
        m.C.mul_(2.0)
        m.S.mul_(2.0)
    assert torch.equal(layer.C, before[0]) and torch.equal(layer.S, before[1])
    assert torch.equal(twin(X), Y) and torch.equal(m(X), 4 * Y)
    m.load_state_dict(twin.state_dict())
    assert torch.equal(m(X), Y)


def test_parameters_in_16_bits():
    """module.bfloat16(): scales go back to float32 for the product, gradients come in the parameters' type."""
    m = autograd.CodesLinear(Layer(48, 192, 16, 2, 64, torch.bfloat16, seed=1).on_gpu(binding)).bfloat16()
    X = draw((5, 192), torch.bfloat16, 1).cuda()
    m(X).sum().backward()
    assert m.C.grad.dtype == m.S.grad.dtype == torch.bfloat16 and m.words.dtype == torch.int32
    ref = autograd.CodesLinear(m.layer(torch.bfloat16))
    ref(X).sum().backward()
    assert torch.equal(ref.C.grad.bfloat16(), m.C.grad) and torch.equal(ref.S.grad.bfloat16(), m.S.grad)


@pytest.mark.parametrize("group", [0, 64])
def test_stored_between_forward_and_backward(group):
    """Storing a layer (this one's other weights, here) leaves the state that its backward pass needs."""
    W, G, C0 = draw((24, 128), torch.float32, 1).cuda(), draw((24, 128), torch.float32, 2).cuda(), torch.linspace(-2, 2, 4, device="cuda").view(4, 1)
    shape = (24, 128) if group else (24 * 128, 1)
    grads = []
    for between in (False, True):
        q = autograd.SoftKMeansQuantize(0.3, binding.DIST_SQL2, tol=1e-7, group=group)
        w = W.view(shape).clone().requires_grad_()
        Wq, _ = q(w, C0)
        if between:
            q.stored(draw((24, 128), torch.float32, 3).cuda(), C0 * 0.5)
        Wq.backward(G.view(shape))
        grads.append(w.grad)
        q.close()
    assert torch.equal(*grads)


def test_backward_of_an_earlier_grouped_call_is_refused():
    q = autograd.SoftKMeansQuantize(0.3, binding.DIST_SQL2, group=64)
    W, C0 = draw((24, 128), torch.float32, 1).cuda().requires_grad_(), torch.linspace(-2, 2, 4, device="cuda").view(4, 1)
    first, second = q(W, C0)[0], q(W * 1.5, C0)[0]
    with pytest.raises(RuntimeError, match="quantised again"):
        first.sum().backward()
    second.sum().backward()
    assert W.grad.isfinite().all()
    q.close()
