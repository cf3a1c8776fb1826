"""A product's gradient uses the codebook and the scales that its forward used."""
import pytest
import torch

from layer_cases import Layer, draw
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 5, 300])
@pytest.mark.parametrize("group", [0, 64])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_parameters_changed_through_data_between_forward_and_backward(dtype, group, n):
    X, G = draw((n, 192), dtype, 1).cuda(), draw((n, 48), dtype, 2).cuda()
    grads = []
    for change in (False, True):
        m = autograd.CodesLinear(Layer(48, 192, 16, 2, group, dtype, seed=1).on_gpu(binding))
        x = X.clone().requires_grad_()
        Y = m(x)
        if change:
            m.C.data.mul_(3.0)
            if group:
                m.S.data.add_(1.0)
        Y.backward(G)
        grads.append([x.grad, m.C.grad] + ([m.S.grad] if group else []))
    assert [bool(torch.equal(a, b)) for a, b in zip(*grads)] == [True] * len(grads[0])


def test_nothing_is_copied_without_a_gradient():
    m = autograd.CodesLinear(Layer(48, 192, 16, 2, 64, torch.float32, seed=1).on_gpu(binding))
    X, made = draw((5, 192), torch.float32, 1).cuda(), []
    plain = m.layer
    m.layer = lambda dtype, copy=False: made.append(plain(dtype, copy)) or made[-1]
    with torch.no_grad():
        m(X)
    m(X)
    assert [x.C.data_ptr() == m.C.data_ptr() for x in made] == [x.S.data_ptr() == m.S.data_ptr() for x in made] == [True, False]


def test_parameters_that_are_no_longer_contiguous():
    """A codebook and scales replaced by views."""
    m = autograd.CodesLinear(Layer(48, 192, 16, 2, 64, torch.float32, seed=1).on_gpu(binding))
    X = draw((5, 192), torch.float32, 1).cuda()
    Y = m(X).detach()
    m.C.data, m.S.data = m.C.data.t().contiguous().t(), m.S.data.t().contiguous().t()
    assert not m.C.is_contiguous() and not m.S.is_contiguous()
    Z = m(X)
    Z.sum().backward()
    assert bool(torch.equal(Z, Y)) and bool(m.S.grad.isfinite().all())
