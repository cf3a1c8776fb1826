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
