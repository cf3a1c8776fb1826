"""The differentiable front ends on inputs whose rows the kernels do not take as they lie: transposed, repeated, every second column."""
import pytest
import torch

from layer_cases import Layer, draw
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu

# n, width -> (leaf, view of it of shape [n, width])
VIEWS = {
    "transposed": lambda n, width, dtype: (leaf := draw((width, n), dtype, 1).cuda().requires_grad_(), leaf.t()),
    "one row repeated": lambda n, width, dtype: (leaf := draw((width,), dtype, 2).cuda().requires_grad_(), leaf.expand(n, width)),
    "one column repeated": lambda n, width, dtype: (leaf := draw((n, 1), dtype, 3).cuda().requires_grad_(), leaf.expand(n, width)),
    "every second column": lambda n, width, dtype: (leaf := draw((n, 2 * width), dtype, 4).cuda().requires_grad_(), leaf[:, ::2]),
    "overlapping windows": lambda n, width, dtype: (leaf := draw((n + width,), dtype, 5).cuda().requires_grad_(), leaf.as_strided((n, width), (1, 1))),
    "rows apart": lambda n, width, dtype: (leaf := draw((n, width + 9), dtype, 6).cuda().requires_grad_(), leaf[:, 4:width + 4]),
}


def same(view, n, width, dtype, call):
    """Result and gradient of the view as it lies equal those of a contiguous copy, and the leaf gets its own.  (Of the view: torch adds
    up what a repeated or overlapping element gets in an order that changes.)"""
    out = []
    for copy in (False, True):
        leaf, X = VIEWS[view](n, width, dtype)
        X.retain_grad()
        Y = call(X.contiguous() if copy else X)
        Y.backward(draw(tuple(Y.shape), Y.dtype, 7).cuda())
        assert leaf.grad.shape == leaf.shape and bool(leaf.grad.isfinite().all())
        out.append((Y.detach(), X.grad))
    equal = [bool(torch.equal(a, b)) for a, b in zip(*out)]
    assert equal == [True, True]


@pytest.mark.parametrize("n", [1, 5, 70])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("view", sorted(VIEWS))
def test_product(view, dtype, n):
    m = autograd.CodesLinear(Layer(48, 192, 16, 1, 64, dtype, seed=1).on_gpu(binding))
    same(view, n, 192, dtype, m)


def test_product_of_a_single_repeated_number():
    m = autograd.CodesLinear(Layer(48, 192, 16, 1, 64, torch.float32, seed=1).on_gpu(binding))
    x = torch.tensor(0.5, device="cuda")
    assert torch.equal(m(x.expand(192)), m(torch.full((192,), 0.5, device="cuda")))
    assert torch.equal(m(x.expand(3, 2, 192)), m(torch.full((3, 2, 192), 0.5, device="cuda")))


@pytest.mark.parametrize("n,V", [(1, 300), (5, 300), (5, 40_000)])
@pytest.mark.parametrize("view", sorted(VIEWS))
def test_loss(view, n, V):
    index = torch.arange(n * 4, dtype=torch.int32).view(n, 4).cuda()
    teacher = draw((n, 4), torch.float32, 8).cuda()
    same(view, n, V, torch.float32, lambda z: autograd.distill(z, index, teacher, 2.0))
