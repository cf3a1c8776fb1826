"""CodesLinear(keep8=True) keeps something only where a backward pass may come."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from layer_cases import Layer, draw
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu


@pytest.fixture
def kept(monkeypatch):
    """The shapes of what is kept, in order."""
    shapes, keep8 = [], binding.Context.keep8

    def counted(self, X):
        shapes.append(tuple(X.shape))
        return keep8(self, X)

    monkeypatch.setattr(binding.Context, "keep8", counted)
    return shapes


def layer():
    return Layer(90, 640, 16, 1, 64, torch.bfloat16, seed=1).on_gpu(binding)


@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("untracked", [torch.no_grad, torch.inference_mode])
def test_nothing_is_kept_without_a_graph(kept, untracked, n):
    module, X = autograd.CodesLinear(layer(), keep8=True), draw((n, 640), torch.bfloat16, n).cuda()
    with untracked():
        Y = module(X)
    assert kept == [] and torch.equal(Y, autograd.CodesLinear(layer())(X))
    Y = module(X)  # and with one it is, once
    assert kept == [(n, 640)] and Y.requires_grad


def test_nothing_is_kept_for_frozen_parameters(kept):
    module, X = autograd.CodesLinear(layer(), keep8=True), draw((40, 640), torch.bfloat16, 1).cuda().requires_grad_()
    module.requires_grad_(False)
    module(X).sum().backward()  # dX alone, which does not need X
    assert kept == [] and X.grad is not None


def test_recomputed_forward_passes(kept):
    """Of a checkpointed block the first pass keeps nothing; gradients are those of a block that is not."""
    X = draw((40, 640), torch.bfloat16, 2).cuda()
    grads = []
    for block in (lambda m, x: m(x), lambda m, x: checkpoint(m, x, use_reentrant=True)):
        module, x = autograd.CodesLinear(layer(), keep8=True), X.clone().requires_grad_()
        kept.clear()
        Y = block(module, x)
        at_forward = len(kept)
        Y.float().square().sum().backward()
        grads.append((x.grad, module.C.grad, module.S.grad))
        assert len(kept) == 1 and at_forward == (1 if len(grads) == 1 else 0)
    assert all(torch.equal(a, b) for a, b in zip(*grads))
