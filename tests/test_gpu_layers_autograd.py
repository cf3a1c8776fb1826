"""The differentiable front ends of coded layers, group scales and the loss against a teacher, alone and one after another."""
import pytest
import torch

from layer_cases import HALF_STEP, Layer, check, draw, sum_error
from oracle import idkm_oracle as orc
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu


def rel(a, b):
    a, b = a.detach().double().cpu(), b.detach().double().cpu()
    return float((a - b).norm() / b.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group", [0, 64])
def test_codes_linear_module(dtype, group):
    layer = Layer(48, 192, 16, 2, group, dtype, seed=1)
    m = autograd.CodesLinear(layer.on_gpu(binding))
    X = draw((3, 7, 192), dtype, 1).cuda().requires_grad_()
    G = draw((3, 7, 48), dtype, 2)
    Y = m(X)
    assert Y.shape == (3, 7, 48) and Y.dtype == dtype
    Y.backward(G.cuda())
    C = layer.C.double().requires_grad_()
    S = layer.S.double().requires_grad_() if group else None
    x = X.detach().double().cpu().requires_grad_()
    w = C[torch.from_numpy(layer.codes)].reshape(48, 192)
    if group:
        w = w * S.repeat_interleave(group, 1)
    (x @ w.t()).backward(G.double())
    terms = x.detach().abs() @ w.detach().abs().t()
    bound = HALF_STEP[dtype] * (x @ w.t()).detach().abs() + sum_error(terms, 192)
    check(Y.cpu(), (x @ w.t()).detach(), bound)
    # In the norm: rounding a scaled weight and the result, each by at most half a step, and L float32 additions, each off by at
    # most 2^-24 of a partial sum, whose mean square is at most the whole sum's (the terms are independent): sqrt(L) 2^-24.
    two = lambda length: 2 * HALF_STEP[dtype] + length ** 0.5 * 2.0 ** -24  # noqa: E731
    dx = rel(X.grad, x.grad)
    assert dx < two(48)
    assert rel(m.C.grad, C.grad) < 1e-5
    if group:
        assert rel(m.S.grad, S.grad) < 1e-5
    else:
        assert m.S is None
    # only what is asked for; a parameter that changes is seen by the next call
    X2 = draw((4, 192), dtype, 3).cuda()
    m.C.grad = None
    m(X2).float().sum().backward()
    assert m.C.grad is not None
    with torch.no_grad():
        m.C.mul_(2)
        doubled = rel(m(X2), 2 * (X2.double().cpu() @ w.detach().t()))
        assert doubled < two(192)


def test_a_changed_parameter_is_noticed_between_forward_and_backward():
    m = autograd.CodesLinear(Layer(16, 64, 4, 1, 32, torch.float32).on_gpu(binding))
    Y = m(draw((5, 64), torch.float32, 1).cuda().requires_grad_())
    with torch.no_grad():
        m.S.add_(1)
    with pytest.raises(RuntimeError):
        Y.sum().backward()


@pytest.mark.parametrize("d,group", [(1, 64), (2, 32), (1, 500)])
def test_grouped_quantiser_gradient(d, group):
    """The gradient through scales, solve and unscaling against the oracle's gradient between the scales' formulas."""
    rows, cols, k, tau = 24, 130 * d, 4, 0.3
    W = (draw((rows, cols), torch.float32, 1) * torch.exp(draw((rows, 1), torch.float32, 2))).cuda().requires_grad_()
    C0 = torch.linspace(-1.5, 1.5, k).reshape(k, 1).repeat(1, d).contiguous().cuda()
    q = autograd.SoftKMeansQuantize(tau, binding.DIST_SQL2, tol=1e-7, bwd_tol=1e-7, bwd_mode=binding.BWD_GMRES, group=group)
    Wq, C = q(W, C0)
    G = draw((rows, cols), torch.float32, 3)
    Wq.backward(G.cuda())
    w = W.detach().double().cpu().requires_grad_()
    g = min(group, cols)
    S = torch.stack([w[:, c:c + g].square().mean(1).sqrt() for c in range(0, cols, g)], 1)
    wide = S.repeat_interleave(g, 1)[:, :cols]
    Z = w / wide
    z = Z.detach().numpy().reshape(-1, d)
    Cg = C.double().cpu().numpy()
    Zq = torch.from_numpy(orc.soft_quantize(z, Cg, tau, binding.DIST_SQL2)).reshape(rows, cols)
    assert rel(Wq, Zq * wide.detach()) < 1e-4
    dZq = (G.double() * wide).detach().numpy().reshape(-1, d)
    dZ = torch.from_numpy(orc.backward(z, Cg, tau, binding.DIST_SQL2, dZq, "dense")["dW"]).reshape(rows, cols)
    ((Z * dZ).sum() + (wide * (G.double() * Zq)).sum()).backward()
    assert rel(W.grad, w.grad) < 1e-3
    q.close()


def test_distill_is_differentiable():
    z = (3 * draw((6, 300), torch.float32, 1)).cuda().requires_grad_()
    index = torch.randint(-1, 300, (6, 9), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    teacher = draw((6, 9), torch.float32, 2)
    loss = autograd.distill(z, index.cuda(), teacher.cuda(), 2.0)
    weight = draw((6,), torch.float32, 3).abs()
    (loss * weight.cuda()).sum().backward()
    zr = z.detach().double().cpu().requires_grad_()
    total = 0
    for t in range(6):
        held = index[t] >= 0
        lp = torch.log_softmax(teacher[t][held].double() / 2.0, 0)
        lq = torch.log_softmax(zr[t] / 2.0, 0)[index[t][held].long()]
        total = total + weight[t].double() * (lp.exp() * (lp - lq)).sum()
    total.backward()
    assert rel(z.grad, zr.grad) < 1e-5 and abs(float((loss.double().cpu() * weight.double()).sum()) - float(total)) < 1e-5 * abs(float(total))
    # the mean over rows: an expanded upstream gradient
    z.grad = None
    autograd.distill(z, index.cuda(), teacher.cuda(), 2.0).mean().backward()
    assert z.grad.isfinite().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_from_weights_to_a_trained_codebook(dtype):
    """A two-layer classifier quantised with group scales, stored, and its codebooks, scales and input trained one step against the
    unquantised network's largest logits: every gradient against float64 of the same stored network."""
    torch.manual_seed(0)
    n, width, hidden, classes, top, tau = 37, 128, 192, 515, 8, 2.0
    W1, W2 = torch.randn(hidden, width) / width ** 0.5, torch.randn(classes, hidden) / hidden ** 0.5
    x0 = torch.randn(n, width)
    teacher, index = torch.topk(torch.relu(x0 @ W1.t()) @ W2.t(), top, 1)
    q = autograd.SoftKMeansQuantize(0.05, binding.DIST_SQL2, max_iter=30, group=64)
    C0 = torch.linspace(-2, 2, 16).reshape(16, 1).cuda()
    l1, l2 = (autograd.CodesLinear(q.stored(w.cuda(), C0, dtype)) for w in (W1, W2))
    x = x0.to(dtype).cuda().requires_grad_()
    h = torch.relu(l1(x))
    loss = autograd.distill(l2(h), index.to(torch.int32).cuda(), teacher.cuda(), tau).mean()
    loss.backward()

    leaves = []

    def weights(layer):
        with torch.no_grad():
            unscaled = q.ctx.unpack_quantize(layer.words, layer.rows * layer.cols, torch.arange(16.0, device="cuda").reshape(16, 1))
        codes = unscaled.long().cpu().view(layer.rows, layer.cols)
        C, S = layer.C.detach().to(dtype).double().cpu().view(-1).requires_grad_(), layer.S.detach().double().cpu().requires_grad_()
        leaves.append((layer, C, S))
        return C[codes] * S.repeat_interleave(64, 1)[:, : layer.cols]

    w1, w2 = weights(l1), weights(l2)
    assert rel(w1, W1) < 0.3 and rel(w2, W2) < 0.3                      # 16 levels
    xr = x.detach().double().cpu().requires_grad_()
    hr = torch.relu(xr @ w1.t())
    if dtype == torch.bfloat16:
        hr = hr + (h.detach().double().cpu() - hr).detach()             # the same rounded activations
    lp = torch.log_softmax(teacher.double() / tau, 1)
    lq = torch.log_softmax(hr @ w2.t() / tau, 1).gather(1, index)
    ref = (lp.exp() * (lp - lq)).sum(1).mean()
    ref.backward()
    step = HALF_STEP[dtype]
    assert abs(float(loss) - float(ref)) < 8 * step * (1 + abs(float(ref)))
    # a few roundings of independent values on the way to each gradient: their size, not their number, tells in the norm
    assert rel(x.grad, xr.grad) < 8 * step + 1e-5
    for layer, C, S in leaves:
        assert rel(layer.C.grad.view(-1), C.grad) < 8 * step + 1e-5 and rel(layer.S.grad, S.grad) < 8 * step + 1e-5
    q.close()


def test_refusals():
    m = autograd.CodesLinear(Layer(16, 64, 4, 1, 32, torch.float32).on_gpu(binding))
    with pytest.raises(ValueError):
        m(torch.zeros(2, 63, device="cuda"))
    with pytest.raises(TypeError):
        m(torch.zeros(2, 64, device="cuda", dtype=torch.float64))
    q = autograd.SoftKMeansQuantize(0.1, binding.DIST_SQL2, group=33)
    with pytest.raises(ValueError):
        q.stored(torch.zeros(4, 64, device="cuda"), torch.zeros(4, 1, device="cuda"))
    with pytest.raises(ValueError):
        q(torch.zeros(4, 63, device="cuda"), torch.zeros(4, 2, device="cuda"))
    with pytest.raises(ValueError):
        autograd.SoftKMeansQuantize(0.1, binding.DIST_SQL2, group=-1)
    q.close()
    X = torch.zeros(2, 64, device="cuda")
    with torch.no_grad():
        m(X)                                                            # makes the layer outside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="captured"):
            m(X)
        with torch.no_grad():
            Y = m(X)
    for i in range(3):
        X.copy_(draw((2, 64), torch.float32, i).cuda())
        graph.replay()
        with torch.no_grad():
            assert torch.equal(Y, m(X))
