"""The differentiable front ends of embedding tables, of inputs kept in 8 bits and of layers in 8-bit integers, alone and one after another."""
import copy

import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, Layer, check, draw, sum_error
from paper_2312_07759_amd import autograd, binding

pytestmark = pytest.mark.gpu


def table_gradients(layer, ids, G, alpha):
    """dC and dS of sum(G * lookup) in float64."""
    C = layer.C.double().requires_grad_()
    w = C[torch.from_numpy(layer.codes)].reshape(layer.rows, layer.cols)
    S = None
    if layer.S is not None:
        S = layer.S.double().requires_grad_()
        w = w * S.repeat_interleave(layer.group, 1)[:, :layer.cols]
    held = ids >= 0
    (alpha * w[ids[held]] * G.double()[held]).sum().backward()
    return C.grad, None if S is None else S.grad


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("k,d,group", [(16, 1, 64), (256, 4, 0), (512, 2, 32)])
def test_codes_embedding_module(k, d, group, dtype):
    t = DTYPES[dtype]
    layer = Layer(90, 192, k, d, group, t, seed=k)
    m = autograd.CodesEmbedding(layer.on_gpu(binding), alpha=3.0)
    ids = torch.randint(-1, 90, (5, 80), generator=torch.Generator().manual_seed(1))
    Y = m(ids.cuda())
    assert Y.shape == (5, 80, 192) and Y.dtype == t
    ref = 3.0 * layer.weights()[ids.clamp(min=0)] * (ids >= 0)[..., None]
    check(Y.reshape(-1, 192), ref.reshape(-1, 192), (HALF_STEP[t] + 3 * 2.0 ** -24) * ref.reshape(-1, 192).abs() + (2.0 ** -25 if t == torch.float16 else 0))
    G = draw((5, 80, 192), t, 2)
    Y.backward(G.cuda())
    dC, dS = table_gradients(layer, ids.reshape(-1), G.reshape(-1, 192), 3.0)
    assert m.C.grad.dtype == torch.float32
    # in the norm: sums of L independent terms in float32 are off by sqrt(L) 2^-24 of their size, and few factors' roundings
    assert float((m.C.grad.double().cpu() - dC).norm() / dC.norm()) < (400 * 192 / d) ** 0.5 * 2.0 ** -24 + 2.0 ** -21
    if group:
        assert float((m.S.grad.double().cpu() - dS).norm() / dS.norm()) < (20 * group) ** 0.5 * 2.0 ** -24 + 2.0 ** -21
    # an expanded upstream gradient, a parameter that needs none, another type
    m.C.requires_grad_(False)
    if group:
        m.S.grad = None
        m(ids[0].int().cuda()).float().mean().backward()
        assert m.S.grad.isfinite().all()
    assert autograd.CodesEmbedding(layer.on_gpu(binding), dtype=torch.float32)(ids.cuda()).dtype == torch.float32


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_embedding_of_a_quantiser(dtype):
    """A table in training: quantised, looked up, and the gradient of its weights through both."""
    rows, cols, t = 40, 64, DTYPES[dtype]
    W = draw((rows, cols), torch.float32, 1).cuda().requires_grad_()
    C0 = torch.linspace(-1.5, 1.5, 4).reshape(4, 1).cuda()
    q = autograd.SoftKMeansQuantize(0.3, binding.DIST_SQL2, tol=1e-7, bwd_tol=1e-7, bwd_mode=binding.BWD_GMRES, group=32)
    ids = torch.randint(-1, rows, (7, 50), generator=torch.Generator().manual_seed(2))
    G = draw((7, 50, cols), t, 3)
    Wq, _ = q(W, C0)
    Wq.retain_grad()
    Y = autograd.embedding(ids.cuda(), Wq, 2.0, t)
    assert Y.shape == (7, 50, cols) and Y.dtype == t
    Y.backward(G.cuda())
    P, A = torch.zeros(rows, cols, dtype=torch.float64), torch.zeros(rows, cols, dtype=torch.float64)
    held = ids >= 0
    P.index_put_((ids[held],), 2 * G.double()[held], accumulate=True)
    A.index_put_((ids[held],), 2 * G.double()[held].abs(), accumulate=True)
    check(Wq.grad, P, sum_error(A, 350))
    # .. and that gradient through the quantiser is what the quantiser gives for it
    direct = W.grad.clone()
    W.grad = None
    Wq, _ = q(W, C0)
    Wq.backward(P.float().cuda())
    assert float((W.grad - direct).norm() / W.grad.norm()) < 1e-4  # the solve's tolerance 1e-7 through a system of condition about 100
    q.close()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("group", [0, 64])
def test_codes_linear_with_inputs_in_8_bits(group, dtype):
    """The output and dX are those of the layer without it; dC and dS those of the input that 8 bits keep, with the same bits."""
    t = DTYPES[dtype]
    layer = Layer(48, 200, 16, 2, group, t, seed=1).on_gpu(binding)
    plain, kept = autograd.CodesLinear(layer), autograd.CodesLinear(layer, keep8=True)
    ctx = binding.Context(0)
    X, G = draw((3, 50, 200), t, 1).cuda(), draw((3, 50, 48), t, 2).cuda()
    a, b = X.clone().requires_grad_(), X.clone().requires_grad_()
    Y, Z = plain(a), kept(b)
    assert torch.equal(Y, Z)
    Y.backward(G)
    Z.backward(G)
    assert torch.equal(a.grad, b.grad)
    ref = autograd.CodesLinear(layer)
    ref(ctx.restore8(ctx.keep8(X.view(-1, 200))).view(3, 50, 200)).backward(G)
    assert torch.equal(kept.C.grad, ref.C.grad) and not torch.equal(kept.C.grad, plain.C.grad)
    if group:
        assert torch.equal(kept.S.grad, ref.S.grad)
    # frozen parameters: nothing is kept, the gradient of the input is there
    for p in kept.parameters():
        p.requires_grad_(False)
    c = X.clone().requires_grad_()
    kept(c).backward(G)
    assert torch.equal(c.grad, a.grad)
    ctx.close()


def test_inputs_in_8_bits_take_less_memory():
    layer = Layer(32, 4096, 16, 1, 0, torch.bfloat16).on_gpu(binding)
    X = draw((2048, 4096), torch.bfloat16, 1).cuda()
    held = {}
    for keep8 in (False, True):
        m = autograd.CodesLinear(layer, keep8)
        before = torch.cuda.memory_allocated()
        Y = m(X.clone())  # the activations live only where the graph holds them
        held[keep8] = torch.cuda.memory_allocated() - before
        del Y
    # 33 bytes for 32 elements instead of 64, beside the output of either and blocks of the allocator
    assert held[True] < held[False] - 2048 * 4096 * (2 - 33 / 32) * 0.9


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_int8_linear_module(dtype):
    t = DTYPES[dtype]
    ctx = binding.Context(0)
    W = draw((50, 200), torch.float32, 1)
    layer = ctx.int8_layer(W.cuda(), t)
    m = autograd.Int8Linear(layer)
    X = draw((2, 30, 200), t, 2).cuda().transpose(0, 1).requires_grad_()  # rows that do not lie in one order
    Y = m(X)
    assert Y.shape == (30, 2, 50) and Y.dtype == t
    assert torch.equal(Y.reshape(-1, 50), ctx.int8_linear(layer, X.detach().reshape(-1, 200)))
    G = draw((30, 2, 50), t, 3)
    Y.backward(G.cuda())
    w = layer.W8[:, :200].double().cpu() * layer.scale.double().cpu()[:, None]
    ref, terms = G.double() @ w, G.double().abs() @ w.abs()
    half = HALF_STEP[t]
    bound = half * ref.abs() + half * terms + sum_error(terms, 50) + (2.0 ** -25 * (1 + G.double().abs().sum(-1, keepdim=True)) if dtype == "f16" else 0)
    check(X.grad, ref, bound)
    # .. and against differences of the product with the layer's own weights, which the gradient is of
    if dtype == "f32":
        x, v = X.detach().double().cpu(), draw((30, 2, 200), torch.float64, 4)
        f = lambda h: float(((x + h * v) @ w.t() * G.double()).sum())  # noqa: E731
        slope = (f(1e-3) - f(-1e-3)) / 2e-3
        assert abs(float((X.grad.double().cpu() * v).sum()) - slope) < 1e-4 * float((X.grad.double().cpu() * v).abs().sum())
    assert sorted(m.state_dict()) == ["W8", "scale"]
    Y = m(X)
    with torch.no_grad():
        m.scale.mul_(2)
    with pytest.raises(RuntimeError):
        Y.sum().backward()
    with pytest.raises(ValueError):
        m(X[..., :100])
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_after_another(dtype):
    """Tokens through a stored table, a stored layer with inputs in 8 bits and a layer of 8-bit integers to the loss against a teacher: the
    gradient of every parameter from the one that reached its stage."""
    width, hidden, vocab, n = 128, 192, 515, 90
    ctx = binding.Context(0)
    table, first = Layer(vocab, width, 16, 1, 32, dtype, seed=1), Layer(hidden, width, 16, 1, 64, dtype, seed=2)
    embed = autograd.CodesEmbedding(table.on_gpu(binding), alpha=0.5)
    linear = autograd.CodesLinear(first.on_gpu(binding), keep8=True)
    head_layer = ctx.int8_layer(draw((vocab, hidden), torch.float32, 3).cuda() / hidden, dtype)
    head = autograd.Int8Linear(head_layer)
    ids = torch.randint(-1, vocab, (n,), generator=torch.Generator().manual_seed(4))
    index = torch.randint(-1, vocab, (n, 6), generator=torch.Generator().manual_seed(5)).to(torch.int32)
    teacher = draw((n, 6), torch.float32, 6)
    X = embed(ids.cuda())
    H = linear(X)
    Z = head(H)
    for v in (X, H, Z):
        v.retain_grad()
    loss = autograd.distill(Z, index.cuda(), teacher.cuda(), 1.0).mean()
    loss.backward()
    half = HALF_STEP[dtype]
    # the head, from the logits' gradient
    w8 = head_layer.W8[:, :hidden].double().cpu() * head_layer.scale.double().cpu()[:, None]
    dZ = Z.grad.double().cpu()
    terms = dZ.abs() @ w8.abs()
    check(H.grad, dZ @ w8, half * ((dZ @ w8).abs() + terms) + sum_error(terms, vocab))
    # the stored layer, from its output's gradient and its kept input
    dH, x8 = H.grad.double().cpu(), ctx.restore8(ctx.keep8(X.detach())).double().cpu()
    w = first.weights()
    terms = dH.abs() @ w.abs()
    check(X.grad, dH @ w, half * ((dH @ w).abs() + terms) + sum_error(terms, hidden))
    P, A = dH.t() @ x8, dH.abs().t() @ x8.abs()
    u, s, codes = first.unscaled(), first.scales(), torch.from_numpy(first.codes)
    per = lambda v: v.reshape(hidden, -1, 64).sum(2)  # noqa: E731
    check(linear.S.grad, per(P * u), sum_error(per(A * u.abs()), n * 64))
    sums = lambda v: torch.zeros(16, 1, dtype=torch.float64).index_add_(0, codes, v.reshape(-1, 1))  # noqa: E731
    check(linear.C.grad, sums(P * s), sum_error(sums(A * s), n * hidden * width))
    # the table, from its rows' gradient
    dC, dS = table_gradients(table, ids, X.grad.double().cpu(), 0.5)
    aC, aS = table_gradients(table, ids, X.grad.double().cpu().abs(), 0.5)
    check(embed.C.grad, dC, sum_error(aC + 1e-30, n * width))
    # terms of dS: |dX| |C|
    most = int(torch.bincount(ids[ids >= 0]).max())
    size = torch.zeros(vocab, width, dtype=torch.float64)
    size.index_put_((ids[ids >= 0],), X.grad.double().cpu().abs()[ids >= 0] * 0.5, accumulate=True)
    check(embed.S.grad, dS, sum_error((size * table.unscaled().abs()).reshape(vocab, -1, 32).sum(2), most * 32))
    ctx.close()


def test_refused_arguments():
    layer = Layer(8, 64, 4, 1, 0, torch.float32).on_gpu(binding)
    m = autograd.CodesEmbedding(layer)
    with pytest.raises(TypeError):
        m(torch.zeros(3, device="cuda"))
    with pytest.raises(TypeError):
        autograd.embedding(torch.zeros(3, device="cuda"), torch.zeros(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        autograd.embedding(torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda"))
    with pytest.raises(TypeError):
        autograd.embedding(torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(4, 5, device="cuda", dtype=torch.float16))
    assert m(torch.empty(2, 0, dtype=torch.int64, device="cuda")).shape == (2, 0, 64)


def test_differentiable_calls_cannot_be_captured():
    layer = Layer(8, 128, 4, 1, 0, torch.float32).on_gpu(binding)
    W = torch.zeros(8, 128, device="cuda", requires_grad=True)
    ids, X = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, 128, device="cuda", requires_grad=True)
    ctx = binding.Context(0)
    embed, linear, head = autograd.CodesEmbedding(layer), autograd.CodesLinear(layer, keep8=True), autograd.Int8Linear(ctx.int8_layer(W.detach()))
    for call in (lambda: embed(ids), lambda: linear(X), lambda: head(X), lambda: autograd.embedding(ids, W)):
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="captured"):
            with torch.cuda.graph(graph):
                call()
    torch.cuda.synchronize()
    # without gradients they can
    out = []
    graph = torch.cuda.CUDAGraph()
    with torch.no_grad():
        ref = [embed(ids), linear(X), head(X), autograd.embedding(ids, W)]
        with torch.cuda.graph(graph):
            out = [embed(ids), linear(X), head(X), autograd.embedding(ids, W)]
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, ref))
    ctx.close()


def test_copies_and_casts_of_an_integer_layer():
    """After a call: a copy, another type of the scales, and what is loaded into them is what the next call uses."""
    ctx = binding.Context(0)
    m = autograd.Int8Linear(ctx.int8_layer(draw((50, 200), torch.float32, 1).cuda(), torch.float32))
    X = draw((7, 200), torch.float32, 2).cuda()
    Y = m(X)
    twin = copy.deepcopy(m)
    assert torch.equal(twin(X), Y)
    twin.half()
    Z = twin(X)
    with torch.no_grad():
        twin.scale.mul_(2)
    assert torch.equal(twin(X), 2 * Z) and torch.equal(m(X), Y)
    m.load_state_dict({"W8": torch.zeros_like(m.W8), "scale": m.scale.clone()})
    assert not bool(m(X).any())
    ctx.close()
