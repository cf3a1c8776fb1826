"""Coded layers and the loss where sizes, addresses and the order of calls are at their edges."""
import numpy as np
import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, Layer, check, draw, sum_error
from oracle import idkm_oracle as orc
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def test_captured_before_any_eager_call():
    """Nothing that a first call does (attributes of kernels with much LDS, workspaces) may fail under capture."""
    c = binding.Context(0)
    cases = [(Layer(200, 640, 64, 1, 32, torch.float16, seed=n), n) for n in (1, 20, 600, 3000)]
    made = [(g.on_gpu(binding), draw((n, 640), torch.float16, n).cuda(), draw((n, 200), torch.float16, n + 1).cuda()) for g, n in cases]
    z = draw((300, 70_000), torch.float16, 9).cuda()
    index, teacher, weight = torch.arange(300 * 4, dtype=torch.int32).view(300, 4).cuda(), draw((300, 4), torch.float32, 1).cuda(), torch.ones(300, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [(c.codes_linear(g, X), c.codes_linear_backward(g, X, dY)) for g, X, dY in made]
        loss = c.distill(z, index, teacher, 1.0, weight)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        for (g, X, dY), (Y, r) in zip(made, got):
            assert torch.equal(Y, c.codes_linear(g, X))
            r2 = c.codes_linear_backward(g, X, dY)
            assert all(torch.equal(r[key], r2[key]) for key in r2)
        assert all(torch.equal(a, b) for a, b in zip(loss, c.distill(z, index, teacher, 1.0, weight)))
    c.close()


def test_two_streams_at_once(ctx):
    layer = Layer(300, 1024, 16, 1, 128, torch.bfloat16, seed=1).on_gpu(binding)
    X = [draw((n, 1024), torch.bfloat16, n).cuda() for n in (1, 40, 400, 41)]
    dY = [draw((x.shape[0], 300), torch.bfloat16, 7).cuda() for x in X]
    ref = [(ctx.codes_linear(layer, x), ctx.codes_linear_backward(layer, x, g)) for x, g in zip(X, dY)]
    streams = [torch.cuda.Stream() for _ in X]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for x, g, s in zip(X, dY, streams):
            with torch.cuda.stream(s):
                got.append((ctx.codes_linear(layer, x), ctx.codes_linear_backward(layer, x, g)))
        torch.cuda.synchronize()
        for (Y, r), (Y0, r0) in zip(got, ref):
            assert torch.equal(Y, Y0) and all(torch.equal(r[key], r0[key]) for key in r0)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n", [1, 3, 20, 500])
def test_tensors_that_begin_anywhere(ctx, n, dtype):
    """Codes, codebook, scales, activations and outputs one element behind an aligned address."""
    t = DTYPES[dtype]
    layer = Layer(50, 320, 16, 1, 64, t, seed=2)

    def off(x):
        flat = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
        flat[1:] = x.reshape(-1).cuda()
        return flat[1:].view(x.shape)

    X, dY = draw((n, 320), t, 1), draw((n, 50), t, 2)
    plain = layer.on_gpu(binding)
    moved = binding.CodesLayer(off(layer.words), 50, 320, off(layer.C), off(layer.S), 64)
    out = off(torch.zeros(n, 50, dtype=t))
    assert torch.equal(ctx.codes_linear(moved, off(X), out=out), ctx.codes_linear(plain, X.cuda()))
    a, b = ctx.codes_linear_backward(moved, off(X), off(dY)), ctx.codes_linear_backward(plain, X.cuda(), dY.cuda())
    assert all(torch.equal(a[key], b[key]) for key in b)


@pytest.mark.parametrize("n,rows,cols,k,d", [(100_003, 3, 5, 4, 1), (70_000, 1, 8, 256, 8), (5_000, 130, 12, 7, 3), (1, 100_000, 40, 16, 1),
                                             (2, 3, 100_000, 16, 2), (33, 2, 60_000, 3, 1)])
def test_long_and_narrow(ctx, n, rows, cols, k, d):
    for dtype in (torch.float32, torch.bfloat16):
        layer = Layer(rows, cols, k, d, 0, dtype, seed=3)
        X, dY = draw((n, cols), dtype, 1), draw((n, rows), dtype, 2)
        w, x, y = layer.weights(), X.double(), dY.double()
        ref = x @ w.t()
        check(ctx.codes_linear(layer.on_gpu(binding), X.cuda()), ref, HALF_STEP[dtype] * ref.abs() + sum_error(x.abs() @ w.abs().t(), cols), "Y")
        got = ctx.codes_linear_backward(layer.on_gpu(binding), X.cuda(), dY.cuda())
        ref = y @ w
        check(got["dX"], ref, HALF_STEP[dtype] * ref.abs() + sum_error(y.abs() @ w.abs(), rows), "dX")
        P, Pa = y.t() @ x, y.abs().t() @ x.abs()
        codes = torch.from_numpy(layer.codes)
        parts = lambda v: torch.zeros(k, d, dtype=torch.float64).index_add_(0, codes, v.reshape(-1, d))  # noqa: E731
        check(got["dC"], parts(P), sum_error(parts(Pa), n + rows * cols // k) + 2.0 ** -24 * parts(P).abs(), "dC")


def big_layer(rows, cols, k, group, dtype):
    """A layer too large for the host's oracle: random words (k a power of two makes every stream valid), weights on the GPU."""
    bits = binding.code_bits(k)
    g = torch.Generator(device="cuda").manual_seed(5)
    words = torch.randint(-2 ** 31, 2 ** 31, (binding.code_words(rows * cols, k),), dtype=torch.int64, device="cuda", generator=g).to(torch.int32)
    Cb = torch.randn(k, 1, device="cuda", generator=g).to(dtype)
    S = torch.rand(rows, -(-cols // group), device="cuda", generator=g) + 0.5 if group else None
    layer = binding.CodesLayer(words, rows, cols, Cb, S, group)

    def weights(r0, r1):
        at = torch.arange(r0 * cols, r1 * cols, device="cuda") * bits
        code = ((words[at >> 5].long() & 0xFFFFFFFF) >> (at & 31)) & (k - 1)     # bits divides 32
        w = Cb.double()[code, 0].view(r1 - r0, cols)
        return w if S is None else w * S[r0:r1].double().repeat_interleave(group, 1)[:, :cols]

    return layer, weights


@pytest.mark.parametrize("n", [1, 4, 20])
def test_more_weights_than_31_bits_count(ctx, n):
    """Offsets of codes beyond 2^31 and of bits beyond 2^32, first, middle and last rows."""
    rows, cols, dtype = 36_000, 65_536, torch.bfloat16
    layer, weights = big_layer(rows, cols, 16, 128, dtype)
    X = draw((n, cols), dtype, 1).cuda()
    Y = ctx.codes_linear(layer, X)
    for r0 in (0, 17_990, 32_760, rows - 16):
        w = weights(r0, r0 + 16)
        ref, terms = X.double() @ w.t(), X.double().abs() @ w.abs().t()
        check(Y[:, r0:r0 + 16], ref.cpu(), (HALF_STEP[dtype] * ref.abs() + sum_error(terms, cols)).cpu())


def test_layers_in_panels(ctx):
    """A layer that is written out and whose P is formed in several pieces, against the layer's parts."""
    rows, cols, n, k, dtype = 40_000, 4_096, 700, 16, torch.bfloat16
    layer, weights = big_layer(rows, cols, k, 128, dtype)
    X, dY = draw((n, cols), dtype, 1).cuda(), draw((n, rows), dtype, 2).cuda()
    Y = ctx.codes_linear(layer, X)
    r = ctx.codes_linear_backward(layer, X, dY)
    step = HALF_STEP[dtype]
    dX, dXa = torch.zeros(n, cols, dtype=torch.float64, device="cuda"), torch.zeros(n, cols, dtype=torch.float64, device="cuda")
    for r0 in range(0, rows, 8_000):
        w = weights(r0, r0 + 8_000)
        y = dY[:, r0:r0 + 8_000].double()
        dX += y @ w
        dXa += y.abs() @ w.abs()
        if r0 in (0, 32_000):
            s = slice(r0 + 7_900, r0 + 8_000)
            ws = w[7_900:]
            ref, terms = X.double() @ ws.t(), X.double().abs() @ ws.abs().t()
            check(Y[:, s], ref.cpu(), (step * ref.abs() + sum_error(terms, cols) + step * terms).cpu(), "Y")
            P, Pa = dY[:, s].double().t() @ X.double(), dY[:, s].double().abs().t() @ X.double().abs()
            u = ws / layer.S[s].double().repeat_interleave(128, 1)
            by = lambda v: v.view(100, 32, 128).sum(2)  # noqa: E731
            check(r["dS"][s], by(P * u).cpu(), sum_error(by(Pa * u.abs()), n + 128).cpu(), "dS")
    check(r["dX"], dX.cpu(), (step * dX.abs() + sum_error(dXa, rows) + step * dXa).cpu(), "dX")
    # sum of all bins times codewords = sum of scales times their gradients = sum of dY Y (before its rounding)
    a = float((r["dC"].double() * layer.C.double()).sum())
    b = float((r["dS"].double() * layer.S.double()).sum())
    assert abs(a - b) < 1e-5 * float((r["dS"].double() * layer.S.double()).abs().sum())


@pytest.mark.parametrize("n,V,top", [(70_001, 16, 3), (5, 4_000, 1024), (1, 1_048_577, 7), (300, 131_073, 2), (257, 65_537, 1)])
def test_many_rows_long_lists_and_long_rows(ctx, n, V, top):
    g = torch.Generator(device="cuda").manual_seed(n)
    z = 3 * torch.randn(n, V, device="cuda", generator=g)
    index = torch.randint(0, V, (n, top), device="cuda", generator=g).to(torch.int32)
    teacher, weight = torch.randn(n, top, device="cuda", generator=g), torch.rand(n, device="cuda", generator=g)
    loss, lse, dz = ctx.distill(z, index, teacher, 1.5, weight)
    q, lp = torch.log_softmax(z.double() / 1.5, 1), torch.log_softmax(teacher.double() / 1.5, 1)
    ref = (lp.exp() * (lp - q.gather(1, index.long()))).sum(1)
    tol = 2.0 ** -24 * 300
    check(loss, ref.cpu(), tol * (10 + ref.abs()).cpu())
    check(lse, torch.logsumexp(z.double() / 1.5, 1).cpu(), torch.full((n,), tol * 20, dtype=torch.float64))
    size = q.exp().scatter_add(1, index.long(), lp.exp())
    grad = (weight.double() / 1.5)[:, None] * q.exp().scatter_add(1, index.long(), -lp.exp())
    bound = (weight.double() / 1.5)[:, None] * size * tol + 1e-38
    assert bool(((dz.double() - grad).abs() <= bound).all())


def test_oracle_words_equal_packed_codes(ctx):
    """The stream that a layer takes is that of pack_codes."""
    layer = Layer(20, 64, 6, 2, 0, torch.float32, seed=4)
    words = ctx.pack_codes(torch.from_numpy(layer.codes.astype(np.int32)).cuda(), 6)
    assert torch.equal(words.cpu(), layer.words) and np.array_equal(orc.unpack_codes(layer.words.numpy().view(np.uint32), 640, 6), layer.codes)


@pytest.mark.parametrize("rows,cols,k,d", [(65, 128, 2, 8), (81, 128, 2, 8), (97, 136, 2, 8), (113, 128, 2, 8), (65, 192, 2, 8), (129, 128, 3, 8), (129, 128, 2, 4)])
def test_last_rows_of_few_bits(ctx, rows, cols, k, d):
    """The last 16 rows of the layer are one row whose codes lie in the stream's last word, which a window of two words begins before."""
    for dtype in (torch.float32, torch.float16):
        layer = Layer(rows, cols, k, d, 0, dtype, seed=6)
        w = layer.weights()
        for n in (17, 40, 130):
            X = draw((n, cols), dtype, n)
            ref = X.double() @ w.t()
            check(ctx.codes_linear(layer.on_gpu(binding), X.cuda()), ref, HALF_STEP[dtype] * ref.abs() + sum_error(X.double().abs() @ w.abs().t(), cols))


def test_more_rows_of_logits_than_a_launch_takes(ctx):
    """2^26 + 5 rows of one wavefront each are more than 2^32 threads; single logits, and pairs."""
    n = 2 ** 26 + 5
    z = torch.arange(n * 2, device="cuda", dtype=torch.int32).remainder_(1009).to(torch.float16).mul_(2.0 ** -8).view(n, 2)
    index = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    teacher, weight = torch.zeros(n, 1, device="cuda"), torch.ones(n, device="cuda")
    loss, lse, dz = ctx.distill(z, index, teacher, 1.0, weight)
    for s in (slice(0, 1000), slice(2 ** 22 - 500, 2 ** 22 + 500), slice(n - 1000, n)):
        q = torch.log_softmax(z[s].double(), 1)
        check(loss[s], -q[:, 0].cpu(), torch.full((1000,), 1e-5, dtype=torch.float64))
        check(dz[s], (q.exp() - torch.tensor([1.0, 0.0], device="cuda", dtype=torch.float64)).cpu(), torch.full((1000, 2), 1e-3, dtype=torch.float64))
    assert bool(lse.isfinite().all()) and bool((dz.abs().sum(1) > 0).all())


def test_smallest_and_largest_temperatures(ctx):
    z, index, teacher = draw((3, 50), torch.float32, 1).cuda(), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, 1, device="cuda")
    for tau in (0.0, -1.0, 2.0 ** -127, float("inf"), float("nan")):
        with pytest.raises(binding.IdkmError):
            ctx.distill(z, index, teacher, tau)
    loss, _ = ctx.distill(z, index, teacher, 3e38)
    check(loss, torch.full((3,), 50.0, dtype=torch.float64).log(), torch.full((3,), 2e-6, dtype=torch.float64))
    z = torch.zeros(3, 50, device="cuda")
    loss, lse, dz = ctx.distill(z, index, teacher, 2.0 ** -126, torch.full((3,), 2.0 ** -126, device="cuda"))
    check(loss, torch.full((3,), 50.0, dtype=torch.float64).log(), torch.full((3,), 2e-6, dtype=torch.float64))
    check(dz[:, 1:], torch.full((3, 49), 0.02, dtype=torch.float64), torch.full((3, 49), 1e-8, dtype=torch.float64))


@pytest.mark.parametrize("rows,cols,group,n", [(2000, 96, 32, 5), (1500, 200, 64, 70), (96, 1000, 0, 6000), (700, 1100, 1100, 300), (108, 734, 64, 7)])
@pytest.mark.parametrize("k,d", [(16, 1), (100, 2)])
def test_gradients_whose_sums_are_long(ctx, rows, cols, group, n, k, d):
    """dX sums over many rows, the layer's own gradients over many tokens: parts of either, in one launch or in two."""
    from test_gpu_codes_linear import run_gradient
    for dtype in (torch.float32, torch.bfloat16):
        layer = Layer(rows, cols, k, d, group, dtype, seed=8)
        got = run_gradient(ctx, layer, n)
        again = ctx.codes_linear_backward(layer.on_gpu(binding), draw((n, cols), dtype, 1).cuda(), draw((n, rows), dtype, 2).cuda(), want_dC=False, want_dS=False)
        assert list(again) == ["dX"] and torch.equal(again["dX"], got["dX"])
