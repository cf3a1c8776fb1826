"""Products with coded layers (idkm_codes_linear) and their gradients (idkm_codes_linear_backward) against float64."""
import numpy as np
import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, Layer, check, draw, sum_error
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def product_bound(layer, X, ref, dense):
    terms = X.double().abs() @ layer.weights().abs().t()
    bound = HALF_STEP[layer.dtype] * ref.abs() + sum_error(terms, layer.cols)
    if dense and layer.rounds_weights():
        bound = bound + HALF_STEP[layer.dtype] * terms
    if layer.dtype == torch.float16:
        bound = bound + 2.0 ** -25          # half a step of the subnormal results
        if dense and layer.rounds_weights():
            bound = bound + 2.0 ** -25 * X.double().abs().sum(1, keepdim=True)  # .. and of the subnormal weights
    return bound


def run_product(ctx, layer, X):
    ref = X.double() @ layer.weights().t()
    got = ctx.codes_linear(layer.on_gpu(binding), X.cuda())
    assert got.dtype == layer.dtype
    check(got, ref, product_bound(layer, X, ref, True))
    return got


CODEBOOKS = [(1, 1), (2, 1), (3, 1), (4, 1), (8, 1), (16, 1), (32, 1), (64, 1), (100, 1), (256, 1), (512, 1), (2, 2), (16, 2), (64, 2),
             (3, 4), (16, 4), (256, 4), (2, 8), (16, 8), (100, 8), (256, 8), (1024, 2), (5, 3), (7, 16), (9, 64)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("k,d", CODEBOOKS)
def test_product_every_codebook(ctx, k, d, dtype):
    """Rows that begin inside words and rows that begin with one, whole and broken chunks, with and without scales, for one
    token, a few and more than the direct form takes."""
    for cols, group in [(192 * d if d > 8 else 768, 0), (576, 64), (37 * d, 0), (133 * d, 37 * d * 4)]:
        if cols % d or (group and group < cols and (group % 32 or group % d)):
            continue
        layer = Layer(37, cols, k, d, group, DTYPES[dtype], seed=k)
        for n in (1, 5, 70):
            run_product(ctx, layer, draw((n, cols), DTYPES[dtype], n))


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 64, 65, 129, 300])
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 0), (16, 128, 128), (17, 129, 128), (1000, 512, 96), (250, 2304, 32), (513, 1000, 64),
                                             (100, 4608, 4608)])
def test_product_sizes(ctx, rows, cols, group, n):
    for dtype in (torch.bfloat16, torch.float32):
        run_product(ctx, Layer(rows, cols, 16, 1, group, dtype, seed=1), draw((n, cols), dtype, n))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_few_tokens_round_only_the_result(ctx, dtype):
    """The direct form keeps codewords and scales apart: nothing but the result is rounded."""
    layer = Layer(48, 1024, 16, 1, 128, DTYPES[dtype], seed=3)
    for n in (1, 7, 64):
        X = draw((n, 1024), DTYPES[dtype], n)
        ref = X.double() @ layer.weights().t()
        check(ctx.codes_linear(layer.on_gpu(binding), X.cuda()), ref, product_bound(layer, X, ref, False))


@pytest.mark.parametrize("n", [3, 40, 200])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_strides_and_neighbours(ctx, n, dtype):
    """Rows of X and Y that lie apart and begin anywhere; what lies between them stays as it was."""
    t = DTYPES[dtype]
    layer = Layer(77, 300, 16, 1, 0, t, seed=4)
    wide = draw((n, 320), t, n)
    out = torch.full((n + 1, 91), 7.0, dtype=t, device="cuda")
    X = wide[:, 3:303]
    res = ctx.codes_linear(layer.on_gpu(binding), wide.cuda()[:, 3:303], out=out[:n, 5:82])
    ref = X.double() @ layer.weights().t()
    check(res, ref, product_bound(layer, X, ref, True))
    assert bool((out[n] == 7).all()) and bool((out[:, :5] == 7).all()) and bool((out[:, 82:] == 7).all())


@pytest.mark.parametrize("n", [1, 30, 100])
def test_codes_that_are_none_and_weights_that_are_no_numbers(ctx, n):
    """A code >= k makes its row's outputs NaN and no others; infinities and NaN stay in the rows and tokens they belong to."""
    layer = Layer(40, 70, 3, 1, 0, torch.float32, seed=5)
    layer.codes[11 * 70 + 69] = 3
    from oracle import idkm_oracle as orc
    layer.words = torch.from_numpy(orc.pack_codes(layer.codes, 4).view(np.int32))
    X = draw((n, 70), torch.float32, n)
    got = ctx.codes_linear(layer.on_gpu(binding), X.cuda()).cpu()
    assert bool(got[:, 11].isnan().all())
    rest = [r for r in range(40) if r != 11]
    assert bool(got[:, rest].isfinite().all())
    X[n // 2, 5] = float("nan")
    got = ctx.codes_linear(layer.on_gpu(binding), X.cuda()).cpu()
    assert bool(got[n // 2].isnan().all())
    assert bool(got[[t for t in range(n) if t != n // 2]][:, rest].isfinite().all())


def test_no_tokens(ctx):
    layer = Layer(8, 64, 4, 1, 32, torch.float32)
    g = layer.on_gpu(binding)
    assert ctx.codes_linear(g, torch.empty(0, 64, device="cuda")).shape == (0, 8)
    r = ctx.codes_linear_backward(g, torch.empty(0, 64, device="cuda"), torch.empty(0, 8, device="cuda"))
    assert r["dX"].shape == (0, 64) and not r["dC"].any() and not r["dS"].any()


def run_gradient(ctx, layer, n, seed=0):
    X, dY = draw((n, layer.cols), layer.dtype, seed + 1), draw((n, layer.rows), layer.dtype, seed + 2)
    got = ctx.codes_linear_backward(layer.on_gpu(binding), X.cuda(), dY.cuda())
    w, u, s = layer.weights(), layer.unscaled(), layer.scales()
    x, y = X.double(), dY.double()
    ref = y @ w
    terms = y.abs() @ w.abs()
    bound = HALF_STEP[layer.dtype] * ref.abs() + sum_error(terms, layer.rows)
    if layer.rounds_weights():
        bound = bound + HALF_STEP[layer.dtype] * terms
    if layer.dtype == torch.float16:
        bound = bound + 2.0 ** -25 + 2.0 ** -25 * y.abs().sum(1, keepdim=True)
    check(got["dX"], ref, bound, "dX")
    P, Pa = y.t() @ x, y.abs().t() @ x.abs()
    codes = torch.from_numpy(layer.codes)
    parts = lambda v: torch.zeros(layer.k, layer.d, dtype=torch.float64).index_add_(0, codes, v.reshape(-1, layer.d))  # noqa: E731
    many = n + layer.rows * layer.cols // layer.k
    check(got["dC"], parts(P * s), sum_error(parts(Pa * s), many) + 2.0 ** -24 * parts(P * s).abs(), "dC")
    if layer.S is not None:
        group = min(layer.group, layer.cols)
        by_group = lambda v: torch.stack([v[:, c:c + group].sum(1) for c in range(0, layer.cols, group)], 1)  # noqa: E731
        check(got["dS"], by_group(P * u), sum_error(by_group(Pa * u.abs()), n + group), "dS")
    else:
        assert "dS" not in got
    return got


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("k,d", CODEBOOKS)
def test_gradient_every_codebook(ctx, k, d, dtype):
    for cols, group in [(192 * d if d > 8 else 384, 0), (576, 64), (133 * d, 37 * d * 4)]:
        if cols % d or (group and group < cols and (group % 32 or group % d)):
            continue
        run_gradient(ctx, Layer(37, cols, k, d, group, DTYPES[dtype], seed=k), 19)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 257, 1001])
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 0), (17, 129, 128), (200, 512, 96), (70, 1000, 32), (64, 2304, 2304)])
def test_gradient_sizes(ctx, rows, cols, group, n):
    for dtype in (torch.bfloat16, torch.float32):
        run_gradient(ctx, Layer(rows, cols, 16, 1, group, dtype, seed=2), n)


def test_gradient_of_each_part_alone_and_bit_for_bit_again(ctx):
    layer = Layer(130, 640, 16, 1, 64, torch.bfloat16, seed=7)
    g = layer.on_gpu(binding)
    X, dY = draw((90, 640), torch.bfloat16, 1).cuda(), draw((90, 130), torch.bfloat16, 2).cuda()
    ref = ctx.codes_linear_backward(g, X, dY)
    for want in ("dX", "dC", "dS"):
        r = ctx.codes_linear_backward(g, X if want != "dX" else None, dY, want_dX=want == "dX", want_dC=want == "dC", want_dS=want == "dS")
        assert list(r) == [want] and torch.equal(r[want], ref[want])
    again = ctx.codes_linear_backward(g, X, dY)
    assert all(torch.equal(again[key], ref[key]) for key in ref)


def test_gradient_against_differences(ctx):
    """d/de of sum(G * Y(C + e D, S + e E, X + e F)) from two products in float32 whose exact difference the gradients give."""
    layer = Layer(60, 384, 16, 1, 128, torch.float32, seed=8)
    n = 33
    X, G = draw((n, 384), torch.float32, 1), draw((n, 60), torch.float32, 2)
    D, E, F = draw((16, 1), torch.float32, 3), draw((60, 3), torch.float32, 4), draw((n, 384), torch.float32, 5)
    r = ctx.codes_linear_backward(layer.on_gpu(binding), X.cuda(), G.cuda())
    slope = sum(float((r[key].double().cpu() * v.double()).sum()) for key, v in (("dC", D), ("dS", E), ("dX", F)))
    e = 2.0 ** -6
    base_C, base_S = layer.C, layer.S
    value = []
    for sign in (1, -1):
        layer.C, layer.S = base_C + sign * e * D, base_S + sign * e * E
        Y = ctx.codes_linear(layer.on_gpu(binding), (X + sign * e * F).cuda())
        value.append(float((Y.double().cpu() * G.double()).sum()))
    # the product is cubic in e: the central difference is off by e^2 times the third-order term
    codes = torch.from_numpy(layer.codes)
    cubic = float((((F.double()) @ (D.double()[codes].reshape(60, 384) * E.double().repeat_interleave(128, 1)).t()) * G.double()).sum())
    rough = 2.0 ** -24 * 60 * float((X.abs().double() @ layer.weights().abs().t() * G.abs().double()).sum()) / e
    assert abs((value[0] - value[1]) / (2 * e) - e * e * cubic - slope) < rough


@pytest.mark.parametrize("n", [1, 40, 300])
def test_other_streams_and_captured_graphs(ctx, n):
    """A call on a side stream, and a captured one replayed beside eager work on changed inputs."""
    layer = Layer(96, 512, 16, 1, 128, torch.bfloat16, seed=9)
    g = layer.on_gpu(binding)
    X, dY = draw((n, 512), torch.bfloat16, 1).cuda(), draw((n, 96), torch.bfloat16, 2).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Y1 = ctx.codes_linear(g, X)
        r1 = ctx.codes_linear_backward(g, X, dY)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y1, ctx.codes_linear(g, X))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y2 = ctx.codes_linear(g, X)
        r2 = ctx.codes_linear_backward(g, X, dY)
    for i in range(3):
        X.copy_(draw((n, 512), torch.bfloat16, 10 + i).cuda())
        dY.copy_(draw((n, 96), torch.bfloat16, 20 + i).cuda())
        graph.replay()
        Y3, r3 = ctx.codes_linear(g, X), ctx.codes_linear_backward(g, X, dY)
        torch.cuda.synchronize()
        assert torch.equal(Y2, Y3) and all(torch.equal(r2[key], r3[key]) for key in r3)
    assert r1["dX"].shape == (n, 512)


def test_refusals(ctx):
    layer = Layer(16, 64, 16, 1, 32, torch.float32)
    words, Cb, S = layer.words.cuda(), layer.C.cuda(), layer.S.cuda()
    make = binding.CodesLayer
    for bad in (lambda: make(words, 16, 63, Cb.reshape(8, 2), None, 0), lambda: make(words, 16, 64, Cb, S, 0),
                lambda: make(words, 16, 64, Cb, S, 33), lambda: make(words, 0, 64, Cb)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: make(words[:-1], 16, 64, Cb), lambda: make(words, 16, 64, Cb.double()), lambda: make(words, 16, 64, Cb, S.half(), 32),
                lambda: make(words.cpu(), 16, 64, Cb)):
        with pytest.raises(TypeError):
            bad()
    g = make(words, 16, 64, Cb, S, 32)
    X = torch.zeros(2, 64, device="cuda")
    for bad in (X.half(), X[:, :63], X.cpu(), torch.zeros(64, 2, device="cuda").t(), torch.zeros(64, device="cuda")):
        with pytest.raises(TypeError):
            ctx.codes_linear(g, bad)
    with pytest.raises(TypeError):
        ctx.codes_linear(g, X, out=torch.zeros(3, 16, device="cuda"))
    with pytest.raises(TypeError):
        ctx.codes_linear_backward(g, None, torch.zeros(2, 16, device="cuda"))
    lib = ctx._lib
    n = 4000
    many, Y = torch.zeros(n, 64, device="cuda"), torch.zeros(n, 16, device="cuda")
    call = lambda ws, size: lib.idkm_codes_linear(ctx._h, g._at, many.data_ptr(), n, 64, Y.data_ptr(), 16, ws, size, None)  # noqa: E731
    need = lib.idkm_codes_linear_workspace(g._at, n)
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    assert need > 0 and call(None, need) == 1 and call(ws.data_ptr(), need - 1) == 1 and call(ws.data_ptr() + 4, need) == 1
    assert b"workspace" in lib.idkm_last_error(ctx._h)
    assert call(ws.data_ptr(), need) == 0
