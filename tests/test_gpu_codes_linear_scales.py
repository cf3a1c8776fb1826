"""Products of layers with group scales that are written out for the matrix cores: codewords and scales stay apart there, too, so that
nothing but the result is rounded, whatever the number of tokens."""
import numpy as np
import pytest
import torch

from layer_cases import DTYPES, Layer, check, draw
from paper_2312_07759_amd import binding
from test_gpu_codes_linear import ctx, product_bound  # noqa: F401

pytestmark = pytest.mark.gpu


def run(ctx, layer, X, rows=None):  # noqa: F811
    got = ctx.codes_linear(layer.on_gpu(binding), X.cuda())
    ref = X.double() @ layer.weights().t()
    check(got, ref, product_bound(layer, X, ref, False))
    return got


# codebooks without a direct form are written out for any number of tokens
@pytest.mark.parametrize("n", [1, 5, 64, 65, 129, 300])
@pytest.mark.parametrize("rows,cols,group", [(1, 33, 32), (17, 64, 32), (37, 96, 32), (65, 99, 96), (64, 160, 64), (130, 1000, 128), (129, 1001, 160), (40, 321, 288),
                                             (70, 512, 512), (70, 510, 600), (3, 2000, 1024), (257, 70, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_codebooks_that_are_always_written_out(ctx, rows, cols, group, n, dtype):  # noqa: F811
    run(ctx, Layer(rows, cols, 300, 1, group, DTYPES[dtype], seed=1), draw((n, cols), DTYPES[dtype], n))


@pytest.mark.parametrize("k,d,group", [(5, 3, 96), (7, 16, 32), (9, 64, 64), (1024, 2, 128), (300, 4, 32)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_longer_codewords(ctx, k, d, group, dtype):  # noqa: F811
    for n in (2, 200):
        run(ctx, Layer(50, 11 * 192, k, d, group, DTYPES[dtype], seed=2), draw((n, 11 * 192), DTYPES[dtype], n))


@pytest.mark.parametrize("group", [32, 64, 96, 128, 640, 1920])
@pytest.mark.parametrize("k,d", [(16, 1), (8, 1), (256, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_tokens(ctx, k, d, group, dtype):  # noqa: F811
    """Tiles of every shape, sums in parts, rows that are not a multiple of a tile."""
    for n, rows in ((2100, 520), (1500, 100), (5000, 33)):
        run(ctx, Layer(rows, 1920, k, d, group, DTYPES[dtype], seed=3), draw((n, 1920), DTYPES[dtype], n))


@pytest.mark.parametrize("n", [1, 40, 200, 2000])
@pytest.mark.parametrize("k", [16, 300])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("scale,size", [(2.0 ** 18, 2.0 ** -12), (2.0 ** -20, 2.0 ** 12)])
def test_scales_beyond_the_range_of_float16(ctx, scale, size, group, k, n):  # noqa: F811
    """S C is beyond 65504, or below what float16 holds; the products are not."""
    layer = Layer(150, 640, k, 1, group, torch.float16, seed=4)
    layer.S = layer.S.clamp(max=4.0) * scale
    run(ctx, layer, (draw((n, 640), torch.float32, n) * size).to(torch.float16))


@pytest.mark.parametrize("n", [1, 70, 600, 2500])
@pytest.mark.parametrize("k", [16, 300])
@pytest.mark.parametrize("cols,group", [(96, 32), (80, 32), (80, 64), (352, 96), (1024, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales_that_are_no_numbers(ctx, cols, group, k, n, dtype):  # noqa: F811
    """An infinite scale stands for weights of plus and minus infinity, whose sum is none; it and NaN leave nothing finite in their row, zero
    leaves the group out, and other rows stay as they are."""
    layer = Layer(70, cols, k, 1, group, DTYPES[dtype], seed=5)
    X = draw((n, cols), DTYPES[dtype], n)
    plain = run(ctx, layer, X).cpu()
    layer.S[3, -1], layer.S[20, -1], layer.S[69, 0] = float("inf"), float("nan"), 0.0
    got = ctx.codes_linear(layer.on_gpu(binding), X.cuda()).cpu()
    assert not bool(got[:, 3].isfinite().any()) and bool(got[:, 20].isnan().all())
    rest = [r for r in range(70) if r not in (3, 20, 69)]
    assert bool(torch.equal(got[:, rest], plain[:, rest]))
    ref = X.double() @ layer.weights()[69:].t()
    terms = X.double().abs() @ layer.weights()[69:].abs().t()
    assert bool(((got[:, 69:].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -16 * terms + 2.0 ** -24).all())


def test_panels(ctx):  # noqa: F811
    """A layer written out in several panels takes its scales from the panel's rows on."""
    from test_gpu_codes_linear_edges import big_layer
    rows, cols, n = 34_000, 2_048, 300
    for group in (96, 128):
        layer, weights = big_layer(rows, cols, 16, group, torch.bfloat16)
        X = draw((n, cols), torch.bfloat16, 1).cuda()
        Y = ctx.codes_linear(layer, X)
        for r0 in (0, 32_700, rows - 100):
            w = weights(r0, r0 + 100)
            ref, terms = X.double() @ w.t(), X.double().abs() @ w.abs().t()
            check(Y[:, r0:r0 + 100], ref.cpu(), (2.0 ** -8 * ref.abs() + (4 * cols ** 0.5 + 4) * 2.0 ** -24 * terms).cpu())


def test_a_captured_call(ctx):  # noqa: F811
    layer = Layer(300, 960, 16, 1, 96, torch.bfloat16, seed=6).on_gpu(binding)
    X = draw((2300, 960), torch.bfloat16, 1).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = ctx.codes_linear(layer, X)
    for i in range(3):
        X.copy_(draw((2300, 960), torch.bfloat16, 2 + i).cuda())
        layer.S.copy_(torch.from_numpy(np.random.default_rng(i).random(tuple(layer.S.shape)).astype(np.float32)).cuda())
        graph.replay()
        ref = ctx.codes_linear(layer, X)
        torch.cuda.synchronize()
        assert bool(torch.equal(Y, ref))
