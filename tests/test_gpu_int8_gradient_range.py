"""The gradient through a layer of 8-bit integers whose scales lie anywhere in float32's range, not only where scale times integer is a normal
number of the type, and with dY that is no number."""
import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, check, draw, sum_error
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def integers(rows, cols):
    return torch.randint(-127, 128, (rows, cols), generator=torch.Generator().manual_seed(rows + cols), dtype=torch.int8)


def check_gradient(ctx, W8, scale, dY):
    layer = binding.Int8Layer(W8.cuda(), scale.cuda(), dY.dtype)
    w = W8.double() * scale.double()[:, None]
    ref, terms = dY.double() @ w, dY.double().abs() @ w.abs()
    half = HALF_STEP[dY.dtype]
    # the result's rounding and, relative to each term, one of a factor to the type; the sums of up to three parts
    bound = half * ref.abs() + (half + 2.0 ** -23) * terms + 2 * sum_error(terms, W8.shape[0])
    if dY.dtype == torch.float16:
        bound = bound + 2.0 ** -25  # half a step of subnormal results
    check(ctx.int8_linear_backward(layer, dY.cuda()), ref, bound)
    return ref


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,rows,cols", [(1, 300, 100), (65, 129, 200), (300, 512, 640)])
@pytest.mark.parametrize("power", [-30, -24, -20, -16, -10])
def test_small_layers(ctx, power, n, rows, cols, dtype):
    """Layers whose weights are small: results are numbers that the type holds in full."""
    scale = 2.0 ** power * (1 + torch.rand(rows, generator=torch.Generator().manual_seed(rows)))
    dY = (draw((n, rows), torch.float32, n).clamp(-3, 3) * 2.0 ** min(13, -power - 9)).to(DTYPES[dtype])
    ref = check_gradient(ctx, integers(rows, cols), scale, dY)
    assert 2.0 ** -14 < float(ref.abs().median()) < 2.0 ** 10


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_large_layers(ctx, dtype):
    """Weights beyond float16's largest number, gradients small enough for results that it holds."""
    scale = 2.0 ** 12 * (1 + torch.rand(200, generator=torch.Generator().manual_seed(1)))
    check_gradient(ctx, integers(200, 300), scale, (draw((40, 200), torch.float32, 1) * 2.0 ** -13).to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_rows_of_very_different_scales(ctx, dtype):
    """Only the rows of small scales have gradients for some tokens, rows of all scales for others."""
    rows = 256
    power = torch.arange(rows) % 48 - 36  # 2^-36 to 2^11
    scale = torch.ldexp(1 + torch.rand(rows, generator=torch.Generator().manual_seed(2)), power)
    dY = draw((80, rows), torch.float32, 3).clamp(-3, 3)
    dY[:40, power > -16] = 0
    dY[:40] *= 2.0 ** 12
    dY[40:] *= 2.0 ** -9
    check_gradient(ctx, integers(rows, 150), scale, dY.to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n", [2, 70, 300])
def test_gradients_that_are_no_numbers(ctx, n, dtype):
    """An infinity or NaN of dY goes to its own token's results and to no other's."""
    rows, cols = 130, 90
    W8 = integers(rows, cols)
    W8[7], W8[8] = 3, -5  # nowhere zero: infinity times zero would be NaN
    W8[7, 4] = 0
    scale = 0.01 * (1 + torch.rand(rows, generator=torch.Generator().manual_seed(4)))
    layer = binding.Int8Layer(W8.cuda(), scale.cuda(), DTYPES[dtype])
    dY = draw((n, rows), DTYPES[dtype], n)
    clean = ctx.int8_linear_backward(layer, dY.cuda()).cpu()
    for row, value, sign in ((7, float("inf"), 1), (8, float("inf"), -1), (7, float("-inf"), -1)):
        bad = dY.clone()
        bad[n - 1, row] = value
        got = ctx.int8_linear_backward(layer, bad.cuda()).cpu()
        assert torch.equal(got[: n - 1], clean[: n - 1])
        last = got[n - 1].double()
        held = torch.arange(cols) != 4 if row == 7 else torch.ones(cols, dtype=torch.bool)
        assert bool((last[held] == sign * float("inf")).all()) and (row != 7 or bool(last[4].isnan()))
    bad = dY.clone()
    bad[0, 9], bad[n - 1, 7], bad[n - 1, 8] = float("nan"), float("inf"), float("inf")  # of opposite signs in the sum
    got = ctx.int8_linear_backward(layer, bad.cuda()).cpu()
    assert bool(got[0].isnan().all()) and bool(got[n - 1].isnan().all()) and torch.equal(got[1: n - 1], clean[1: n - 1])


def test_nan_with_only_low_bits(ctx):
    """A NaN whose upper sixteen bits are those of an infinity stays one."""
    dY = torch.ones(3, 20, device="cuda")
    dY.view(torch.int32)[1, 5] = 0x7f800001
    dX = ctx.int8_linear_backward(binding.Int8Layer(torch.ones(20, 130, dtype=torch.int8, device="cuda"), torch.ones(20, device="cuda"), torch.float32), dY)
    assert bool(dX[1].isnan().all()) and bool((dX[[0, 2]] == 20).all())


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,rows,cols", [(5, 4097, 70), (3, 8200, 130), (2, 300_000, 520), (70_001, 40, 24)])
def test_long_layers_and_many_tokens(ctx, n, rows, cols, dtype):
    """More rows than a workgroup holds of a token, layers that are written out in panels of columns, tokens beyond 16 bits."""
    t = DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(rows)
    W8 = torch.randint(-127, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8)
    scale = torch.exp(torch.randn(rows, generator=g, device="cuda") - 5)
    dY = torch.randn(n, rows, generator=g, device="cuda").to(t)
    got = ctx.int8_linear_backward(binding.Int8Layer(W8, scale, t), dY)
    ref = torch.zeros(n, cols, dtype=torch.float64, device="cuda")
    terms = torch.zeros_like(ref)
    for r in range(0, rows, 50_000):
        w, y = W8[r:r + 50_000].double() * scale[r:r + 50_000].double()[:, None], dY[:, r:r + 50_000].double()
        ref += y @ w
        terms += y.abs() @ w.abs()
    half = HALF_STEP[t]
    bound = half * ref.abs() + (half + 2.0 ** -23) * terms + 2 * sum_error(terms, rows)
    check(got, ref.cpu(), (bound + (2.0 ** -25 if t == torch.float16 else 0.0)).cpu())
