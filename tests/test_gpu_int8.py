"""Products in 8-bit integers with a scale for each token and each row of the layer, and their gradient, against float64."""
from fractions import Fraction

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


def integers(X):
    """Rows in integers and their scales.  The quotient of two float32 numbers that lies beside a tie differs from it by more than 2^-52 of its
    size (numerator and denominator have 24 bits each), so float64 keeps it on its side; ties are exact."""
    x = X.float().numpy()
    with np.errstate(all="ignore"):
        s = np.maximum(np.abs(x).max(1) / np.float32(127), np.float32(2.0 ** -126))
        q = np.rint(x.astype(np.float64) / s.astype(np.float64)[:, None])
    none = ~np.isfinite(x).all(1)
    s[none], q[none] = np.nan, 0
    return torch.from_numpy(q), torch.from_numpy(s)


def layer_of(rows, cols, dtype, seed=0):
    rng = np.random.default_rng([rows, cols, seed])
    W8 = torch.from_numpy(rng.integers(-127, 128, size=(rows, cols)).astype(np.int8))
    scale = torch.from_numpy(np.exp(rng.standard_normal(rows) - 5).astype(np.float32))
    return W8, scale, binding.Int8Layer(W8.cuda(), scale.cuda(), dtype)


def check_product(got, X, W8, scale):
    q, s = integers(X)
    assert got.dtype == X.dtype
    ref = (q @ W8.double().t()) * s.double()[:, None] * scale.double()
    # the sum to float32, two products, and the result's own rounding; subnormal results of float16 by half a step
    check(got, ref, (HALF_STEP[X.dtype] + 3 * 2.0 ** -24) * ref.abs() + (2.0 ** -25 if X.dtype == torch.float16 else 0.0))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,cols", [(1, 1), (2, 7), (5, 128), (3, 1000), (2, 8192), (2, 8193), (1, 20001)])
def test_rows(ctx, n, cols, dtype):
    X = draw((n, cols), DTYPES[dtype], cols) * 3
    Q, s = ctx.int8_rows(X.cuda())
    q, t = integers(X)
    assert torch.equal(Q.cpu().double(), q) and torch.equal(s.cpu(), t)


def test_rows_at_ties_and_beside_them(ctx):
    """Quotients at and next to halves, for scales whose inverse is rounded up and down: against rational arithmetic."""
    rows = []
    for top in (127.0, 126.999, 1.0, 3.3333333, 1e-30, 2.0 ** -120, 1e30, 254.0, 255.9, 2.0 ** -126 * 3, 2.0 ** -140):
        top = np.float32(top)
        s = np.maximum(top / np.float32(127), np.float32(2.0 ** -126))
        row = [top, -top]
        for k in range(-126, 127):
            x = np.float32(np.float64(s) * (k + 0.5))
            for y in (x, np.nextafter(x, np.float32(np.inf)), np.nextafter(x, np.float32(-np.inf))):
                row.append(y if abs(y) <= top else np.float32(0))
        rows.append(row)
    X = torch.from_numpy(np.array(rows, dtype=np.float32))
    Q, s = ctx.int8_rows(X.cuda())
    s, Q = s.cpu().numpy(), Q.cpu().numpy()
    for t in range(len(rows)):
        assert s[t] == np.maximum(np.float32(np.abs(X[t].numpy()).max()) / np.float32(127), np.float32(2.0 ** -126))
        for c, x in enumerate(X[t].tolist()):
            assert Q[t, c] == round(Fraction(x) / Fraction(float(s[t]))), (t, c)  # Python's round of a fraction: ties to even


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 128), (17, 129), (100, 64), (250, 1000), (512, 4608), (130, 8200)])
@pytest.mark.parametrize("n", [1, 2, 4, 5, 15, 16, 17, 33, 64, 65, 200])
def test_product(ctx, n, rows, cols, dtype):
    W8, scale, layer = layer_of(rows, cols, DTYPES[dtype])
    X = draw((n, cols), DTYPES[dtype], n)
    check_product(ctx.int8_linear(layer, X.cuda()), X, W8, scale)


@pytest.mark.parametrize("n,rows,cols", [(1000, 1024, 1024), (2049, 513, 300), (300, 4096, 512), (129, 2000, 4096), (4100, 260, 130)])
def test_product_of_many_tokens(ctx, n, rows, cols):
    W8, scale, layer = layer_of(rows, cols, torch.bfloat16)
    X = draw((n, cols), torch.bfloat16, n)
    check_product(ctx.int8_linear(layer, X.cuda()), X, W8, scale)


def test_the_largest_sums(ctx):
    """All integers at their ends, the longest rows: the sums come near 2^31 and stay exact."""
    W8 = torch.full((20, 131072), 127, dtype=torch.int8)
    W8[1] = -127
    X = torch.ones(70, 131072)
    X[3] = -1
    layer = binding.Int8Layer(W8.cuda(), torch.ones(20, device="cuda"), torch.float32)
    for n in (1, 40, 70):
        check_product(ctx.int8_linear(layer, X[:n].cuda()), X[:n], W8, torch.ones(20))
    with pytest.raises(ValueError):
        binding.Int8Layer(torch.zeros(2, 131073, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda"), torch.float32)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n", [1, 9, 40, 150])
def test_rows_of_zeros_and_of_no_numbers(ctx, n, dtype):
    W8, scale, layer = layer_of(33, 200, DTYPES[dtype])
    X = draw((n, 200), DTYPES[dtype], 1)
    X[n // 2] = 0
    got = ctx.int8_linear(layer, X.cuda())
    check_product(got, X, W8, scale)
    assert not got[n // 2].any()
    X[n - 1, 199] = float("nan")
    X[0, 3] = float("inf")
    got = ctx.int8_linear(layer, X.cuda()).cpu()
    held = torch.ones(n, dtype=torch.bool)
    held[0] = held[n - 1] = False
    assert bool(got[~held].isnan().all()) and bool(got[held].isfinite().all())
    bad = scale.clone()
    bad[5] = float("nan")
    got = ctx.int8_linear(binding.Int8Layer(W8.cuda(), bad.cuda(), DTYPES[dtype]), X.cuda()).cpu()
    assert bool(got[:, 5].isnan().all()) and bool(got[held][:, 6:].isfinite().all())


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n", [3, 30, 100])
def test_strides_and_neighbours(ctx, n, dtype):
    t = DTYPES[dtype]
    W8, scale, layer = layer_of(77, 300, t)
    wide, out = draw((n, 320), t, n), torch.full((n + 1, 91), 7.0, dtype=t, device="cuda")
    check_product(ctx.int8_linear(layer, wide.cuda()[:, 3:303], out=out[:n, 5:82]), wide[:, 3:303], W8, scale)
    assert bool((out[n] == 7).all()) and bool((out[:, :5] == 7).all()) and bool((out[:, 82:] == 7).all())
    dY = draw((n, 90), t, n).cuda()
    assert torch.equal(ctx.int8_linear_backward(layer, dY[:, 3:80]), ctx.int8_linear_backward(layer, dY[:, 3:80].contiguous()))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (1, 100, 300), (40, 129, 77), (300, 512, 1000), (1001, 1000, 512)])
def test_gradient(ctx, n, rows, cols, dtype):
    W8, scale, layer = layer_of(rows, cols, DTYPES[dtype])
    dY = draw((n, rows), DTYPES[dtype], n)
    w = W8.double() * scale.double()[:, None]
    ref, terms = dY.double() @ w, dY.double().abs() @ w.abs()
    half = HALF_STEP[DTYPES[dtype]]
    bound = half * ref.abs() + half * terms + sum_error(terms, rows)  # the result's rounding, the weights'
    if dtype == "f16":
        bound = bound + 2.0 ** -25 * (1 + dY.double().abs().sum(1, keepdim=True))  # subnormal results and weights
    check(ctx.int8_linear_backward(layer, dY.cuda()), ref, bound)


@pytest.mark.parametrize("k,d,group", [(16, 1, 64), (256, 4, 0), (100, 2, 640), (512, 5, 0)])
def test_layers_of_weights_and_of_stored_layers(ctx, k, d, group):
    stored = Layer(90, 640, k, d, group, torch.bfloat16, seed=k)
    layer = ctx.int8_layer(stored.on_gpu(binding))
    assert layer.dtype == torch.bfloat16 and (layer.rows, layer.cols) == (90, 640)
    q, s = integers((stored.unscaled().float() * stored.scales().float()))
    assert torch.equal(layer.W8[:, :640].cpu().double(), q) and torch.equal(layer.scale.cpu(), s)
    W = draw((40, 333), torch.float32, 1)
    layer = ctx.int8_layer(W.cuda(), torch.float16)
    q, s = integers(W)
    assert torch.equal(layer.W8[:, :333].cpu().double(), q) and torch.equal(layer.scale.cpu(), s)
    X = draw((20, 333), torch.float16, 2)
    check_product(ctx.int8_linear(layer, X.cuda()), X, q, s)


def test_none_and_refusals(ctx):
    W8, scale, layer = layer_of(8, 64, torch.bfloat16)
    assert ctx.int8_linear(layer, torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")).shape == (0, 8)
    assert ctx.int8_linear_backward(layer, torch.empty(0, 8, dtype=torch.bfloat16, device="cuda")).shape == (0, 64)
    assert ctx.int8_rows(torch.empty(0, 64, device="cuda"))[0].shape == (0, 64)
    X = torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (X.float(), X[:, :63], X.cpu(), X.t()):
        with pytest.raises(TypeError):
            ctx.int8_linear(layer, bad)
    with pytest.raises(TypeError):
        ctx.int8_linear_backward(layer, X)
    with pytest.raises(TypeError):
        ctx.int8_linear(layer, X, out=torch.empty(4, 8, dtype=torch.bfloat16, device="cuda"))
    for W, s, t in ((W8.cuda().int(), scale.cuda(), torch.float32), (W8.cuda(), scale.cuda()[:7], torch.float32), (W8.cuda(), scale.cuda().double(), torch.float32),
                    (W8.cuda(), scale.cuda(), torch.int8), (W8.cuda().t(), scale.cuda(), torch.float32), (W8, scale, torch.float32)):
        with pytest.raises(TypeError):
            binding.Int8Layer(W, s, t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows,cols", [(1, 40, 512), (3, 40, 512), (20, 40, 700), (300, 200, 512), (70, 64, 8192)])
def test_tokens_near_the_largest_number(ctx, n, rows, cols, dtype):
    """A sum times the token's scale has no float32 number here, the result has one."""
    X = (draw((n, cols), torch.float32, 1).clamp(-3, 3) * 1e38).to(DTYPES[dtype])
    W8, scale, _ = layer_of(rows, cols, X.dtype, 2)
    scale *= 1e-8
    got = ctx.int8_linear(binding.Int8Layer(W8.cuda(), scale.cuda(), X.dtype), X.cuda())
    assert bool(got.isfinite().all()) and float(got.abs().max()) > 1e30
    check_product(got.cpu(), X, W8, scale)


@pytest.mark.parametrize("n,cols", [(3, 10_900), (3, 10_880), (2, 16_384), (2, 16_300), (1, 32_700), (4, 8192), (4, 8100), (1, 32_769)])
def test_as_many_columns_as_a_workgroup_holds(ctx, n, cols):
    """Tokens brought to integers by the product's own workgroups, up to the last column that fits, and by a launch before it."""
    X = draw((n, cols), torch.bfloat16, 1)
    W8, scale, layer = layer_of(20, cols, torch.bfloat16, 3)
    check_product(ctx.int8_linear(layer, X.cuda()).cpu(), X, W8, scale)
