"""Lookups of tokens' rows in stored and float32 tables and their gradients, against float64."""
import numpy as np
import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, Layer, check, draw, sum_error
from oracle import idkm_oracle as orc
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu
ALPHA = 1.375  # a float32 number


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def tokens(kind, n, rows, seed=0):
    rng = np.random.default_rng([seed, n, rows])
    ids = rng.integers(0, rows, size=n)
    if kind == "text":  # a few rows hold most tokens; some padding, some ids of no row
        ids = np.minimum((rows + 1.0) ** rng.random(n) - 1, rows - 1).astype(np.int64)
        ids[rng.random(n) < 0.1] = -1
        ids[rng.random(n) < 0.02] = rows + 3
    elif kind == "one":
        ids[:] = rows - 1
    elif kind == "none":
        ids[:] = -1
    elif kind == "runs":  # already in order, and a row's tokens one after another
        ids = np.sort(ids) // 2
    return torch.from_numpy(ids.astype(np.int64))


def by_row(ids, dY, rows):
    """P and the sums of the terms' sizes, float64, and the longest sum."""
    held = (ids >= 0) & (ids < rows)
    P = torch.zeros(rows, dY.shape[1], dtype=torch.float64)
    P.index_put_((ids[held],), dY[held].double() * ALPHA, accumulate=True)
    A = torch.zeros_like(P)
    A.index_put_((ids[held],), dY[held].double().abs() * ALPHA, accumulate=True)
    return P, A, int(torch.bincount(ids[held], minlength=1).max()) if bool(held.any()) else 0


def error(terms, length):
    """A sum's error, and up to four roundings of factors (alpha, a scale, a codeword's product, a part's)."""
    return sum_error(terms, max(length, 1)) + 4 * 2.0 ** -24 * terms


def check_lookup(got, W, ids, dtype):
    rows = W.shape[0]
    held = (ids >= 0) & (ids < rows)
    ref = W[ids.clamp(0, rows - 1)] * ALPHA
    ref[~held] = 0
    nan = ids >= rows
    assert got.dtype == dtype and bool(got[nan.cuda()].isnan().all())
    got = got.clone()
    got[nan.cuda()] = 0
    # three factors at most and their rounding to the type, subnormal results of float16 by half a step
    check(got, ref, (HALF_STEP[dtype] + 3 * 2.0 ** -24) * ref.abs() + (2.0 ** -25 if dtype == torch.float16 else 0.0))


def run_codes(ctx, layer, ids, seed=0, wide=True):
    n = len(ids)
    handle, at = layer.on_gpu(binding), (ids if wide else ids.int()).cuda()
    check_lookup(ctx.codes_embedding(handle, at, ALPHA), layer.weights(), ids, layer.dtype)
    dY = draw((n, layer.cols), layer.dtype, seed + 1)
    got = ctx.codes_embedding_backward(handle, at, dY.cuda(), ALPHA)
    P, A, most = by_row(ids, dY, layer.rows)
    SP, SA = P * layer.scales(), A * layer.scales()
    codes = torch.from_numpy(layer.codes)
    sums = lambda v: torch.zeros(layer.k, layer.d, dtype=torch.float64).index_add_(0, codes, v.reshape(-1, layer.d))  # noqa: E731
    check(got["dC"], sums(SP), error(sums(SA), n * layer.cols // layer.d), "dC")
    if layer.S is not None:
        u, g = layer.unscaled(), min(layer.group, layer.cols)
        per = lambda v: torch.stack([v[:, c:c + g].sum(1) for c in range(0, layer.cols, g)], 1)  # noqa: E731
        check(got["dS"], per(P * u), error(per(A * u.abs()), most * g), "dS")
    else:
        assert "dS" not in got
    return got


CODEBOOKS = [(1, 1), (2, 1), (3, 1), (8, 1), (16, 1), (64, 1), (100, 1), (256, 1), (512, 1), (2, 2), (16, 2), (100, 2), (3, 4), (16, 4), (64, 4),
             (256, 4), (2, 8), (16, 8), (256, 8), (1024, 2), (5, 3), (7, 16), (9, 64)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("k,d", CODEBOOKS)
def test_stored_every_codebook(ctx, k, d, dtype):
    """Rows that begin inside words, whole and broken groups, one scale a row, none; ids of no row among the tokens."""
    for cols, group in [(192 * d if d > 8 else 768, 0), (576, 64), (640, 128), (37 * d, 0), (133 * d, 37 * d * 4)]:
        if cols % d or (group and group < cols and (group % 32 or group % d)):
            continue
        layer = Layer(53, cols, k, d, group, DTYPES[dtype], seed=k)
        for n in (1, 90):
            run_codes(ctx, layer, tokens("text", n, 53, n), n, wide=n > 1)


@pytest.mark.parametrize("kind", ["any", "text", "one", "none", "runs"])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 64, 65, 300, 1025])
def test_stored_orders_of_tokens(ctx, n, kind):
    for rows, cols, k, d, group, dtype in [(200, 256, 16, 1, 32, torch.bfloat16), (40, 72, 256, 4, 72, torch.float32), (1, 8, 2, 1, 0, torch.float16)]:
        run_codes(ctx, Layer(rows, cols, k, d, group, dtype, seed=n), tokens(kind, n, rows, 3), n)


@pytest.mark.parametrize("kind", ["any", "text", "one"])
@pytest.mark.parametrize("n", [4096, 16384, 16385, 40000])
def test_stored_many_tokens(ctx, n, kind):
    """Both forms of the sort, rows whose tokens lie in many parts."""
    run_codes(ctx, Layer(700, 64, 16, 1, 32, torch.bfloat16, seed=n), tokens(kind, n, 700, 3), n)


@pytest.mark.parametrize("n,cols,k,d", [(17000, 16, 256, 8), (6000, 1496, 256, 8), (16384, 16, 256, 8), (3000, 1032, 256, 4), (3000, 1032, 100, 8), (2000, 520, 64, 1),
                                        (2000, 520, 65, 1), (2000, 520, 100, 4), (2000, 520, 256, 2), (450, 1030, 100, 2), (513, 1032, 256, 8), (700, 9, 129, 1)])
def test_stored_codebooks_of_many_tokens(ctx, n, cols, k, d):
    """Bins of a lane's own, of two to sixteen lanes in turn, and sums written out, on both sides of where they change."""
    for group, dtype, kind in ((0, torch.float32, "text"), (32, torch.bfloat16, "runs"), (cols, torch.float16, "any")):
        run_codes(ctx, Layer(500, cols, k, d, group, dtype, seed=n), tokens(kind, n, 500, 4), n)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (50, 7), (300, 512), (333, 1001), (70000, 24)])
@pytest.mark.parametrize("n", [1, 33, 700, 20000])
def test_table(ctx, rows, cols, n, dtype):
    """The float32 table; 70000 rows take three passes of the sort."""
    t = DTYPES[dtype]
    W, ids, dY = draw((rows, cols), torch.float32, 1), tokens("text", n, rows, 2), draw((n, cols), t, 3)
    check_lookup(ctx.embedding(W.cuda(), ids.cuda(), ALPHA, t), W.double(), ids, t)
    P, A, most = by_row(ids, dY, rows)
    got = ctx.embedding_backward(dY.cuda(), ids.int().cuda(), rows, ALPHA)
    check(got, P, error(A, most))


@pytest.mark.parametrize("kind", ["any", "text", "one", "none", "runs"])
@pytest.mark.parametrize("rows,cols,n", [(40_001, 260, 600), (40_001, 260, 16_384), (9_001, 1001, 5000), (32_768, 256, 513), (40_001, 260, 16_385), (300, 32_000, 700)])
def test_large_tables(ctx, rows, cols, n, kind):
    """Rows without a token are zero in memory that held something else."""
    torch.cuda.empty_cache()
    held = torch.full((rows, cols), float("nan"), device="cuda")
    del held
    ids, dY = tokens(kind, n, rows, 2), draw((n, cols), torch.bfloat16, 3)
    got = ctx.embedding_backward(dY.cuda(), ids.cuda(), rows, ALPHA)
    some = ((ids >= 0) & (ids < rows)).nonzero()[:, 0]
    P, A, most = by_row(ids, dY, rows)
    check(got, P, error(A, most))
    assert bool(got[ids[some].cuda()].isfinite().all())


def test_rows_beyond_16_bits_of_the_sort(ctx):
    """Ids that differ in their high bits only, more than one launch ranks."""
    ids = torch.arange(20_000) % 5 * 65_536
    dY = draw((20_000, 8), torch.float32, 1)
    P, A, most = by_row(ids, dY, 300_000)
    check(ctx.embedding_backward(dY.cuda(), ids.cuda(), 300_000, ALPHA), P, error(A, most))


def test_no_tokens_and_no_gradients(ctx):
    layer = Layer(9, 64, 4, 1, 32, torch.float32)
    g = layer.on_gpu(binding)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    dY = torch.empty(0, 64, device="cuda")
    assert ctx.codes_embedding(g, none).shape == (0, 64)
    r = ctx.codes_embedding_backward(g, none, dY)
    assert r["dC"].shape == (4, 1) and r["dS"].shape == (9, 2) and not r["dC"].any() and not r["dS"].any()
    assert ctx.embedding(torch.zeros(3, 5, device="cuda"), none).shape == (0, 5)
    assert not ctx.embedding_backward(torch.empty(0, 5, device="cuda"), none, 3).any()
    assert ctx.codes_embedding_backward(g, none, dY, want_dC=False, want_dS=False) == {}
    ids = tokens("text", 40, 9).cuda()
    dY = draw((40, 64), torch.float32, 1).cuda()
    both = ctx.codes_embedding_backward(g, ids, dY)
    for key in ("dC", "dS"):
        assert torch.equal(ctx.codes_embedding_backward(g, ids, dY, want_dC=key == "dC", want_dS=key == "dS")[key], both[key])


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_strides_and_neighbours(ctx, dtype):
    """Rows of Y and dY that lie apart and begin anywhere; what lies between them stays as it was."""
    t = DTYPES[dtype]
    for layer in (Layer(31, 76, 16, 1, 0, t, seed=4), Layer(31, 64, 256, 4, 64, t, seed=5)):
        cols, ids = layer.cols, tokens("text", 50, 31, 1)
        out = torch.full((51, cols + 14), 7.0, dtype=t, device="cuda")
        check_lookup(ctx.codes_embedding(layer.on_gpu(binding), ids.cuda(), ALPHA, out=out[:50, 5:cols + 5]), layer.weights(), ids, t)
        W = draw((31, cols), torch.float32, 2)
        wide = torch.full((51, cols + 14), 7.0, dtype=t, device="cuda")
        check_lookup(ctx.embedding(W.cuda(), ids.cuda(), ALPHA, out=wide[:50, 5:cols + 5]), W.double(), ids, t)
        for o in (out, wide):
            assert bool((o[50] == 7).all()) and bool((o[:, :5] == 7).all()) and bool((o[:, cols + 5:] == 7).all())
        dY = draw((50, cols + 9), t, 3).cuda()
        got = ctx.codes_embedding_backward(layer.on_gpu(binding), ids.cuda(), dY[:, 3:cols + 3], ALPHA)
        same = ctx.codes_embedding_backward(layer.on_gpu(binding), ids.cuda(), dY[:, 3:cols + 3].contiguous(), ALPHA)
        assert all(torch.equal(got[key], same[key]) for key in same)
        assert torch.equal(ctx.embedding_backward(dY[:, 3:cols + 3], ids.cuda(), 31, ALPHA),
                           ctx.embedding_backward(dY[:, 3:cols + 3].contiguous(), ids.cuda(), 31, ALPHA))


def test_codes_that_are_none_and_numbers_that_are_none(ctx):
    """A code >= k makes its weights NaN, and its group's gradient; a NaN in dY stays in its row, its column's codewords and its group."""
    layer = Layer(20, 64, 3, 1, 32, torch.float32, seed=5)
    layer.codes[11 * 64 + 63] = 3
    layer.words = torch.from_numpy(orc.pack_codes(layer.codes, 4).view(np.int32))
    ids = torch.arange(20)
    Y = ctx.codes_embedding(layer.on_gpu(binding), ids.cuda()).cpu()
    assert bool(Y[11, 63].isnan()) and int(Y.isnan().sum()) == 1
    dY = draw((20, 64), torch.float32, 1)
    dS = ctx.codes_embedding_backward(layer.on_gpu(binding), ids.cuda(), dY.cuda())["dS"].cpu()
    assert bool(dS[11, 1].isnan()) and int(dS.isnan().sum()) == 1
    dY[3, 5] = float("nan")
    dS = ctx.codes_embedding_backward(layer.on_gpu(binding), ids.cuda(), dY.cuda())["dS"].cpu()
    assert bool(dS[3, 0].isnan()) and int(dS.isnan().sum()) == 2
    dW = ctx.embedding_backward(dY.cuda(), ids.cuda(), 20).cpu()
    assert bool(dW[3, 5].isnan()) and int(dW.isnan().sum()) == 1
    # tokens of no row may hold anything
    ids[3] = -1
    assert bool(ctx.embedding_backward(dY.cuda(), ids.cuda(), 20).isfinite().all())
    r = ctx.codes_embedding_backward(layer.on_gpu(binding), ids.cuda(), dY.cuda())
    assert bool(r["dC"].isfinite().all()) and int(r["dS"].isnan().sum()) == 1


def test_refusals(ctx):
    layer = Layer(20, 64, 16, 1, 32, torch.bfloat16).on_gpu(binding)
    ids, dY, W = torch.zeros(5, dtype=torch.int64, device="cuda"), torch.zeros(5, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(20, 64, device="cuda")
    for bad in (ids.float(), ids.cpu(), ids.view(5, 1), torch.zeros(10, dtype=torch.int64, device="cuda")[::2]):
        for call in (lambda i: ctx.codes_embedding(layer, i), lambda i: ctx.embedding(W, i), lambda i: ctx.codes_embedding_backward(layer, i, dY),
                     lambda i: ctx.embedding_backward(dY, i, 20)):
            with pytest.raises(TypeError):
                call(bad)
    for call in (lambda: ctx.codes_embedding_backward(layer, ids, dY.float()), lambda: ctx.codes_embedding_backward(layer, ids, dY[:4]),
                 lambda: ctx.codes_embedding_backward(layer, ids, dY[:, :32]), lambda: ctx.embedding(W.half(), ids), lambda: ctx.embedding(W[:, :32], ids),
                 lambda: ctx.embedding(W, ids, dtype=torch.float64), lambda: ctx.embedding_backward(dY.double(), ids, 20),
                 lambda: ctx.codes_embedding(layer, ids, out=dY.float()), lambda: ctx.embedding(W, ids, out=dY[:4])):
        with pytest.raises(TypeError):
            call()
    for alpha in (float("inf"), float("nan"), 1e39):
        with pytest.raises(binding.IdkmError):
            ctx.codes_embedding(layer, ids, alpha)
        with pytest.raises(binding.IdkmError):
            ctx.embedding_backward(dY, ids, 20, alpha)
