"""Gradients of lookups on both sides of where their forms change: tokens as they come, grouped in one launch, sorted.  The sizes are asked of the
library, so that they stay on their sides when it changes."""
import ctypes

import pytest
import torch

from layer_cases import Layer, draw
from paper_2312_07759_amd import binding
from test_gpu_embedding import run_codes, tokens

pytestmark = pytest.mark.gpu


def last_where(holds, low, high):
    """The largest n with holds(n), which is true at `low` and no longer at `high`."""
    while high - low > 1:
        middle = (low + high) // 2
        low, high = (middle, high) if holds(middle) else (low, middle)
    return low


LIB = binding.load_library()


def workspace(n):
    return LIB.idkm_embedding_backward_workspace(8, 1, n)


# up to FEW tokens nothing is sorted, which needs no workspace; up to GROUPED one launch groups them; more are sorted, between two lists, which is where the
# workspace grows by two words a token at once
FEW = last_where(lambda n: workspace(n) == 0, 1, 4_000_000)
GROUPED = next(n for n in range(FEW + 1, 200_000) if workspace(n + 1) - workspace(n) > 4 * n)


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def test_the_sizes_are_where_the_forms_change():
    assert workspace(FEW) == 0 < workspace(FEW + 1) and FEW < GROUPED


@pytest.mark.parametrize("rows,cols,k,d,group", [(3, 8, 16, 1, 0), (5, 9, 16, 1, 0), (7, 513, 3, 1, 32), (2, 1032, 256, 8, 0), (4, 516, 16, 4, 96), (9, 2048, 128, 1, 512),
                                                 (6, 2048, 16, 1, 1024), (5, 24, 16, 8, 24), (3, 4, 2, 1, 4), (40, 1056, 16, 1, 96), (12, 4096, 16, 1, 1024),
                                                 (90, 960, 16, 1, 160), (30, 1500, 100, 2, 736), (200, 1056, 256, 4, 96), (8, 3000, 64, 2, 1504)])
@pytest.mark.parametrize("more", [1, 388])
def test_rows_that_end_anywhere(ctx, rows, cols, k, d, group, more):
    """Grouped tokens: the last lane's columns overlap its neighbour's, several groups of a row go through segments, rows go on over blocks of places."""
    for dtype in (torch.float32, torch.bfloat16):
        for kind in ("any", "text"):
            run_codes(ctx, Layer(rows, cols, k, d, group, dtype, seed=cols), tokens(kind, FEW + more, rows, 1), cols)


@pytest.mark.parametrize("rows,cols,k,d,group", [(300, 96, 16, 1, 0), (900, 224, 16, 1, 96), (5, 130, 100, 2, 0), (300, 192, 256, 4, 64)])
@pytest.mark.parametrize("n", [GROUPED, GROUPED + 1])
def test_sorted_rows_that_end_anywhere(ctx, rows, cols, k, d, group, n):
    run_codes(ctx, Layer(rows, cols, k, d, group, torch.float32, seed=cols), tokens("text", n, rows, 1), cols)


@pytest.mark.parametrize("n", [6, FEW - 1, FEW + 88, GROUPED - 1, GROUPED + 416])
def test_ids_that_int32_cannot_hold(ctx, n):
    """An int64 id is compared as a whole in every form: 2^32 is no row 0, and a large negative one is padding."""
    ids = torch.tensor([2 ** 32, 2 ** 32 + 3, -2 ** 40, 3, 2 ** 31, -2 ** 31, 2 ** 62 + 1, -2 ** 63, -2 ** 32, 1], device="cuda").repeat(-(-n // 10))[:n]
    counts = torch.stack([(ids == r).sum() for r in range(5)]).float()
    dW = ctx.embedding_backward(torch.ones(n, 16, device="cuda"), ids, 5)
    assert torch.equal(dW, counts[:, None].expand(5, 16))
    stored = Layer(5, 64, 16, 1, 32, torch.float32, seed=1)
    layer, dY = stored.on_gpu(binding), draw((n, 64), torch.float32, 2).cuda()
    got = ctx.codes_embedding_backward(layer, ids, dY)
    ref = ctx.codes_embedding_backward(layer, torch.where((ids >= 0) & (ids < 5), ids, torch.full_like(ids, -1)), dY)
    assert torch.equal(got["dC"], ref["dC"]) and torch.equal(got["dS"], ref["dS"]) and not got["dS"][[0, 2, 4]].any()
    small = torch.tensor([-1, -2 ** 31, 2 ** 31 - 1, 4, 5], dtype=torch.int32, device="cuda").repeat(-(-n // 5))[:n]
    dW = ctx.embedding_backward(torch.ones(n, 16, device="cuda"), small, 5)
    assert bool((dW[4] == float((small == 4).sum())).all()) and not dW[:4].any()


def into_nan(ctx, ids, dY, dW):
    """idkm_embedding_backward into memory that holds NaN."""
    rows, cols = dW.shape
    dW.fill_(float("nan"))
    need = LIB.idkm_embedding_backward_workspace(rows, cols, len(ids))
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    st = LIB.idkm_embedding_backward(ctx._h, rows, cols, ids.data_ptr(), 8, len(ids), ctypes.c_float(1.0), dY.data_ptr(), cols, binding.F32, dW.data_ptr(),
                                     ws.data_ptr(), need, ctx._raw_stream())
    assert st == 0


def whole_numbers(n, cols, seed):
    """dY whose sums are exact in any order."""
    return torch.randint(-8, 9, (n, cols), generator=torch.Generator().manual_seed(seed)).float().cuda()


@pytest.mark.parametrize("kind", ["any", "text", "one", "none", "runs"])
@pytest.mark.parametrize("rows,cols", [(40_001, 260), (9_001, 1001), (1, 5), (32_768, 256)])
@pytest.mark.parametrize("n", [0, 1, FEW, FEW + 1, GROUPED, GROUPED + 1])
def test_every_row_is_written(ctx, n, rows, cols, kind):
    """All of dW, wherever it begins, and nothing beside it."""
    ids, dY = tokens(kind, n, rows, 2).cuda(), whole_numbers(n, cols, 3)
    held = (ids >= 0) & (ids < rows)
    ref = torch.zeros(rows, cols, device="cuda").index_add_(0, ids[held], dY[held])
    for offset in (0, 1):
        room = torch.full((rows * cols + 8,), 7.0, device="cuda")
        dW = room[4 + offset:4 + offset + rows * cols].view(rows, cols)
        into_nan(ctx, ids, dY, dW)
        assert torch.equal(dW, ref)
        assert bool((room[:4 + offset] == 7).all()) and bool((room[4 + offset + rows * cols:] == 7).all())


@pytest.mark.parametrize("rows,cols,k,d,group", [(5000, 96, 16, 1, 32), (3001, 105, 16, 1, 105), (3000, 1056, 16, 1, 96), (2000, 96, 512, 1, 32), (777, 192, 256, 8, 64)])
@pytest.mark.parametrize("n", [1, FEW, FEW + 1, GROUPED, GROUPED + 1])
def test_every_scale_is_written(ctx, n, rows, cols, k, d, group):
    """All of a stored table's dS and dC, from a workspace that holds something else."""
    stored = Layer(rows, cols, k, d, group, torch.float32, seed=rows)
    layer, ids, dY = stored.on_gpu(binding), tokens("text", n, rows, 2).cuda(), draw((n, cols), torch.float32, 3).cuda()
    ref = ctx.codes_embedding_backward(layer, ids, dY)
    dS, dC = torch.full((rows, layer.groups), float("nan"), device="cuda"), torch.full((k, d), float("nan"), device="cuda")
    ws = torch.full((layer.workspace_bytes(n, lookup=True),), 255, dtype=torch.uint8, device="cuda")
    st = LIB.idkm_codes_embedding_backward(ctx._h, layer._at, ids.data_ptr(), 8, n, ctypes.c_float(1.0), dY.data_ptr(), cols, dC.data_ptr(), dS.data_ptr(),
                                           ws.data_ptr(), ws.numel(), ctx._raw_stream())
    assert st == 0 and torch.equal(dS, ref["dS"]) and torch.equal(dC, ref["dC"])
    without = torch.ones(rows, dtype=torch.bool, device="cuda")
    without[ids[(ids >= 0) & (ids < rows)]] = False
    assert not dS[without].any()


@pytest.mark.parametrize("n", [7, FEW + 188, GROUPED + 616])
def test_gradient_of_more_than_2_31_elements(ctx, n):
    """Every element: rows without a token are zero in memory that held NaN, the others have their sums, also behind the 2^31st."""
    rows, cols = 3_600_000, 640
    ids = torch.tensor([0, rows - 1, 5, rows - 2, rows - 1, -1, 3_355_444], device="cuda").repeat(-(-n // 7))[:n]
    dY, dW = whole_numbers(n, cols, 1), torch.empty(rows, cols, device="cuda")
    assert dW.numel() > 2 ** 31
    into_nan(ctx, ids, dY, dW)
    at = torch.tensor([0, 5, 3_355_444, rows - 2, rows - 1], device="cuda")
    for row in at.tolist():
        assert torch.equal(dW[row], dY[ids == row].sum(0)), row
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[at] = False
    for r in range(0, rows, 400_000):
        assert not dW[r:r + 400_000][other[r:r + 400_000]].any(), r


@pytest.mark.parametrize("n", [7, FEW + 188])
def test_scales_of_the_largest_stored_tables(ctx, n):
    """dS beyond 2^32 bytes, of a table whose codes take as many: every scale, from memory that held NaN."""
    rows, cols, group = 4_000_000, 16_384, 32
    words = torch.zeros(rows, cols // 32, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 5, 1_700_000, rows - 2, rows - 1], device="cuda")
    ids = torch.tensor([0, rows - 1, 5, rows - 2, rows - 1, -1, 1_700_000], device="cuda").repeat(-(-n // 7))[:n]
    words[at] = torch.randint(-2 ** 31, 2 ** 31 - 1, (5, cols // 32), generator=torch.Generator().manual_seed(1)).int().cuda()
    C = torch.tensor([[1.0], [2.0]], device="cuda")
    S = torch.empty(rows, cols // group, device="cuda")
    S.fill_(1.0)
    layer = binding.CodesLayer(words.view(-1), rows, cols, C, S, group)
    dY, dS, dC = whole_numbers(n, cols, 2), torch.empty(rows, cols // group, device="cuda"), torch.empty(2, 1, device="cuda")
    dS.fill_(float("nan"))
    ws = torch.empty(layer.workspace_bytes(n, lookup=True), dtype=torch.uint8, device="cuda")
    st = LIB.idkm_codes_embedding_backward(ctx._h, layer._at, ids.data_ptr(), 8, n, ctypes.c_float(1.0), dY.data_ptr(), cols, dC.data_ptr(), dS.data_ptr(),
                                           ws.data_ptr(), ws.numel(), ctx._raw_stream())
    assert st == 0
    sums = torch.zeros(2, dtype=torch.float64, device="cuda")
    for row in at.tolist():
        codes = ((words[row][:, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).reshape(-1)
        P = dY[ids == row].sum(0)
        assert torch.equal(dS[row], (P * (1 + codes)).view(-1, group).sum(1)), row
        sums += torch.stack([P[codes == 0].sum(dtype=torch.float64), P[codes == 1].sum(dtype=torch.float64)])
    assert torch.equal(dC[:, 0].double(), sums)  # whole numbers below 2^24
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[at] = False
    for r in range(0, rows, 400_000):
        assert not dS[r:r + 400_000][other[r:r + 400_000]].any(), r
