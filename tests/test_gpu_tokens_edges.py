"""Lookups, inputs in 8 bits and products in 8-bit integers where offsets pass 32 bits, calls overlap, are captured, or get arguments that the binding
does not let through."""
import ctypes

import pytest
import torch

from layer_cases import HALF_STEP, Layer, draw
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def some_calls(ctx):
    """Every operator at sizes of each of its forms: a list of calls and what they give eagerly."""
    g = torch.Generator().manual_seed(1)
    calls = []
    for n, k, d, group in ((1, 16, 1, 64), (200, 16, 1, 64), (300, 100, 2, 0), (5000, 16, 1, 192), (300, 256, 4, 64), (20000, 16, 1, 64)):
        layer = Layer(700, 192, k, d, group, torch.bfloat16, seed=n).on_gpu(binding)
        ids = torch.randint(-1, 700, (n,), generator=g).cuda()
        dY = draw((n, 192), torch.bfloat16, n).cuda()
        calls.append(lambda layer=layer, ids=ids: [ctx.codes_embedding(layer, ids)])
        calls.append(lambda layer=layer, ids=ids, dY=dY: list(ctx.codes_embedding_backward(layer, ids, dY).values()))
        calls.append(lambda ids=ids, dY=dY: [ctx.embedding_backward(dY, ids, 700)])
    W = draw((700, 192), torch.float32, 5).cuda()
    calls.append(lambda: [ctx.embedding(W, ids)])
    for n in (1, 30, 300):
        X, dY = draw((n, 640), torch.float16, n).cuda(), draw((n, 90), torch.float16, n + 1).cuda()
        layer = Layer(90, 640, 16, 1, 64, torch.float16, seed=n).on_gpu(binding)
        eight = ctx.int8_layer(layer)
        calls.append(lambda X=X: [ctx.restore8(ctx.keep8(X))])
        calls.append(lambda X=X, dY=dY, layer=layer: list(ctx.codes_linear_backward(layer, ctx.keep8(X), dY).values()))
        calls.append(lambda X=X, eight=eight: [ctx.int8_linear(eight, X)])
        calls.append(lambda dY=dY, eight=eight: [ctx.int8_linear_backward(eight, dY)])
    return calls


def test_captured_before_any_eager_call():
    """Nothing that a first call does may fail under capture, and every replay gives the eager results, with eager work between them."""
    c = binding.Context(0)
    calls = some_calls(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [call() for call in calls]
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        for held, call in zip(got, calls):
            assert all(torch.equal(a, b) for a, b in zip(held, call()))
        torch.cuda.synchronize()
    c.close()


def test_many_streams_at_once(ctx):
    calls = some_calls(ctx)
    ref = [call() for call in calls]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for i, call in enumerate(calls):
            with torch.cuda.stream(streams[i % 4]):
                got.append(call())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, ref) for a, b in zip(x, y))


def test_tables_beyond_32_bits(ctx):
    """A float32 table of more than 2^31 elements, and its gradient; a stored one of more than 2^31 weights."""
    rows, cols = 3_600_000, 640
    ids = torch.tensor([0, rows - 1, 5, rows - 2, rows - 1, -1, 3_355_444], device="cuda")
    W = torch.empty(rows, cols, device="cuda")
    W[ids] = draw((7, cols), torch.float32, 1).cuda()
    assert torch.equal(ctx.embedding(W, ids)[ids >= 0], W[ids[ids >= 0]])
    del W
    for n in (7, 700):
        many = ids.repeat(n // 7)
        dY = torch.ones(n, cols, device="cuda")
        dW = ctx.embedding_backward(dY, many, rows)
        assert torch.equal(dW[ids[:3]], torch.tensor([1.0, 2.0, 1.0], device="cuda")[:, None].expand(3, cols) * (n // 7))
        assert float(dW.view(-1, 2 ** 16 * 3).sum(1, dtype=torch.float64).sum()) == n // 7 * 6 * cols if dW.numel() % (2 ** 16 * 3) == 0 else True
        assert not dW[1:5].any() and not dW[rows - 100:rows - 2].any()
        del dW
    words = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows * cols * 4 // 32,), dtype=torch.int64, device="cuda").to(torch.int32)
    C = torch.linspace(-1, 1, 16, device="cuda")[:, None].contiguous()
    layer = binding.CodesLayer(words, rows, cols, C)
    held = ids[ids >= 0]
    codes = (words.view(rows, cols // 8)[held][:, :, None] >> torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)) & 15
    codes = codes.reshape(len(held), cols).long()
    assert torch.equal(ctx.codes_embedding(layer, ids)[ids >= 0], C[:, 0][codes])
    dC = ctx.codes_embedding_backward(layer, ids, torch.ones(7, cols, device="cuda"))["dC"]
    assert torch.equal(dC[:, 0], torch.bincount(codes.reshape(-1), minlength=16).float())


def test_stored_tables_of_more_than_2_31_words(ctx):
    """Rows whose words lie further from the stream's end than 32 bits tell."""
    rows, cols = 3_600_000, 2400
    ids = torch.tensor([0, rows - 1, 5, rows - 2, rows - 1, -1, 1_700_000], device="cuda")
    words = torch.zeros(rows, cols // 4, dtype=torch.int32, device="cuda")
    held = ids[ids >= 0]
    words[held] = torch.randint(-2 ** 31, 2 ** 31 - 1, (6, cols // 4), generator=torch.Generator().manual_seed(1)).int().cuda()
    C = torch.linspace(-1, 1, 256, device="cuda")[:, None].contiguous()
    layer = binding.CodesLayer(words.view(-1), rows, cols, C)
    codes = ((words[held][:, :, None] >> torch.arange(0, 32, 8, device="cuda", dtype=torch.int32)) & 255).reshape(6, cols).long()
    assert torch.equal(ctx.codes_embedding(layer, ids)[ids >= 0], C[:, 0][codes])
    for n in (7, 700):
        dC = ctx.codes_embedding_backward(layer, ids.repeat(n // 7), torch.ones(n, cols, device="cuda"))["dC"]
        assert torch.equal(dC[:, 0], n // 7 * torch.bincount(codes.reshape(-1), minlength=256).float())


def test_activations_beyond_32_bits(ctx):
    """More than 2^31 elements of activations: kept, brought back, in integers, looked up and summed."""
    n, cols = 600_000, 4096
    X = torch.zeros(n, cols, dtype=torch.bfloat16, device="cuda")
    X[-1] = draw((cols,), torch.bfloat16, 1).cuda()
    X[524_289, 7] = 3.0
    kept = ctx.keep8(X)
    back = ctx.restore8(kept)
    assert torch.equal(back[-1], ctx.restore8(ctx.keep8(X[-1:]))[0]) and float(back[524_289, 7]) == 3.0 and not back[524_290:n - 1].any()
    del kept, back
    eight = ctx.int8_layer(draw((3, cols), torch.float32, 2).cuda(), torch.bfloat16)
    assert torch.equal(ctx.int8_linear(eight, X)[-1], ctx.int8_linear(eight, X[-1:])[0])
    ids = torch.full((n,), -1, device="cuda")
    ids[-1], ids[524_289] = 3, 4
    dW = ctx.embedding_backward(X, ids, 9)
    assert torch.equal(dW[3], X[-1].float()) and float(dW[4].sum()) == 3.0 and not dW[5:].any() and not dW[:3].any()
    layer = Layer(9, cols, 16, 1, 128, torch.bfloat16, seed=3).on_gpu(binding)
    got, ref = ctx.codes_embedding_backward(layer, ids, X), ctx.codes_embedding_backward(layer, ids[[524_289, n - 1]], X[[524_289, n - 1]])
    # the sums of a row are the same; over rows dC may be added up in another order: two terms' difference of 2^-24 each
    assert torch.equal(got["dS"], ref["dS"]) and bool(((got["dC"] - ref["dC"]).abs() <= 2.0 ** -18 * ref["dC"].abs().max()).all())
    ids[:] = torch.arange(n, device="cuda") % 9
    Y = ctx.codes_embedding(layer, ids)
    assert torch.equal(Y[-9:], ctx.codes_embedding(layer, ids[-9:])) and torch.equal(Y[524_280:524_289], ctx.codes_embedding(layer, ids[524_280:524_289]))


@pytest.mark.parametrize("rows,cols,k,d,group", [(3, 8, 16, 1, 0), (5, 9, 16, 1, 0), (7, 513, 3, 1, 32), (2, 1032, 256, 8, 0), (4, 516, 16, 4, 96), (9, 2048, 128, 1, 512),
                                                 (6, 2048, 16, 1, 1024), (5, 24, 16, 8, 24), (3, 4, 2, 1, 4)])
def test_rows_that_end_anywhere(ctx, rows, cols, k, d, group):
    """The last lane's columns overlap its neighbour's; groups that end inside a wavefront's columns, and are as long as rows."""
    from test_gpu_embedding import run_codes, tokens
    for n in (3, 400):
        for dtype in (torch.float32, torch.float16):
            run_codes(ctx, Layer(rows, cols, k, d, group, dtype, seed=cols), tokens("any", n, rows, 1), n)


def test_the_same_sums_however_they_are_split(ctx):
    """A call's results repeat, and do not depend on what else is wanted or on the ids' type."""
    layer = Layer(500, 256, 16, 1, 64, torch.float32, seed=1).on_gpu(binding)
    ids = torch.randint(-1, 500, (3000,), generator=torch.Generator().manual_seed(1))
    ids[::3] = 7
    dY = draw((3000, 256), torch.float32, 2).cuda()
    a, b = ctx.codes_embedding_backward(layer, ids.cuda(), dY), ctx.codes_embedding_backward(layer, ids.int().cuda(), dY)
    assert torch.equal(a["dC"], b["dC"]) and torch.equal(a["dS"], b["dS"])
    assert torch.equal(ctx.codes_embedding_backward(layer, ids.cuda(), dY, want_dS=False)["dC"], a["dC"])
    assert torch.equal(ctx.codes_embedding_backward(layer, ids.cuda(), dY, want_dC=False)["dS"], a["dS"])
    assert torch.equal(ctx.embedding_backward(dY, ids.cuda(), 500), ctx.embedding_backward(dY, ids.int().cuda(), 500))


def test_ids_that_int32_cannot_hold(ctx):
    """An int64 id is compared as a whole: 2^32 is no row 0, and a large negative one is padding."""
    W = draw((5, 16), torch.float32, 1).cuda()
    ids = torch.tensor([2 ** 32, 2 ** 32 + 3, -2 ** 40, 3, 2 ** 31, -2 ** 31], device="cuda")
    Y = ctx.embedding(W, ids)
    assert bool(Y[[0, 1, 4]].isnan().all()) and not Y[[2, 5]].any() and torch.equal(Y[3], W[3])
    for n in (1, 60):  # up to 256 tokens and more
        dW = ctx.embedding_backward(torch.ones(6 * n, 16, device="cuda"), ids.repeat(n), 5)
        assert bool((dW[3] == n).all()) and not dW[[0, 1, 2, 4]].any()
    small = torch.tensor([-1, -2 ** 31, 2 ** 31 - 1, 4], dtype=torch.int32, device="cuda")
    Y = ctx.embedding(W, small)
    assert not Y[:2].any() and bool(Y[2].isnan().all()) and torch.equal(Y[3], W[4])
    for n in (1, 100):
        dW = ctx.embedding_backward(torch.ones(4 * n, 16, device="cuda"), small.repeat(n), 5)
        assert bool((dW[4] == n).all()) and not dW[:4].any()


def test_arguments_that_the_library_refuses(ctx):
    """Through the C entry points: nothing is launched, the message says why."""
    lib, h = ctx._lib, ctx._h
    t = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = t.data_ptr()
    layer = Layer(8, 64, 16, 1, 32, torch.bfloat16).on_gpu(binding)
    eight = ctx.int8_layer(torch.zeros(8, 64, device="cuda"), torch.bfloat16)
    w, q, f = layer._at, eight._at, ctypes.c_float
    big = 1 << 15

    def refused(name, *args, status=1):
        assert getattr(lib, name)(h, *args) == status, (name, args)
        assert lib.idkm_last_error(h)

    for ids, width, n, alpha, Y, ld in ((0, 8, 4, 1.0, p, 64), (p, 3, 4, 1.0, p, 64), (p + 4, 8, 4, 1.0, p, 64), (p, 8, -1, 1.0, p, 64), (p, 8, 4, float("nan"), p, 64),
                                        (p, 8, 4, 1.0, 0, 64), (p, 8, 4, 1.0, p + 1, 64), (p, 8, 4, 1.0, p, 63)):
        refused("idkm_codes_embedding", w, ids, width, n, f(alpha), Y, ld, None)
        refused("idkm_embedding", p, 8, 64, ids, width, n, f(alpha), Y, ld, 2, None)
        refused("idkm_codes_embedding_backward", w, ids, width, n, f(alpha), Y, ld, p, p, p, big, None)
        refused("idkm_embedding_backward", 8, 64, ids, width, n, f(alpha), Y, ld, 2, p, p, big, None)
    refused("idkm_codes_embedding", w, p, 8, 4_000_001, f(1.0), p, 64, None, status=6)
    refused("idkm_codes_embedding_backward", w, p, 8, 4, f(1.0), p, 64, p, p, p, 8, None)          # a workspace that is too small
    refused("idkm_codes_embedding_backward", w, p, 8, 4, f(1.0), p, 64, p, p, p + 8, big, None)    # .. not aligned
    refused("idkm_codes_embedding_backward", w, p, 8, 4, f(1.0), p, 64, p + 2, p, p, big, None)
    refused("idkm_embedding_backward", 8, 64, p, 8, 600, f(1.0), p, 64, 2, p, p, 16, None)
    refused("idkm_embedding_backward", 8, 64, p, 8, 4, f(1.0), p, 64, 2, None, None, 0, None)
    refused("idkm_embedding", p, 0, 64, p, 8, 4, f(1.0), p, 64, 2, None)
    refused("idkm_embedding", p, 8, 64, p, 8, 4, f(1.0), p, 64, 5, None)
    refused("idkm_embedding", 0, 8, 64, p, 8, 4, f(1.0), p, 64, 2, None)
    refused("idkm_embedding", p, 4_000_001, 64, p, 8, 4, f(1.0), p, 64, 2, None, status=6)
    for X, n, cols, ld, dtype, Q, E in ((0, 4, 64, 64, 2, p, p), (p, 4, 64, 63, 2, p, p), (p, 4, 64, 64, 3, p, p), (p, 4, 64, 64, 2, p + 4, p), (p, 4, 64, 64, 2, p, 0),
                                        (p, -1, 64, 64, 2, p, p), (p, 4, 0, 64, 2, p, p), (p + 1, 4, 64, 64, 2, p, p)):
        refused("idkm_keep8", X, n, cols, ld, dtype, Q, E, None)
        refused("idkm_restore8", Q, E, n, cols, dtype, X, ld, None)
    refused("idkm_codes_linear_backward_kept", w, p, None, p, 8, 4, p, 64, p, p, p, big, None)
    refused("idkm_codes_linear_backward_kept", w, None, p, p, 8, 4, p, 64, p, p, p, big, None)
    refused("idkm_codes_linear_backward_kept", w, p + 4, p, p, 8, 4, p, 64, p, p, p, big, None)
    for X, n, cols, ld, dtype, Q, ldq, s in ((0, 4, 64, 64, 2, p, 64, p), (p, 4, 64, 64, 2, p, 72, p), (p, 4, 64, 64, 2, p, 48, p), (p, 4, 64, 64, 2, p + 8, 64, p),
                                             (p, 4, 64, 63, 2, p, 64, p), (p, 4, 64, 64, 2, p, 64, 0), (p, 4, 64, 64, 9, p, 64, p)):
        refused("idkm_int8_rows", X, n, cols, ld, dtype, Q, ldq, s, None)
    for X, n, ldx, Y, ldy, ws, have in ((0, 9, 64, p, 8, p, big), (p, 9, 63, p, 8, p, big), (p, 9, 64, p, 7, p, big), (p + 1, 9, 64, p, 8, p, big), (p, -1, 64, p, 8, p, big),
                                        (p, 9, 64, p, 8, p, 16), (p, 9, 64, p, 8, 0, 0)):
        refused("idkm_int8_linear", q, X, n, ldx, Y, ldy, ws, have, None)
        refused("idkm_int8_linear_backward", q, Y, ldy, n, X, ldx, ws, have, None)
    torch.cuda.synchronize()
    assert not t.any()
