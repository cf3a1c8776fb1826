"""The loss against a teacher's largest logits and its gradient (idkm_distill) against float64."""
import math

import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, check, draw
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def make(n, V, top, dtype, seed, holes=True):
    g = torch.Generator().manual_seed(seed)
    z = (3 * torch.randn(n, V, generator=g)).to(dtype)
    index = torch.stack([torch.randperm(V, generator=g)[:top] if top <= V else torch.randint(0, V, (top,), generator=g) for _ in range(n)])
    teacher = 4 * torch.randn(n, top, generator=g)
    if holes:
        index[torch.rand(n, top, generator=g) < 0.2] = -1
        if n > 2:
            index[n // 2] = -1
    return z, index.to(torch.int32), teacher, torch.rand(n, generator=g)


def reference(z, index, teacher, tau, weight):
    """loss, lse, gradient and p, q in float64."""
    z = z.double() / tau
    n, V = z.shape
    lse = torch.logsumexp(z, 1)
    q = torch.exp(z - lse[:, None])
    p = torch.zeros(n, V, dtype=torch.float64)
    loss = torch.zeros(n, dtype=torch.float64)
    for t in range(n):
        held = index[t] >= 0
        if not bool(held.any()):
            q[t] = 0
            continue
        lp = torch.log_softmax(teacher[t][held].double() / tau, 0)
        at = index[t][held].long()
        p[t].index_add_(0, at, lp.exp())
        some = lp.exp() > 0
        loss[t] = (lp.exp() * (lp - (z[t, at] - lse[t])))[some].sum()
    return loss, lse, weight.double()[:, None] / tau * (q - p), p, q


def compare(got, z, index, teacher, tau, weight):
    loss, lse, dz, p, q = reference(z, index, teacher, tau, weight)
    # float32 exponents of values up to `big` and sums of V terms of one sign: a few steps each
    big = float(z.double().abs().max() / tau + teacher.double().abs().max() / tau) + 10
    rel = 2.0 ** -24 * (16 + 4 * big)
    check(got[1], lse, rel * (1 + lse.abs()), "lse")
    check(got[0], loss, rel * (big + loss.abs()), "loss")
    if len(got) > 2:
        t = z.dtype
        size = weight.double()[:, None] / tau * (q + p)
        small = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -126}[t]   # subnormal steps; q below them is 0
        check(got[2], dz, HALF_STEP[t] * dz.abs() + rel * size + small, "dlogits")


SIZES = [(1, 1, 1), (2, 7, 3), (5, 64, 8), (3, 1000, 5), (300, 1000, 5), (4, 2049, 64), (3, 8192, 20), (257, 8200, 7), (2, 33333, 100),
         (260, 17001, 16), (1, 131072, 64), (2, 140001, 64), (258, 70001, 3)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n,V,top", SIZES)
def test_loss_and_gradient(ctx, n, V, top, dtype):
    z, index, teacher, weight = make(n, V, top, DTYPES[dtype], n + V)
    for tau in ((1.0, 2.5) if n < 100 else (2.5,)):
        args = (z.cuda(), index.cuda(), teacher.cuda(), tau)
        got = ctx.distill(*args, weight.cuda())
        compare(got, z, index, teacher, tau, weight)
        plain = ctx.distill(*args)
        assert len(plain) == 2 and torch.equal(plain[0], got[0]) and torch.equal(plain[1], got[1])


@pytest.mark.parametrize("n,V", [(3, 500), (2, 40000), (300, 3000), (260, 40001)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_in_place_and_strides(ctx, n, V, dtype):
    t = DTYPES[dtype]
    z, index, teacher, weight = make(n, V, 9, t, 3)
    ref = ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), 2.0, weight.cuda())
    wide = torch.full((n, V + 10), 7.0, dtype=t, device="cuda")
    inner = wide[:, 3:V + 3]
    inner.copy_(z.cuda())
    got = ctx.distill(inner, index.cuda(), teacher.cuda(), 2.0, weight.cuda(), out=inner)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    assert bool((wide[:, :3] == 7).all()) and bool((wide[:, V + 3:] == 7).all())


@pytest.mark.parametrize("n,V", [(4, 300), (4, 30000), (300, 30000)])
def test_repeated_indices_add_up(ctx, n, V):
    z, index, teacher, weight = make(n, V, 12, torch.float32, 4, holes=False)
    index[:, 5], index[:, 9], index[:, 11] = index[:, 2], index[:, 2], index[:, 0]
    compare(ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), 1.5, weight.cuda()), z, index, teacher, 1.5, weight)


@pytest.mark.parametrize("n,V", [(6, 300), (6, 30000), (256, 30000)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_masks_and_extremes(ctx, n, V, dtype):
    t = DTYPES[dtype]
    z, index, teacher, weight = make(n, V, 6, t, 5, holes=False)
    lowest = torch.finfo(t).min
    keep = index[0].long()
    z[0] = -math.inf
    z[0, keep] = 1.0                              # all of the vocabulary masked but the teacher's places
    z[1] = lowest                                 # a row of the type's lowest value: even
    z[2, ::2] = lowest
    teacher[3, 1:] = -math.inf                    # one entry only
    index[4] = -1                                 # nothing, and logits that are no numbers
    z[4] = math.nan
    teacher[5] = -math.inf                        # entries without any mass
    got = [x.cpu() for x in ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), 2.0, weight.cuda())]
    loss, lse, dz, p, q = reference(z, index, teacher, 2.0, weight)
    assert got[0][4] == 0 and not got[2][4].any() and got[0][5] == 0 and not got[2][5].any()
    assert abs(float(got[1][1]) - float(lse[1])) <= 2.0 ** -22 * abs(float(lse[1]))
    uniform = weight[1].double() / 2.0 / V
    free = torch.ones(V, dtype=torch.bool)
    free[index[1].long()] = False
    small = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0, torch.float32: 0.0}[t]
    assert bool(((got[2][1][free].double() - uniform).abs() <= (HALF_STEP[t] + 2.0 ** -18) * uniform + small).all())
    sel = [0, 2, 3]
    rel = 2.0 ** -24 * 200
    check(got[0][sel], loss[sel], rel * (10 + loss[sel].abs()), "loss")
    size = weight.double()[:, None] / 2.0 * (q + p)
    check(got[2][sel], dz[sel], (HALF_STEP[t] * dz.abs() + rel * size + (small or 2.0 ** -126))[sel], "dlogits")
    if n > 6:
        check(got[0][6:], loss[6:], rel * (10 + loss[6:].abs()), "loss")


@pytest.mark.parametrize("n,V", [(3, 300), (3, 30000), (256, 30000)])
def test_lists_that_are_none(ctx, n, V):
    """An index outside the row or a NaN in the list: NaN there, nowhere else."""
    z, index, teacher, weight = make(n, V, 6, torch.float32, 6, holes=False)
    index[0, 3] = V
    teacher[1, 2] = math.nan
    loss, lse, dz = (x.cpu() for x in ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), 1.0, weight.cuda()))
    assert bool(loss[:2].isnan().all()) and bool(dz[:2].isnan().all()) and bool(lse.isfinite().all())
    assert bool(loss[2:].isfinite().all()) and bool(dz[2:].isfinite().all())


def test_gradient_against_differences(ctx):
    z, index, teacher, weight = make(4, 257, 10, torch.float32, 7)
    dz = ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), 1.7, weight.cuda())[2].double().cpu()
    D = draw((4, 257), torch.float32, 1).double()
    e = 1e-5
    value = [float((weight.double() * reference(z.double() + s * e * D, index, teacher, 1.7, weight)[0]).sum()) for s in (1, -1)]
    assert abs((value[0] - value[1]) / (2 * e) - float((dz * D).sum())) < 1e-5


@pytest.mark.parametrize("n,V", [(2, 300), (3, 40000), (256, 9000)])
def test_captured_graph(ctx, n, V):
    z, index, teacher, weight = (x.cuda() for x in make(n, V, 6, torch.bfloat16, 8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ctx.distill(z, index, teacher, 2.0, weight)
    for i in range(3):
        for old, new in zip((z, index, teacher, weight), make(n, V, 6, torch.bfloat16, 9 + i)):
            old.copy_(new.cuda())
        graph.replay()
        ref = ctx.distill(z, index, teacher, 2.0, weight)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_refusals(ctx):
    z, index, teacher, weight = (x.cuda() for x in make(3, 100, 6, torch.float32, 8))
    for bad in ((z, index.long(), teacher, 1.0), (z, index, teacher.half(), 1.0), (z, index[:, :5], teacher, 1.0), (z.double(), index, teacher, 1.0),
                (z[0], index, teacher, 1.0), (z, index.cpu(), teacher, 1.0), (z, index, teacher, 1.0, weight[:2]), (z.t(), index, teacher, 1.0)):
        with pytest.raises(TypeError):
            ctx.distill(*bad)
    with pytest.raises(TypeError):
        ctx.distill(z, index, teacher, 1.0, None, z)
    for tau in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(binding.IdkmError) as e:
            ctx.distill(z, index, teacher, tau)
        assert e.value.status == 1 and "tau" in e.value.detail
    with pytest.raises(binding.IdkmError):
        ctx.distill(z, torch.zeros(3, 1025, dtype=torch.int32, device="cuda"), torch.zeros(3, 1025, device="cuda"), 1.0)
    assert ctx.distill(z[:0], index[:0], teacher[:0], 1.0)[0].shape == (0,)
