"""The loss against a teacher over the whole range of logits and temperatures: maxima far from zero and small temperatures, where the
exponents' common part is large, against float64."""
import math

import pytest
import torch

from layer_cases import DTYPES, HALF_STEP, check
from paper_2312_07759_amd import binding
from test_gpu_distill import ctx, make, reference  # noqa: F401

pytestmark = pytest.mark.gpu

# one wavefront, one workgroup, several workgroups to a row, a row longer than its workgroup's registers
FORMS = [(6, 300), (6, 30_000), (6, 40_000), (256, 70_001)]


def compare(got, z, index, teacher, tau, weight):
    """An exponent is a difference times 1 / tau: three roundings of 2^-24 of it, and it counts up to 104 (below e^-104 float32 holds
    nothing); sums of terms of one sign are off by some steps.  So q, p and their logarithms are off by `rel` of themselves, and an
    exponential below 2^-126, which the hardware's instruction gives as nothing, by as much, times weight / tau."""
    # differences to the maximum first: float64, too, loses log V beside 1e30
    top = z.double().amax(1, keepdim=True)
    loss, lse, dz, p, q = reference(z.double() - top, index, teacher, tau, weight)
    zt = (z.double() - top).gather(1, index.long()) / tau
    rest, lse = lse, lse + top[:, 0] / tau
    rel = 2.0 ** -24 * (32 + 4 * 104)
    check(got[1], lse, rel * (1 + lse.abs()), "lse")
    lp = torch.log_softmax(teacher.double() / tau, 1)
    size = (lp.exp() * torch.where(lp.exp() > 0, lp.abs() + (zt - rest[:, None]).abs(), 0.0)).sum(1)
    check(got[0], loss, rel * (1 + size), "loss")
    small = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126, torch.float32: 2.0 ** -126}[z.dtype]
    check(got[2], dz, HALF_STEP[z.dtype] * dz.abs() + weight.double()[:, None] / tau * (rel * (q + p) + 2.0 ** -126) + small, "dlogits")


@pytest.mark.parametrize("n,V", FORMS)
@pytest.mark.parametrize("tau", [1.0, 0.3, 2.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_maxima_far_from_zero(ctx, n, V, tau, dtype):  # noqa: F811
    z, index, teacher, weight = make(n, V, 6, DTYPES[dtype], 11, holes=False)
    z[0] = -1e10                                  # a row that a finite mask covers as a whole: even
    z[1] = -1e9
    z[2] = -1e30
    z[3, 7] = 3e20                                # one logit that is all of the softmax
    z[4, ::2] = -1e30                             # ordinary logits between masked ones
    z[5] = 1e12
    z[5, ::3] = 1e12 * (1 - 2.0 ** -6)
    got = ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), tau, weight.cuda())
    compare(got, z, index, teacher, tau, weight)


@pytest.mark.parametrize("n,V", FORMS)
@pytest.mark.parametrize("tau", [1e-3, 1e-7, 1e-12, 2.0 ** -126])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_small_temperatures(ctx, n, V, tau, dtype):  # noqa: F811
    z, index, teacher, weight = make(n, V, 6, DTYPES[dtype], 12, holes=False)
    z, teacher = (z.float() / 32).to(z.dtype), teacher / 32          # differences over 2^-126 stay finite
    tau, weight = float(torch.tensor(tau, dtype=torch.float32)), weight * tau
    got = ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), tau, weight.cuda())
    compare(got, z, index, teacher, tau, weight.float())


@pytest.mark.parametrize("exponent", [21, 22, 23, 24, 25, 30, 31, 32])
def test_on_both_sides_of_the_change_of_form(ctx, exponent):  # noqa: F811
    """Rows that lie 2^exponent below zero: their lse moves with them, loss and gradient stay."""
    g = torch.Generator().manual_seed(exponent)
    step = max(1.0, 2.0 ** (exponent - 23))       # representable differences
    z = torch.randint(0, 5, (4, 700), generator=g).float() * step - 2.0 ** exponent
    index, teacher = torch.randint(0, 700, (4, 3), generator=g).to(torch.int32), torch.randn(4, 3, generator=g)
    index[:, 1], index[:, 2] = (index[:, 0] + 1) % 700, (index[:, 0] + 2) % 700
    weight = torch.ones(4)
    got = ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), step, weight.cuda())
    compare(got, z, index, teacher, step, weight)


def test_logits_that_are_no_numbers(ctx):  # noqa: F811
    for n, V in FORMS:
        z, index, teacher, weight = make(n, V, 6, torch.float32, 13, holes=False)
        z[0, 5], z[1, 6], z[2, 9] = math.inf, math.nan, math.inf
        index[2] = -1
        loss, lse, dz = (x.cpu() for x in ctx.distill(z.cuda(), index.cuda(), teacher.cuda(), 1.0, weight.cuda()))
        assert bool(lse[:3].isnan().all()) and bool(loss[:2].isnan().all()) and bool(dz[:2].isnan().all())
        assert loss[2] == 0 and not dz[2].any()
        assert bool(lse[3:].isfinite().all()) and bool(loss[3:].isfinite().all()) and bool(dz[3:].isfinite().all())


@pytest.mark.parametrize("V", [300, 40_000])
def test_an_index_listed_twice(ctx, V):  # noqa: F811
    """Its entries stay apart in the loss: two equal ones at a logit that is all of the softmax give -log 2.  The gradient is that of one
    entry with their sum, and so is the loss but for the entries' own term, whatever the logits are."""
    z = torch.full((2, V), -200.0)
    z[:, 7] = 100.0
    index = torch.tensor([[7, 7], [7, -1]], dtype=torch.int32)
    loss, lse, dz = (x.cpu() for x in ctx.distill(z.cuda(), index.cuda(), torch.zeros(2, 2, device="cuda"), 1.0, torch.ones(2, device="cuda")))
    assert abs(float(loss[0]) + math.log(2)) < 1e-6 and abs(float(loss[1])) < 1e-6
    assert float((dz[0] - dz[1]).abs().max()) <= 2.0 ** -22          # 1/2 + 1/2 and 1, of an exponential off by two steps at most
    z, index, teacher, weight = make(4, V, 6, torch.float32, 14, holes=False)
    twice, merged, both = index.clone(), index.clone(), teacher.clone()
    twice[:, 1] = index[:, 0]
    merged[:, 1] = -1
    both[:, 0] = torch.logsumexp(teacher[:, :2].double(), 1).float()
    a, b = (ctx.distill(z.cuda(), i.cuda(), t.cuda(), 1.0, weight.cuda()) for i, t in ((twice, teacher), (merged, both)))
    lp = torch.log_softmax(teacher.double(), 1)
    own = (lp[:, :2].exp() * lp[:, :2]).sum(1) - torch.logsumexp(lp[:, :2], 1).exp() * torch.logsumexp(lp[:, :2], 1)
    # logarithms up to 40 in float32, exponents and the merged teacher's rounding of 2^-24 of up to 40
    rel = 2.0 ** -24 * (32 + 4 * 40)
    check(a[0], b[0].double().cpu() + own, torch.full((4,), 40 * rel, dtype=torch.float64), "loss")
    check(a[2], b[2].double().cpu(), 2 * rel * weight.double()[:, None] * torch.ones(V), "dlogits")
