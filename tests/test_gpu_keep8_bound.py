"""How far inputs kept in 8 bits are off: the bound that the header states, which blocks reach."""
import pytest
import torch

from layer_cases import DTYPES
from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def errors(ctx, X):
    """Largest error and largest size of each block, float64."""
    off = (ctx.restore8(ctx.keep8(X.cuda())).cpu().double() - X.double()).abs()
    return off.view(-1, 32).amax(1), X.double().abs().view(-1, 32).amax(1)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_relative_to_the_largest(ctx, dtype):
    """Half a step, 1 / 127.5 of the block's largest size, at every significand of the largest (bfloat16's 128, where they change the step) and
    many smaller numbers."""
    lead = (128 + torch.arange(128)) / 128.0
    for power in (0, -9, 9):
        size = lead * 2.0 ** power
        rest = torch.linspace(-1, 1, 31)[None, :] * size[:, None]
        rest[:, 0] = size / lead * 0.4921875  # 31.5 or 15.75 steps
        rest[:, 1] = size / lead * 1.015625   # 32.5 of the larger steps
        X = torch.cat([size[:, None], rest], 1).to(DTYPES[dtype])
        off, largest = errors(ctx, X)
        assert bool((off <= largest / 127.5).all())
        assert float((off / largest).max()) > 1 / 128  # 2^e is 1/64 to 1/63.75 of the largest in the last blocks of a binade


def test_blocks_below_normal_numbers(ctx):
    """Float32 blocks below 2^-126 share e = -132, whatever their largest size."""
    tiny = torch.tensor([2.0 ** -127, 1.9 * 2.0 ** -127, 2.0 ** -130, 2.0 ** -133, 2.0 ** -140, 2.0 ** -149], dtype=torch.float32)
    X = torch.zeros(len(tiny), 32)
    X[:, 0], X[:, 5] = tiny, -tiny / 2
    off, largest = errors(ctx, X)
    assert bool((off <= 2.0 ** -133).all())
    assert not ctx.restore8(ctx.keep8(X.cuda()))[3:].any()  # 2^-133 is a tie, which goes to zero
    assert bool((ctx.keep8(X.cuda()).E == 1).all())
