"""Products with coded layers and their gradients over seeded shapes of the whole range of codebooks, groups, types and token counts."""
import random

import pytest

from layer_cases import DTYPES, Layer, draw
from test_gpu_codes_linear import ctx, run_gradient, run_product  # noqa: F401

pytestmark = pytest.mark.gpu


def shape(seed):
    r = random.Random(seed)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))  # noqa: E731
    d = r.choice([1, 1, 1, 2, 2, 4, 4, 8, 8, 3, 16, 64])
    k = r.choice([2, 3, 4, 7, 8, 16, 30, 64, 100, 128, 200, 256, 300, 1024])
    cols = max(1, log(1, 3000) // d) * d
    groups = [0, cols, cols + 5] + [g for g in (32, 64, 96, 128, 160, 256, 384) if g < cols and g % d == 0]
    return log(1, 1200), cols, k, d, r.choice(groups), r.choice(sorted(DTYPES)), sorted({log(1, 20), log(1, 200), log(10, 1500)})


@pytest.mark.parametrize("seed", range(60))
def test_shape(ctx, seed):  # noqa: F811
    rows, cols, k, d, group, dtype, tokens = shape(seed)
    layer = Layer(rows, cols, k, d, group, DTYPES[dtype], seed=seed)
    for n in tokens:
        run_product(ctx, layer, draw((n, cols), DTYPES[dtype], n))
    run_gradient(ctx, layer, tokens[seed % len(tokens)], seed)
