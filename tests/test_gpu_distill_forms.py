"""The loss against a teacher where several workgroups share a row, and where a row is longer than its workgroup's registers: masks,
repeated places, lists that are none, rows in place, graphs."""
import pytest

import test_gpu_distill as base
from layer_cases import DTYPES
from test_gpu_distill import ctx  # noqa: F401

pytestmark = pytest.mark.gpu

SHARED, LONG = [(6, 40000), (127, 33001)], [(256, 70001), (130, 140003)]


@pytest.mark.parametrize("n,V", SHARED + LONG)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_masks_and_extremes(ctx, n, V, dtype):  # noqa: F811
    base.test_masks_and_extremes(ctx, n, V, dtype)


@pytest.mark.parametrize("n,V", SHARED + LONG)
def test_repeated_indices_add_up(ctx, n, V):  # noqa: F811
    base.test_repeated_indices_add_up(ctx, n, V)


@pytest.mark.parametrize("n,V", SHARED + LONG)
def test_lists_that_are_none(ctx, n, V):  # noqa: F811
    base.test_lists_that_are_none(ctx, n, V)


@pytest.mark.parametrize("n,V", SHARED + LONG + [(128, 32769), (5, 32768), (5, 32769)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_in_place_and_strides(ctx, n, V, dtype):  # noqa: F811
    base.test_in_place_and_strides(ctx, n, V, dtype)


@pytest.mark.parametrize("n,V,top", [(1, 32768, 4), (127, 32769, 8), (128, 32769, 8), (40, 65537, 3), (1, 500_001, 16)])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_loss_and_gradient(ctx, n, V, top, dtype):  # noqa: F811
    base.test_loss_and_gradient(ctx, n, V, top, dtype)


@pytest.mark.parametrize("n,V", [(9, 50001), (200, 70001)])
def test_captured_graph(ctx, n, V):  # noqa: F811
    base.test_captured_graph(ctx, n, V)
