"""Which form a product of a stored layer takes, as its workspace tells (a layer that is written out needs room for it): no GPU needed."""
import pytest

from paper_2312_07759_amd import binding
from test_layers_abi import sizes


@pytest.mark.parametrize("k,group,n,written", [
    (16, 0, 256, False), (16, 128, 256, False), (256, 128, 256, False),   # 24 us from the codes and 39 written out; 24 and 35
    (256, 32, 256, True), (64, 32, 256, True),                            # 58 and 38: a lookup for every weight, a scale for every 32
    (16, 128, 700, True), (256, 128, 700, True), (16, 0, 2048, True),     # 61 and 53, 64 and 53
    (16, 64, 512, True), (16, 32, 64, False), (256, 32, 64, False),       # 70 and 46; 19 and 30, 22 and 27
])
def test_form_by_measured_times(k, group, n, written):
    """4096 x 4096 in bfloat16; the times are those of calls captured into a graph."""
    need = sizes(n, rows=4096, cols=4096, k=k, S=16 if group else None, group=group, dtype=binding.BF16)[0]
    assert (need >= 4096 * 4096 * 2) == written
