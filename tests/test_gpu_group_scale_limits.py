"""Rows too long for the group scales' 32-bit places, which begin anew 64 weights on: refused before a pointer is looked at."""
import pytest

from paper_2312_07759_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,fits", [(1, 2 ** 31 - 64, True), (1, 2 ** 31 - 63, False), (1, 2 ** 31 - 1, False), (32, 2 ** 31 - 1, False),
                                            (0, 2 ** 31 - 63, False), (32, 2 ** 31 - 64, True), (33, 2 ** 31 - 64, False)])
def test_longest_rows(rows, cols, fits):
    ctx = binding.Context(0)
    lib, said = ctx._lib, b"non-NULL" if fits else b"too large"
    calls = {"idkm_group_scale": 3, "idkm_group_unscale": 3, "idkm_group_unscale_backward": 5, "idkm_group_scale_backward": 5}
    for group in (cols, 128):
        for name, pointers in calls.items():
            args = [rows, cols, group]
            before = {"idkm_group_scale": 1, "idkm_group_unscale": 2, "idkm_group_unscale_backward": 3, "idkm_group_scale_backward": 4}[name]
            status = getattr(lib, name)(ctx._h, *[None] * before, *args, *[None] * (pointers - before), None)
            assert status == 1 and said in lib.idkm_last_error(ctx._h), (name, group)
    ctx.close()
