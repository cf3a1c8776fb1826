"""Checks of arguments of the operators on coded layers that need no GPU."""
import ctypes

import pytest

from paper_2312_07759_amd import binding


def desc(**kw):
    v = dict(words=16, rows=64, cols=256, C=16, k=16, d=1, S=None, group=0, dtype=binding.BF16)
    v.update(kw)
    return binding.IdkmCodesDesc(v["words"], v["rows"], v["cols"], v["C"], v["k"], v["d"], v["S"], v["group"], v["dtype"])


def sizes(n=100, **kw):
    lib = binding.load_library()
    d = desc(**kw)
    return lib.idkm_codes_linear_workspace(ctypes.byref(d), n), lib.idkm_codes_linear_backward_workspace(ctypes.byref(d), n)


def test_workspace_sizes():
    lib = binding.load_library()
    assert sizes(0) == (0, 0) and sizes(1)[0] == 0
    for n in (1, 17, 300, 5000):
        for kw in ({}, {"S": 16, "group": 64}, {"dtype": binding.F32}, {"k": 1000, "d": 4}, {"d": 8, "k": 256}, {"rows": 1, "cols": 1}):
            a, b = sizes(n, **kw)
            assert a >= 0 and b > 0 and a % 16 == 0 and b % 16 == 0
    # a layer's panel is bounded: the workspace does not grow with the layer without end
    a, _ = sizes(64, rows=128_000, cols=16_384)
    assert 0 <= a < 2 ** 31
    assert lib.idkm_distill_workspace(0, 10, 1, 0) == 0
    assert lib.idkm_distill_workspace(1, 100_000, 64, 2) > 0 and lib.idkm_distill_workspace(2048, 128_000, 64, 2) == 0


@pytest.mark.parametrize("bad", [dict(words=None), dict(C=None), dict(dtype=3), dict(dtype=-1), dict(rows=0), dict(cols=0), dict(k=0), dict(k=1025),
                                 dict(d=0), dict(d=65), dict(d=3), dict(S=16, group=0), dict(S=16, group=33), dict(S=18, group=64),
                                 dict(S=16, group=32, d=64), dict(C=17), dict(words=18), dict(rows=4_000_001), dict(rows=4_000_000, cols=32_768)])
def test_layers_that_are_refused(bad):
    assert sizes(5, **bad) == (-1, -1)


def test_other_refused_sizes():
    lib = binding.load_library()
    assert sizes(-1) == (-1, -1) and sizes(4_000_001) == (-1, -1)
    assert lib.idkm_codes_linear_workspace(None, 1) == -1
    for n, V, top, dtype in ((-1, 10, 1, 0), (1, 0, 1, 0), (1, 10, 0, 0), (1, 10, 1025, 0), (1, 10, 1, 3), (1, 2 ** 29 + 1, 1, 0)):
        assert lib.idkm_distill_workspace(n, V, top, dtype) == -1
    d = desc()
    assert lib.idkm_codes_linear(None, ctypes.byref(d), None, 1, 256, None, 64, None, 0, None) == 1
    assert lib.idkm_codes_linear_backward(None, ctypes.byref(d), None, 256, None, 64, 1, None, 256, None, None, None, 0, None) == 1
    assert lib.idkm_group_scale(None, None, 1, 1, 1, None, None, None) == 1
    assert lib.idkm_distill(None, None, 1, 1, 1, 0, None, None, 1, 1.0, None, None, None, None, 1, None, 0, None) == 1


def test_captured_backward_passes_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2312_07759_amd import autograd
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for function in (autograd._CodesProduct, autograd._Distill):
        with pytest.raises(RuntimeError, match="captured"):
            function.backward(None, torch.zeros(1))
