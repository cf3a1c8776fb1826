"""Checks of arguments of lookups, inputs kept in 8 bits and products in 8-bit integers that need no GPU."""
import ctypes

import pytest

from paper_2312_07759_amd import binding


def codes(**kw):
    v = dict(words=16, rows=64, cols=256, C=16, k=16, d=1, S=None, group=0, dtype=binding.BF16)
    v.update(kw)
    return binding.IdkmCodesDesc(v["words"], v["rows"], v["cols"], v["C"], v["k"], v["d"], v["S"], v["group"], v["dtype"])


def int8(**kw):
    v = dict(W8=16, rows=64, cols=200, ldw=256, scale=16, dtype=binding.BF16)
    v.update(kw)
    return binding.IdkmInt8Desc(v["W8"], v["rows"], v["cols"], v["ldw"], v["scale"], v["dtype"])


def test_workspace_sizes():
    lib = binding.load_library()
    for kw in ({}, {"S": 16, "group": 64}, {"S": 16, "group": 96}, {"dtype": binding.F32}, {"k": 1000, "d": 4}, {"k": 256, "d": 4}, {"rows": 1, "cols": 1}):
        w = codes(**kw)
        assert lib.idkm_codes_embedding_backward_workspace(ctypes.byref(w), 0) == 0
        for n in (1, 256, 257, 512, 513, 16384, 16385, 4_000_000):
            b = lib.idkm_codes_embedding_backward_workspace(ctypes.byref(w), n)
            assert b > 0 and b % 256 == 0
    # the sums of rows are as many as there are rows, not tokens
    small = lib.idkm_codes_embedding_backward_workspace(ctypes.byref(codes(k=256, d=4)), 4_000_000)
    assert small < 4_000_000 * 24 + 2 ** 30
    assert lib.idkm_embedding_backward_workspace(1000, 64, 0) == 0 and lib.idkm_embedding_backward_workspace(1000, 64, 512) == 0
    assert lib.idkm_embedding_backward_workspace(1000, 64, 513) > 0
    for n in (1, 4, 5, 64, 65, 4096):
        f, b = (getattr(lib, name)(ctypes.byref(int8()), n) for name in ("idkm_int8_linear_workspace", "idkm_int8_linear_backward_workspace"))
        assert f >= 0 and b > 0 and f % 16 == 0 and b % 16 == 0
    assert lib.idkm_int8_linear_workspace(ctypes.byref(int8()), 0) == 0 and lib.idkm_int8_linear_workspace(ctypes.byref(int8()), 1) == 0


@pytest.mark.parametrize("bad", [dict(words=None), dict(C=None), dict(dtype=3), dict(rows=0), dict(cols=0), dict(k=0), dict(k=1025), dict(d=65), dict(d=3),
                                 dict(S=16, group=0), dict(S=16, group=33), dict(rows=4_000_001)])
def test_tables_that_are_refused(bad):
    assert binding.load_library().idkm_codes_embedding_backward_workspace(ctypes.byref(codes(**bad)), 5) == -1


@pytest.mark.parametrize("bad", [dict(W8=None), dict(scale=None), dict(W8=17), dict(scale=18), dict(rows=0), dict(cols=0), dict(ldw=199), dict(ldw=200), dict(ldw=240),
                                 dict(dtype=3), dict(dtype=-1), dict(rows=4_000_001), dict(cols=131_073, ldw=131_200)])
def test_layers_of_integers_that_are_refused(bad):
    lib = binding.load_library()
    assert lib.idkm_int8_linear_workspace(ctypes.byref(int8(**bad)), 5) == -1
    assert lib.idkm_int8_linear_backward_workspace(ctypes.byref(int8(**bad)), 5) == -1


def test_other_refused_sizes():
    lib = binding.load_library()
    for n in (-1, 4_000_001):
        assert lib.idkm_codes_embedding_backward_workspace(ctypes.byref(codes()), n) == -1
        assert lib.idkm_int8_linear_workspace(ctypes.byref(int8()), n) == -1
        assert lib.idkm_embedding_backward_workspace(10, 10, n) == -1
    for rows, cols in ((0, 1), (1, 0), (4_000_001, 1), (1, 4_000_001), (4_000_000, 32_768)):
        assert lib.idkm_embedding_backward_workspace(rows, cols, 1) == -1
    for name in ("idkm_codes_embedding_backward_workspace", "idkm_int8_linear_workspace", "idkm_int8_linear_backward_workspace"):
        assert getattr(lib, name)(None, 1) == -1
    w, q = ctypes.byref(codes()), ctypes.byref(int8())
    assert lib.idkm_embedding(None, None, 1, 1, None, 4, 1, 1.0, None, 1, 0, None) == 1
    assert lib.idkm_embedding_backward(None, 1, 1, None, 4, 1, 1.0, None, 1, 0, None, None, 0, None) == 1
    assert lib.idkm_codes_embedding(None, w, None, 4, 1, 1.0, None, 256, None) == 1
    assert lib.idkm_codes_embedding_backward(None, w, None, 4, 1, 1.0, None, 256, None, None, None, 0, None) == 1
    assert lib.idkm_keep8(None, None, 1, 1, 1, 0, None, None, None) == 1
    assert lib.idkm_restore8(None, None, None, 1, 1, 0, None, 1, None) == 1
    assert lib.idkm_codes_linear_backward_kept(None, w, None, None, None, 64, 1, None, 256, None, None, None, 0, None) == 1
    assert lib.idkm_int8_rows(None, None, 1, 1, 1, 0, None, 16, None, None) == 1
    assert lib.idkm_int8_linear(None, q, None, 1, 200, None, 64, None, 0, None) == 1
    assert lib.idkm_int8_linear_backward(None, q, None, 64, 1, None, 200, None, 0, None) == 1


def test_captured_backward_passes_are_refused(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2312_07759_amd import autograd
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for function in (autograd._Embedding, autograd._CodesLookup, autograd._Int8Product):
        with pytest.raises(RuntimeError, match="captured"):
            function.backward(None, torch.zeros(1))
