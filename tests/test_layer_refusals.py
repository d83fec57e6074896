"""The layers' entry points refuse bad calls before any device work (no GPU needed)."""
import ctypes as C

import pytest

from paper_2309_16743_amd import _abi


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(_abi.LIB_PATH):
        from paper_2309_16743_amd.build import build
        build()
    return _abi.load()


BIG = (1 << 26) + 1


@pytest.mark.parametrize("args,word", [
    ((0, 8, 0, 0, 4), b"in or out"), ((8, BIG, 0, 0, 4), b"in or out"), ((1 << 26, 1 << 11, 0, 0, 4), b"2^36"),
    ((8, 8, 2, 0, 4), b"precision"), ((8, 8, 0, 4, 4), b"activation"), ((8, 8, 0, -1, 4), b"activation"),
    ((8, 8, 0, 0, -1), b"max_rows"), ((8, 8, 0, 0, BIG), b"max_rows"), ((2048, 8, 0, 0, 1 << 26), b"2^36")])
def test_dense_create(lib, args, word):
    h = C.c_void_p(1)
    assert lib.dense_create(C.byref(h), *args) == _abi.OT_E_INVAL
    assert word in lib.ot_last_error() and h.value is None


@pytest.mark.parametrize("args,word", [
    ((0, 1, 1, 0, 0, 1e-5, 4), b"channels"), ((65537, 1, 1, 0, 0, 1e-5, 4), b"channels"),
    ((8, 0, 1, 0, 0, 1e-5, 4), b"groups"), ((8, 3, 1, 0, 0, 1e-5, 4), b"groups"), ((8, 16, 1, 0, 0, 1e-5, 4), b"groups"),
    ((8, 2, 0, 0, 0, 1e-5, 4), b"positions"), ((8, 2, BIG, 0, 0, 1e-5, 4), b"positions"),
    ((8, 2, 1, 5, 0, 1e-5, 4), b"precision"), ((8, 2, 1, 0, 9, 1e-5, 4), b"activation"),
    ((8, 2, 1, 0, 0, 0.0, 4), b"eps"), ((8, 2, 1, 0, 0, -1.0, 4), b"eps"), ((8, 2, 1, 0, 0, float("nan"), 4), b"eps"),
    ((8, 2, 1, 0, 0, float("inf"), 4), b"eps"), ((8, 2, 1, 0, 0, 1e-5, -1), b"max_samples"),
    ((8, 2, 1, 0, 0, 1e-5, BIG), b"max_samples"), ((2048, 2, 1 << 26, 0, 0, 1e-5, 0), b"2^36"),
    ((8, 2, 1 << 20, 0, 0, 1e-5, 1 << 14), b"2^36")])
def test_norm_create(lib, args, word):
    h = C.c_void_p(1)
    assert lib.norm_create(C.byref(h), *args) == _abi.OT_E_INVAL
    assert word in lib.ot_last_error() and h.value is None


@pytest.mark.parametrize("args,word", [
    ((-0.1, 1, 0, 0), b"p outside"), ((1.1, 1, 0, 0), b"p outside"), ((float("nan"), 1, 0, 0), b"p outside"),
    ((0.5, 1, 0, 3), b"precision")])
def test_dropout_create(lib, args, word):
    h = C.c_void_p(1)
    assert lib.dropout_create(C.byref(h), *args) == _abi.OT_E_INVAL
    assert word in lib.ot_last_error() and h.value is None


def test_null_objects(lib):
    e = _abi.OT_E_INVAL
    assert lib.dense_create(None, 8, 8, 0, 0, 4) == e
    assert lib.norm_create(None, 8, 2, 1, 0, 0, 1e-5, 4) == e
    assert lib.dropout_create(None, 0.5, 1, 0, 0) == e
    assert lib.dense_forward(None, None, 0, None, 0, None, None, 0, 1, None, 0, 0, None, 0, None) == e
    assert lib.dense_backward(None, None, 0, None, 0, 1, None, 0, None, 0, None, 0, None, 0, None, None) == e
    assert lib.norm_forward(None, None, 0, None, None, 1, None, 0, None, None) == e
    assert lib.norm_backward(None, None, 0, None, None, 1, None, None, 0, None, 0, None, None, None) == e
    assert lib.dropout_forward(None, None, 0, None, 0, 1, 1, None, 0, 0, None, None) == e
    assert lib.dropout_backward(None, None, 0, 1, 1, None, 0, 0, None, None) == e
    for f in (lib.dense_destroy, lib.norm_destroy, lib.dropout_destroy):
        assert f(None) == _abi.OT_OK
