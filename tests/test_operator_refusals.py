"""The adapters', clipping's and Adam's entry points refuse bad calls before any device work (no GPU needed)."""
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


@pytest.mark.parametrize("args,word", [
    ((0, 8, 2, 2, 0, 4), b"in or out"), ((8, 1 << 27, 2, 2, 0, 4), b"in or out"), ((8, 8, 0, 2, 0, 4), b"rank"),
    ((8, 8, 65, 2, 0, 4), b"rank"), ((8, 8, 2, 0, 0, 4), b"n_adapters"), ((8, 8, 2, 4097, 0, 4), b"n_adapters"),
    ((8, 8, 2, 2, 7, 4), b"precision"), ((8, 8, 2, 2, 0, 0), b"max_rows"), ((8, 8, 2, 2, 0, (1 << 20) + 1), b"max_rows")])
def test_adapters_create(lib, args, word):
    h = C.c_void_p(1)
    assert lib.adapters_create(C.byref(h), *args) == _abi.OT_E_INVAL
    assert word in lib.ot_last_error() and h.value is None


def test_null_objects(lib):
    assert lib.adapters_create(None, 8, 8, 2, 2, 0, 4) == _abi.OT_E_INVAL
    assert lib.adapters_forward(None, None, 0, None, 0, None, None, 0, None, 0, None, None, 1, None, 0, 0, None, 0, 0,
                                None) == _abi.OT_E_INVAL
    assert lib.adapters_backward(None, None, 0, None, 0, None, 0, None, 0, None, None, 1, None, 0, None, 0, None, 0,
                                 None, 0, None, 0, 0, None) == _abi.OT_E_INVAL
    assert lib.clip_norm(None, None, None) == _abi.OT_E_INVAL
    assert lib.clip_apply(None, 1.0, None, None) == _abi.OT_E_INVAL
    assert lib.adam_step(None, 1.0, None, None) == _abi.OT_E_INVAL
    assert lib.adam_set_lr(None, 1.0) == _abi.OT_E_INVAL
    assert lib.adam_get_steps(None, None) == _abi.OT_E_INVAL
    assert lib.adam_set_steps(None, 1) == _abi.OT_E_INVAL
    for f in (lib.adapters_destroy, lib.clip_destroy, lib.adam_destroy):
        assert f(None) == _abi.OT_OK


def arr(*values):
    return (C.c_void_p * len(values))(*values)


def test_clip_create(lib):
    h = C.c_void_p(1)
    one, big = (C.c_int64 * 1)(5), (C.c_int64 * 2)(1 << 40, 1)
    assert lib.clip_create(None, 1, arr(64), None, one, None) == _abi.OT_E_INVAL
    for n in (0, -1, 65537):
        assert lib.clip_create(C.byref(h), n, arr(64), None, one, None) == _abi.OT_E_INVAL
    assert lib.clip_create(C.byref(h), 1, None, None, one, None) == _abi.OT_E_INVAL
    assert lib.clip_create(C.byref(h), 1, arr(64), None, None, None) == _abi.OT_E_INVAL
    assert lib.clip_create(C.byref(h), 1, arr(None), None, one, None) == _abi.OT_E_INVAL
    assert lib.clip_create(C.byref(h), 1, arr(66), None, one, None) == _abi.OT_E_INVAL           # fp32 at 2 mod 4
    assert lib.clip_create(C.byref(h), 1, arr(64), arr(None), one, None) == _abi.OT_E_INVAL
    assert lib.clip_create(C.byref(h), 1, arr(64), None, (C.c_int64 * 1)(-1), None) == _abi.OT_E_INVAL
    assert lib.clip_create(C.byref(h), 2, arr(64, 64), None, big, None) == _abi.OT_E_INVAL
    assert b"2^40" in lib.ot_last_error()
    assert lib.clip_create(C.byref(h), 1, arr(64), None, one, (C.c_int32 * 1)(3)) == _abi.OT_E_INVAL
    assert b"types[0]" in lib.ot_last_error() and h.value is None


def test_adam_create(lib):
    h = C.c_void_p(1)
    one = (C.c_int64 * 1)(5)
    ok = [arr(64), arr(64), arr(64), arr(64), None, one, 1e-3, 0.9, 0.999, 1e-8, 0]
    for i, bad in ((0, None), (1, None), (2, None), (3, None), (5, None), (0, arr(None)), (3, arr(65)), (4, arr(65)),
                   (6, float("nan")), (7, 1.0), (7, -0.5), (8, float("nan")), (9, -1e-8), (10, -1)):
        args = list(ok)
        args[i] = bad
        assert lib.adam_create(C.byref(h), 1, *args) == _abi.OT_E_INVAL, i
    assert h.value is None
