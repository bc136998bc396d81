"""llep_route and llep_route_backward without a GPU: parameters and arguments that
do not fit are refused on the host, before anything is enqueued."""

import ctypes
import math
import os

import pytest

B = pytest.importorskip("paper_2601_17111_amd.binding")

BF16, F32 = B.LLEP_BF16, B.LLEP_F32


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libllep.so not built")
    return B.lib()


def _params(**kw):
    d = dict(T=16, K=4, E=64, groups=8, top_groups=4)
    d.update(kw)
    return B.make_route(**d)


def _both(p, dtype=F32):
    """The error codes of both calls, with addresses that are never followed."""
    L, a = _lib(), ctypes.c_void_p(4096)
    return (L.llep_route(ctypes.byref(p), dtype, a, a, a, a, None),
            L.llep_route_backward(ctypes.byref(p), dtype, a, a, a, a, a, None))


def test_struct_layout():
    assert ctypes.sizeof(B.llep_route_params) == 40
    assert B.llep_route_params.E.offset == 12 and B.llep_route_params.scale.offset == 36


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(K=0), dict(K=65), dict(E=0, groups=1, top_groups=1), dict(E=513, groups=1, top_groups=1),
    dict(T=2 ** 29 + 1), dict(T=2 ** 31, K=1), dict(groups=0), dict(groups=65), dict(groups=7),
    dict(top_groups=0), dict(top_groups=9), dict(K=33), dict(K=5, E=64, groups=64, top_groups=4),
    dict(K=20, E=16, groups=1, top_groups=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
    dict(scale=math.inf),
])
def test_bad_params(bad):
    assert _both(_params(**bad)) == (B.LLEP_E_ARG, B.LLEP_E_ARG)
    assert B.last_error()


def test_bad_enumerations():
    for field, value in (("score", 2), ("score", -1), ("group_score", 2), ("renormalize", 2)):
        p = _params()
        setattr(p, field, value)
        assert _both(p) == (B.LLEP_E_ARG, B.LLEP_E_ARG), field
    assert _both(_params(), 7) == (B.LLEP_E_DTYPE, B.LLEP_E_DTYPE)
    with pytest.raises(ValueError):
        B.make_route(1, 1, 1, score="relu")
    with pytest.raises(ValueError):
        B.make_route(1, 1, 1, group_score="sum")


def test_pointers():
    L, a, p = _lib(), ctypes.c_void_p(4096), _params()
    r = ctypes.byref(p)
    assert L.llep_route(None, F32, a, a, a, a, None) == B.LLEP_E_ARG
    for i in (0, 2, 3):  # (the bias may be null)
        args = [a] * 4
        args[i] = None
        assert L.llep_route(r, F32, *args, None) == B.LLEP_E_ARG
    for i in range(4):
        args = [a] * 4
        args[i] = ctypes.c_void_p(4098)
        assert L.llep_route(r, F32, *args, None) == B.LLEP_E_ARG
    assert L.llep_route(r, BF16, ctypes.c_void_p(4097), a, a, a, None) == B.LLEP_E_ARG
    for i in range(1, 5):
        args = [a] * 5
        args[i] = None
        assert L.llep_route_backward(r, F32, *args, None) == B.LLEP_E_ARG
    for i in range(5):
        args = [a] * 5
        args[i] = ctypes.c_void_p(4098)
        assert L.llep_route_backward(r, F32, *args, None) == B.LLEP_E_ARG
    # logits may be null only where they are not read
    for kw in (dict(renormalize=False), dict(score="sigmoid")):
        p = _params(**kw)
        assert L.llep_route_backward(ctypes.byref(p), F32, None, a, a, a, a, None) == B.LLEP_E_ARG


def test_no_tokens_need_no_addresses():
    L, p = _lib(), _params(T=0)
    assert L.llep_route(ctypes.byref(p), F32, None, None, None, None, None) == B.LLEP_OK
    assert L.llep_route_backward(ctypes.byref(p), F32, None, None, None, None, None, None) == B.LLEP_OK
