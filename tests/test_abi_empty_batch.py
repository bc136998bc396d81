"""The grouped FFN on 8-bit rows with no rows, without a GPU: the arrays of a
batch of no tokens have no addresses, and nothing is enqueued."""

import ctypes
import os

import pytest

B = pytest.importorskip("paper_2601_17111_amd.binding")

P = ctypes.c_void_p
A, Z = P(1 << 20), None  # an aligned stand-in that is never read, and null


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libllep.so not built")
    return B.lib()


@pytest.mark.parametrize("name", ["llep_grouped_ffn_int8", "llep_grouped_ffn_int8_f32"])
def test_no_rows(L, name):
    p = B.make_params(T=0, K=2, E=8, P=4, capacity=1)
    bufs = B.llep_plan_buffers(*([8] * 10))
    a = dict(p=ctypes.byref(p), b=ctypes.byref(bufs), device=-1, x=A, xs=A, rp=A, gu=A, gs=A, us=A,
             dn=A, ds=A, D=64, F=64, out=A, ws=A, wsb=1 << 30, stream=Z)
    for none in ([], ["xs"], ["x"], ["out"], ["rp"], ["x", "xs", "rp", "out"]):
        assert getattr(L, name)(*{**a, **{k: Z for k in none}}.values()) == B.LLEP_OK, none
    # weights and scales are asked for all the same
    for k in ("gu", "gs", "us", "dn", "ds"):
        assert getattr(L, name)(*{**a, k: Z}.values()) == B.LLEP_E_ARG, k
