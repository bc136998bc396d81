"""The 4-bit calls without a GPU: sizes, and arguments that are refused on the host
before anything is enqueued."""

import ctypes
import os

import pytest

B = pytest.importorskip("paper_2601_17111_amd.binding")

BF16, F32 = B.LLEP_BF16, B.LLEP_F32
A, NEAR, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4104), ctypes.c_void_p(4097)


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libllep.so not built")
    return B.lib()


def test_sizes():
    L = _lib()
    for D, q, s in ((1, 64, 16), (128, 64, 16), (129, 128, 16), (512, 256, 16), (513, 320, 32),
                    (2880, 1472, 96), (65536, 32768, 2048)):
        assert (B.llep_mxfp4_row_bytes(D), B.llep_mxfp4_scale_bytes(D)) == (q, s)
    for D in list(range(1, 1200)) + [65535, 65536]:
        assert B._mxfp4_bytes(D) == (L.llep_mxfp4_row_bytes(D), L.llep_mxfp4_scale_bytes(D))
    for D in (0, -1, 65537):
        assert L.llep_mxfp4_row_bytes(D) == L.llep_mxfp4_scale_bytes(D) == -1
        with pytest.raises(B.LLEPError):
            B._mxfp4_bytes(D)
    assert L.llep_packed_mxfp4_bytes(3, 17, 129) == 3 * 32 * (128 + 16)
    assert L.llep_packed_mxfp4_bytes(512, 1 << 20, 65536) == 512 * (1 << 20) * (32768 + 2048)
    for bad in ((0, 16, 64), (513, 16, 64), (1, 0, 64), (1, (1 << 20) + 1, 64), (1, 16, 0), (1, 16, 65537)):
        assert L.llep_packed_mxfp4_bytes(*bad) == 0


@pytest.mark.parametrize("name", ["llep_quantize_rows_mxfp4", "llep_dequantize_rows_mxfp4"])
def test_rows(name):
    f = getattr(_lib(), name)

    def call(R=4, D=100, dtype=F32, x=A, q=A, q_pitch=64, s=A, s_pitch=16):
        return f(R, D, dtype, x, q, q_pitch, s, s_pitch, None) if "_quan" in name else \
            f(R, D, dtype, q, q_pitch, s, s_pitch, x, None)
    assert call(dtype=7) == B.LLEP_E_DTYPE
    for bad in (dict(R=-1), dict(D=0), dict(D=65537), dict(q_pitch=48), dict(q_pitch=72),
                dict(q_pitch=65552), dict(s_pitch=0), dict(s_pitch=24), dict(s_pitch=65552), dict(x=None),
                dict(q=None), dict(s=None), dict(q=NEAR), dict(s=NEAR), dict(x=ODD),
                dict(dtype=F32, x=ctypes.c_void_p(4098))):
        assert call(**bad) == B.LLEP_E_ARG, bad
    assert call(R=0, x=None, q=None, s=None) == B.LLEP_OK


def test_pack():
    L = _lib()

    def call(E=2, N=64, K=100, w=A, s=A, wu=None, su=None, w_bytes=50, s_bytes=4, out=A):
        return L.llep_pack_mxfp4(E, N, K, w, s, wu, su, w_bytes, s_bytes, out, None)
    for bad in (dict(E=0), dict(E=513), dict(N=0), dict(K=0), dict(w_bytes=49), dict(s_bytes=3), dict(w=None),
                dict(s=None), dict(out=None), dict(out=NEAR), dict(wu=A), dict(su=A),
                dict(N=48, wu=A, su=A), dict(N=65536 + 32, wu=A, su=A)):
        assert call(**bad) == B.LLEP_E_ARG, bad


def test_matmul():
    L = _lib()

    def call(M=4, N=48, K=100, x=A, q_pitch=64, s=A, s_pitch=16, w=A, dtype=F32, out=A):
        return L.llep_mxfp4_matmul(M, N, K, x, q_pitch, s, s_pitch, w, dtype, out, None)
    assert call(dtype=7) == B.LLEP_E_DTYPE
    for bad in (dict(M=-1), dict(M=0x7fffff01), dict(N=0), dict(N=(1 << 20) + 1), dict(K=0), dict(K=65537),
                dict(q_pitch=48), dict(s_pitch=8), dict(x=None), dict(s=None), dict(w=None), dict(out=None),
                dict(x=NEAR), dict(s=NEAR), dict(w=NEAR), dict(out=NEAR)):
        assert call(**bad) == B.LLEP_E_ARG, bad
    assert call(M=0, x=None, s=None, out=None) == B.LLEP_OK


def test_grouped_ffn():
    L = _lib()
    p = B.make_params(T=16, K=2, E=8, P=4, capacity=16)
    bufs = B.llep_plan_buffers(*[16 * (i + 1) for i in range(10)])
    need = B.llep_grouped_ffn_mxfp4_workspace_bytes(p, 128)
    assert need >= 32 * (64 + 16)
    assert B.llep_grouped_ffn_mxfp4_workspace_bytes(p, 0) == 0
    ws = ctypes.c_void_p(1 << 20)

    def call(device=-1, x=A, gu=A, dn=A, D=64, F=128, dtype=BF16, out=A, ws=ws, nbytes=need, plan=bufs):
        return L.llep_grouped_ffn_mxfp4(ctypes.byref(p), ctypes.byref(plan), device, x, gu, dn, D, F, dtype,
                                        out, ws, nbytes, None)
    assert call(dtype=5) == B.LLEP_E_DTYPE
    for bad in (dict(device=-2), dict(device=4), dict(x=None), dict(gu=None), dict(dn=None), dict(out=None),
                dict(D=96), dict(F=100), dict(D=0), dict(F=65600), dict(x=NEAR), dict(gu=NEAR), dict(dn=NEAR),
                dict(out=NEAR), dict(plan=B.llep_plan_buffers(*([0] * 10)))):
        assert call(**bad) == B.LLEP_E_ARG, bad
    for bad in (dict(ws=None), dict(nbytes=need - 1), dict(ws=ctypes.c_void_p((1 << 20) + 128))):
        assert call(**bad) == B.LLEP_E_WORKSPACE, bad
