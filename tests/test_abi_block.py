"""The calls around the block without a GPU: sizes, and arguments that are
rejected on the host before anything is enqueued (pointers are stand-ins that
are never read)."""

import ctypes

import pytest

B = pytest.importorskip("paper_2601_17111_amd.binding")

P = ctypes.c_void_p
A, Z = P(1 << 20), None  # an aligned stand-in, and null
ODD = P((1 << 20) + 1)


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libllep.so not built")
    return B.lib()


def test_sizes(L):
    assert [L.llep_int8_row_bytes(d) for d in (0, 1, 64, 65, 65536, 65537)] == \
        [-1, 64, 64, 128, 65536, -1]
    assert L.llep_packed_int8_bytes(1, 17, 65) == 32 * 128
    assert L.llep_packed_int8_bytes(4, 64, 64) == 4 * 64 * 64
    assert L.llep_packed_int8_bytes(0, 64, 64) == 0 and L.llep_packed_int8_bytes(1, 0, 64) == 0
    assert L.llep_packed_int8_bytes(1, 64, 65537) == 0
    assert L.llep_packed_int8_bytes(1, (1 << 20) + 1, 64) == 0
    assert L.llep_packed_int8_bytes(513, 64, 64) == 0
    assert L.llep_block_norm_backward_workspace_bytes(1, 8) == 64
    assert L.llep_block_norm_backward_workspace_bytes(0, 8) == 0
    assert L.llep_block_norm_backward_workspace_bytes(5, 8193) == 0
    assert L.llep_block_norm_backward_workspace_bytes(-1, 8) == 0
    # rows of column sums stop growing with the rows
    assert L.llep_block_norm_backward_workspace_bytes(1 << 30, 512) <= 1024 * 2 * 512 * 4
    assert L.llep_clip_gradients_workspace_bytes() > 0
    p = B.make_params(T=100, K=2, E=8, P=4, capacity=60)
    assert L.llep_grouped_ffn_int8_workspace_bytes(ctypes.byref(p), 64) >= 200 * 64 * 5
    assert L.llep_grouped_ffn_int8_workspace_bytes(ctypes.byref(p), 0) == 0


NORM = dict(T=4, D=64, dtype=B.LLEP_F32, x=A, b=A, gate=A, shape=B.LLEP_GATE_CHANNEL, w_post=A,
            w_pre=A, alpha=1.0, eps=1e-5, r=A, h=A, h_q=Z, h_scale=Z, q_bytes=0, stream=Z)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), B.LLEP_E_ARG), (dict(D=0), B.LLEP_E_ARG), (dict(D=8193), B.LLEP_E_ARG),
    (dict(dtype=7), B.LLEP_E_DTYPE), (dict(x=Z), B.LLEP_E_ARG), (dict(b=Z), B.LLEP_E_ARG),
    (dict(shape=4), B.LLEP_E_ARG), (dict(shape=-1), B.LLEP_E_ARG),
    (dict(gate=Z), B.LLEP_E_ARG), (dict(shape=B.LLEP_GATE_NONE), B.LLEP_E_ARG),
    (dict(eps=-1e-9), B.LLEP_E_ARG), (dict(eps=float("nan")), B.LLEP_E_ARG),
    (dict(w_pre=Z), B.LLEP_E_ARG), (dict(r=Z, h=Z), B.LLEP_E_ARG), (dict(r=ODD), B.LLEP_E_ARG),
    (dict(x=ODD), B.LLEP_E_ARG), (dict(w_post=ODD), B.LLEP_E_ARG),
    (dict(h_q=A), B.LLEP_E_ARG), (dict(h_scale=A), B.LLEP_E_ARG),
    (dict(h_q=A, h_scale=A, q_bytes=32), B.LLEP_E_ARG),
    (dict(h_q=A, h_scale=A, q_bytes=96), B.LLEP_E_ARG),
    (dict(h_q=ODD, h_scale=A, q_bytes=64), B.LLEP_E_ARG),
])
def test_norm_refusals(L, bad, code):
    assert L.llep_block_norm(*{**NORM, **bad}.values()) == code
    assert B.last_error()


BACK = dict(T=4, D=64, dtype=B.LLEP_F32, r=A, b=A, gate=A, shape=B.LLEP_GATE_CHANNEL, w_post=A,
            w_pre=A, alpha=1.0, eps=1e-5, d_r=A, d_h=A, dx=A, db=A, d_gate=A, dw_post=A, dw_pre=A,
            ws=A, ws_bytes=1 << 20, stream=Z)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), B.LLEP_E_ARG), (dict(D=8193), B.LLEP_E_ARG), (dict(dtype=-1), B.LLEP_E_DTYPE),
    (dict(r=Z), B.LLEP_E_ARG), (dict(d_r=Z), B.LLEP_E_ARG), (dict(dx=Z), B.LLEP_E_ARG),
    (dict(d_h=Z), B.LLEP_E_ARG), (dict(w_pre=Z), B.LLEP_E_ARG), (dict(dw_pre=Z), B.LLEP_E_ARG),
    (dict(dw_post=Z), B.LLEP_E_ARG), (dict(w_post=Z), B.LLEP_E_ARG), (dict(db=Z), B.LLEP_E_ARG),
    (dict(b=Z), B.LLEP_E_ARG), (dict(d_gate=Z), B.LLEP_E_ARG), (dict(gate=Z), B.LLEP_E_ARG),
    (dict(d_gate=ODD), B.LLEP_E_ARG), (dict(ws=Z), B.LLEP_E_WORKSPACE),
    (dict(ws_bytes=4 * 2 * 64 * 4 - 1), B.LLEP_E_WORKSPACE), (dict(ws=ODD), B.LLEP_E_WORKSPACE),
])
def test_norm_backward_refusals(L, bad, code):
    assert L.llep_block_norm_backward(*{**BACK, **bad}.values()) == code
    assert B.last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(R=-1), B.LLEP_E_ARG), (dict(D=0), B.LLEP_E_ARG), (dict(D=65537), B.LLEP_E_ARG),
    (dict(dtype=2), B.LLEP_E_DTYPE), (dict(x=Z), B.LLEP_E_ARG), (dict(q=Z), B.LLEP_E_ARG),
    (dict(scale=Z), B.LLEP_E_ARG), (dict(bytes=64), B.LLEP_E_ARG), (dict(bytes=100), B.LLEP_E_ARG),
    (dict(q=ODD), B.LLEP_E_ARG), (dict(x=ODD), B.LLEP_E_ARG),
])
def test_rows_refusals(L, bad, code):
    a = dict(R=3, D=100, dtype=B.LLEP_BF16, x=A, q=A, bytes=128, scale=A, stream=Z)
    assert L.llep_quantize_rows(*{**a, **bad}.values()) == code


@pytest.mark.parametrize("bad,code", [
    (dict(M=-1), B.LLEP_E_ARG), (dict(M=1 << 31), B.LLEP_E_ARG), (dict(N=0), B.LLEP_E_ARG),
    (dict(K=65537), B.LLEP_E_ARG), (dict(dtype=9), B.LLEP_E_DTYPE), (dict(x=Z), B.LLEP_E_ARG),
    (dict(bytes=64), B.LLEP_E_ARG), (dict(bytes=130), B.LLEP_E_ARG), (dict(w=Z), B.LLEP_E_ARG),
    (dict(w_scale=ODD), B.LLEP_E_ARG), (dict(x_scale=Z), B.LLEP_E_ARG), (dict(out=Z), B.LLEP_E_ARG),
    (dict(out=P((1 << 20) + 8)), B.LLEP_E_ARG), (dict(ws=P((1 << 20) + 16)), B.LLEP_E_WORKSPACE),
])
def test_product_refusals(L, bad, code):
    a = dict(M=3, N=40, K=100, x=A, bytes=128, x_scale=A, w=A, w_scale=A, dtype=B.LLEP_BF16, out=A,
             ws=A, ws_bytes=1 << 20, stream=Z)
    assert L.llep_int8_matmul(*{**a, **bad}.values()) == code


@pytest.mark.parametrize("bad", [
    dict(E=0), dict(N=0), dict(K=0), dict(E=513), dict(w=Z), dict(out=Z), dict(out=ODD),
    dict(N=40, up=A), dict(N=1 << 17, K=64, up=A),
])
def test_pack_refusals(L, bad):
    a = dict(E=2, N=64, K=100, w=A, up=Z, out=A, stream=Z)
    assert L.llep_pack_int8(*{**a, **bad}.values()) == B.LLEP_E_ARG


@pytest.mark.parametrize("bad,code", [
    (dict(device=4), B.LLEP_E_ARG), (dict(device=-2), B.LLEP_E_ARG), (dict(D=96), B.LLEP_E_ARG),
    (dict(F=0), B.LLEP_E_ARG), (dict(x=Z), B.LLEP_E_ARG), (dict(xs=Z), B.LLEP_E_ARG),
    (dict(gs=Z), B.LLEP_E_ARG), (dict(us=ODD), B.LLEP_E_ARG), (dict(out=Z), B.LLEP_E_ARG),
    (dict(rp=ODD), B.LLEP_E_ARG), (dict(ws=Z), B.LLEP_E_WORKSPACE),
    (dict(wsb=100), B.LLEP_E_WORKSPACE), (dict(ws=P((1 << 20) + 16)), B.LLEP_E_WORKSPACE),
])
def test_grouped_refusals(L, bad, code):
    p = B.make_params(T=100, K=2, E=8, P=4, capacity=60)
    bufs = B.llep_plan_buffers(*([8] * 10))
    a = dict(p=ctypes.byref(p), b=ctypes.byref(bufs), device=-1, x=A, xs=A, rp=A, gu=A, gs=A, us=A,
             dn=A, ds=A, D=64, F=64, out=A, ws=A, wsb=1 << 30, stream=Z)
    assert L.llep_grouped_ffn_int8(*{**a, **bad}.values()) == code


@pytest.mark.parametrize("entry,bad,code", [
    (dict(), dict(n=-1), B.LLEP_E_ARG), (dict(), dict(norm=Z), B.LLEP_E_ARG),
    (dict(), dict(ws=Z), B.LLEP_E_WORKSPACE), (dict(), dict(wsb=8), B.LLEP_E_WORKSPACE),
    (dict(), dict(ws=P((1 << 20) + 8)), B.LLEP_E_WORKSPACE),
    (dict(data=None), {}, B.LLEP_E_ARG), (dict(n=-1), {}, B.LLEP_E_ARG),
    (dict(dtype=5), {}, B.LLEP_E_DTYPE), (dict(reserved=1), {}, B.LLEP_E_ARG),
    (dict(data=(1 << 20) + 2), {}, B.LLEP_E_ARG),
])
def test_gradient_refusals(L, entry, bad, code):
    g = (B.llep_gradient * 1)(B.llep_gradient(**{**dict(data=1 << 20, out=1 << 20, n=8,
                                                        dtype=B.LLEP_F32, reserved=0), **entry}))
    a = dict(n=1, g=g, norm=A, ws=A, wsb=1 << 16, stream=Z)
    a.update(bad)
    assert L.llep_gradient_norm(*a.values()) == code
    assert L.llep_clip_gradients(a["n"], g, 1.0, a["norm"], a["ws"], a["wsb"], Z) == code
    if not entry and not bad:
        assert L.llep_clip_gradients(1, g, -1.0, A, A, 1 << 16, Z) == B.LLEP_E_ARG


def test_clip_needs_outputs_and_a_limit(L):
    g = (B.llep_gradient * 1)(B.llep_gradient(1 << 20, None, 8, B.LLEP_F32, 0))
    assert L.llep_clip_gradients(1, g, 1.0, A, A, 1 << 16, Z) == B.LLEP_E_ARG
    g[0].out = 1 << 20
    for bad in (-1.0, float("nan")):
        assert L.llep_clip_gradients(1, g, bad, A, A, 1 << 16, Z) == B.LLEP_E_ARG
    assert L.llep_gradient_norm(1, None, A, A, 1 << 16, Z) == B.LLEP_E_ARG
