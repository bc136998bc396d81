"""Pins of the oracle's block norms and gradient clipping: closed forms and
central finite differences of the definitions."""

import numpy as np
import pytest

import oracle

EPS = 1e-3


def _inputs(T, D, gate, post, pre, block=True, seed=0):
    g = np.random.default_rng(seed)
    x = g.standard_normal((T, D))
    b = g.standard_normal((T, D)) if block else None
    shape = {"none": None, "channel": (1, D), "token": (T, 1), "full": (T, D)}[gate]
    gt = None if shape is None else g.standard_normal(shape)
    w_post = g.standard_normal(D) if post else None
    w_pre = g.standard_normal(D) if pre else None
    return x, b, gt, w_post, w_pre


def test_closed_forms():
    # one element: norm(v) = v / sqrt(v^2 + eps)
    r, h = oracle.block_norm([[3.0]], [[4.0]], [[2.0]], [5.0], [7.0], 0.5, 0.0)
    assert r[0, 0] == pytest.approx(3.0 + 0.5 * 2.0 * 5.0)
    assert h[0, 0] == pytest.approx(7.0)
    # a zero row stays finite: 0 / sqrt(eps)
    r, h = oracle.block_norm(np.zeros((1, 4)), np.zeros((1, 4)), None, np.ones(4), np.ones(4), 1.0,
                             EPS)
    assert not r.any() and not h.any()
    # (3, 4): mean square 12.5
    n = oracle.rms_norm([[3.0, 4.0]], 0.0)
    assert np.allclose(n, np.array([[3.0, 4.0]]) / np.sqrt(12.5))
    r, h = oracle.block_norm([[3.0, 4.0]], None, None, None, [1.0, 2.0], 9.0, 0.0)
    assert np.allclose(r, [[3.0, 4.0]]) and np.allclose(h, n * [1.0, 2.0])


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre,block", [(True, True, True), (False, True, True),
                                            (True, False, True), (False, True, False)])
def test_backward_against_differences(gate, post, pre, block):
    if not block and (gate != "none" or post):
        pytest.skip("no block: no gate")
    T, D, alpha = 3, 5, 0.7
    x, b, gt, w_post, w_pre = _inputs(T, D, gate, post, pre, block)
    g = np.random.default_rng(9)
    d_r = g.standard_normal((T, D))
    d_h = g.standard_normal((T, D)) if pre else None

    def loss(x, b, gt, w_post, w_pre):
        r, h = oracle.block_norm(x, b, gt, w_post, w_pre, alpha, EPS)
        return np.sum(r * d_r) + (0.0 if h is None else np.sum(h * d_h))

    r, _ = oracle.block_norm(x, b, gt, w_post, w_pre, alpha, EPS)
    got = oracle.block_norm_backward(r, b, gt, w_post, w_pre, alpha, EPS, d_r, d_h)
    args = [x, b, gt, w_post, w_pre]
    for i, key in enumerate(["dx", "db", "d_gate", "dw_post", "dw_pre"]):
        if args[i] is None:
            assert key not in got
            continue
        want = np.zeros_like(args[i])
        for at in np.ndindex(*args[i].shape):
            two = []
            for step in (1e-5, -1e-5):
                moved = [None if a is None else a.copy() for a in args]
                moved[i][at] += step
                two.append(loss(*moved))
            want[at] = (two[0] - two[1]) / 2e-5
        assert got[key].shape == want.shape
        assert np.abs(got[key] - want).max() <= 1e-7 * max(1.0, np.abs(want).max()), key


def test_clip():
    g = [np.array([3.0]), np.zeros(0), np.array([[4.0]])]
    assert oracle.gradient_norm(g) == 5.0 and oracle.gradient_norm([]) == 0.0
    norm, out = oracle.clip_gradients(g, 1.0)
    assert norm == 5.0 and np.allclose([out[0][0], out[2][0, 0]], [0.6, 0.8])
    assert oracle.clip_gradients(g, 5.0)[1][0][0] == 3.0
    norm, out = oracle.clip_gradients([np.array([np.inf, 1.0])], 1.0)
    assert norm == np.inf and out[0][1] == 1.0


def test_int8_rows_and_products():
    q, s = oracle.quantize_rows([[1.0, -2.0, 0.5, 0.0], [0.0] * 4, [np.inf, 1.0, 2.0, 3.0],
                                 [1e-37, 0.0, 0.0, 0.0], [0.0, np.nan, 1.0, 1.0]])
    assert q.tolist() == [[64, -127, 32, 0], [0] * 4, [0] * 4, [0] * 4, [0] * 4]  # 63.5 to even
    assert s[0] == np.float32(2.0) * (np.float32(1) / np.float32(127)) and s[1] == 0 and s[3] == 0
    assert np.isnan(s[2]) and np.isnan(s[4])
    assert oracle.int8_product([[1, -2]], [0.5], [[3, 4], [127, 127]], [1.0, 2.0]).tolist() == \
        [[-2.5, -127.0]]


def test_int8_expert_near_the_real_one():
    """The 8-bit expert on the values that its bytes stand for, against the SwiGLU expert: apart
    only by the activation's own rounding, at most half a step for each of the F values."""
    g = np.random.default_rng(3)
    n, D, F = 5, 16, 24
    q = [g.integers(-127, 128, s).astype(np.int8) for s in ((n, D), (F, D), (F, D), (D, F))]
    sx, sg, su, sd = (g.uniform(0.5, 1.5, k) / 127 for k in (n, F, F, D))
    got, most = oracle.swiglu_ffn_int8(q[0], sx, q[1], sg, q[2], su, q[3], sd)
    real = [a.astype(np.float64) * s[:, None] for a, s in zip(q, (sx, sg, su, sd))]
    want = oracle.swiglu_ffn(real[0], real[1].T, real[2].T, real[3].T)
    bound = (most / 254)[:, None] * np.abs(real[3]).sum(axis=1)[None, :]
    assert (np.abs(got - want) <= bound + 1e-12).all() and np.abs(got - want).max() > 0
