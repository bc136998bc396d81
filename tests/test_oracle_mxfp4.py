"""Pins of the 4-bit oracle: blocks worked by hand, every code and exponent, the
nearest value by search, and sums that the doubt of a rounding covers."""

import math

import numpy as np
import pytest

import oracle


def test_a_block_by_hand():
    # largest 13: 2^3, so steps of 2^1 (exponent byte 128); 13 / 2 = 6.5 -> 6
    x = np.zeros((1, 32))
    x[0, :9] = [13.0, -12.0, 1.0, 0.5, -0.5, 0.51, 5.0, 7.0, 3.5]
    e = oracle.mxfp4_exponents(x)
    assert e.tolist() == [[128]]
    # 0.25 and 2.5, 3.5, 1.75 are ties: 0, 2, 4, 2
    assert oracle.mxfp4_round(x)[0, :9].tolist() == [12.0, -12.0, 1.0, 0.0, 0.0, 1.0, 4.0, 8.0, 4.0]
    assert oracle.mxfp4_codes(x, e)[0, :3].tolist() == [7, 15, 1]


def test_exponents():
    for most, b in ((1.0, 125), (1.999, 125), (2.0, 126), (0.0, 1), (2.0 ** -126, 1),
                    (2.0 ** -123, 2), (2.0 ** -124, 1), (2.0 ** 127, 252), (math.inf, 255),
                    (math.nan, 255)):
        assert oracle.mxfp4_exponents(np.array([[0.0, -most]]))[0, 0] == b, most
    # blocks of 32, the last one shorter
    x = np.ones((2, 70))
    x[1, 64:] = 8.0
    assert oracle.mxfp4_exponents(x).tolist() == [[125, 125, 125], [125, 125, 128]]


def test_every_code_and_exponent_decodes():
    codes = np.arange(16, dtype=np.uint8)[None, :].repeat(256, 0)
    v = oracle.mxfp4_decode(codes, np.arange(256, dtype=np.uint8)[:, None])
    assert np.isnan(v[255]).all()
    for b in (0, 1, 127, 254):
        assert v[b].tolist() == [s * g * 2.0 ** (b - 127) for s in (1, -1)
                                 for g in (0, 0.5, 1, 1.5, 2, 3, 4, 6)]


def test_bytes():
    c = np.array([[1, 2, 3], [15, 0, 9]], dtype=np.uint8)
    b = oracle.mxfp4_pack(c)
    assert b.tolist() == [[0x21, 0x03], [0x0f, 0x09]]
    assert np.array_equal(oracle.mxfp4_unpack(b, 3), c)


def test_nearest_by_search():
    g = np.random.default_rng(0)
    x = g.normal(size=(8, 96)) * np.exp2(g.integers(-20, 20, (8, 96)))
    r, e = oracle.mxfp4_round(x), oracle.mxfp4_exponents(x)
    grid = sorted({s * v for s in (1, -1) for v in (0, 0.5, 1, 1.5, 2, 3, 4, 6)})
    for i in range(8):
        for j in range(96):
            step = 2.0 ** (int(e[i, j // 32]) - 127)
            assert abs(r[i, j] - x[i, j]) == min(abs(step * v - x[i, j]) for v in grid)
    # of the largest of a block at most a quarter is lost (7.99 -> 6), of others half a step
    assert (np.abs(r - x) <= np.maximum(0.25 * np.abs(x), 0.25 * np.exp2(
        e.repeat(32, 1).astype(float) - 127))).all()


def test_doubt_covers_moved_roundings():
    g = np.random.default_rng(1)
    x = g.normal(size=(400, 64))
    x[:, 0] = np.exp2(g.integers(-3, 3, 400)) * (1 + g.uniform(-1e-3, 1e-3, 400))
    near = np.abs(x) * 1e-2
    moved = oracle.mxfp4_round(x + near * g.uniform(-1, 1, x.shape))
    d = oracle.mxfp4_doubt(x, near)
    away = np.abs(moved - oracle.mxfp4_round(x))
    assert (away <= d).all() and (away > 0).sum() > 50
    assert (oracle.mxfp4_doubt(x, near * 0) > 0).sum() == 0


def test_an_expert_by_hand():
    x = np.zeros((1, 64))
    x[0, 0] = 2.0
    w = np.zeros((64, 64))
    w[5, 0] = 1.5
    wd = np.zeros((64, 64))
    wd[7, 5] = -2.0
    y, off = oracle.swiglu_ffn_mxfp4(x, w, w, wd, 1e-6)
    # g = u = 3: 9 sigmoid(3) = 8.57, steps of 2: 4.29 -> 4
    assert 9 / (1 + math.exp(-3)) == pytest.approx(8.573, abs=1e-3)
    assert y[0, 7] == -16.0 and np.count_nonzero(y) == 1
    assert off[0, 7] < 1e-3
