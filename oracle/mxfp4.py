"""CPU oracle for 4-bit floating point with a power of two for every 32 values.

TEST INFRASTRUCTURE ONLY (see the package docstring). Plain definitions in
float64; pins in tests/test_oracle_mxfp4.py (worked blocks, exhaustive codes,
nearest values by search).
"""

from __future__ import annotations

import math

import numpy as np

from .llep import silu

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def _blocks(x):
    R, D = x.shape
    out = np.zeros((R, -(-D // BLOCK) * BLOCK))
    out[:, :D] = x
    return out.reshape(R, -1, BLOCK)


def mxfp4_exponents(x):
    """The exponent byte of every block of rows x [R, D]: [R, blocks]."""
    b = np.abs(_blocks(np.asarray(x, dtype=np.float64)))
    out = np.empty(b.shape[:2], dtype=np.uint8)
    for i in np.ndindex(*out.shape):
        most = b[i].max() if not np.isnan(b[i]).any() else math.inf
        if most == math.inf:
            out[i] = 255
        else:
            out[i] = 1 if most == 0 else max(math.frexp(most)[1] - 1 - 2 + 127, 1)
    return out


def mxfp4_codes(x, exponents):
    """The codes (0..15) of rows x with these exponents: nearest, ties to the even code, at most 6
    (of blocks with exponent 255: 0)."""
    b = _blocks(np.asarray(x, dtype=np.float64))
    fine = (exponents != 255)[..., None]
    y = np.where(fine, np.abs(b), 0.0) / np.exp2(exponents.astype(np.float64) - 127)[..., None]
    away = np.abs(y[..., None] - GRID)
    near = away.min(-1, keepdims=True)
    even = np.arange(8) % 2 == 0
    # of the nearest, the even one where there are two
    code = np.where(away == near, np.where(even, 1, 2), 3).argmin(-1)
    code = code + 8 * (np.signbit(b) & fine)
    return code.reshape(len(b), -1)[:, :np.asarray(x).shape[1]].astype(np.uint8)


def mxfp4_decode(codes, exponents):
    """What codes [R, D] with exponents [R, >= blocks] stand for, float64."""
    R, D = codes.shape
    e = np.repeat(exponents[:, :-(-D // BLOCK)], BLOCK, axis=1)[:, :D]
    v = np.where(codes > 7, -1.0, 1.0) * GRID[codes & 7] * np.exp2(e.astype(np.float64) - 127)
    return np.where(e == 255, np.nan, v)


def mxfp4_round(x):
    """Rows x through 4 bits and back."""
    e = mxfp4_exponents(x)
    return mxfp4_decode(mxfp4_codes(x, e), e)


def mxfp4_unpack(q, D):
    """Bytes [R, >= D / 2] to codes [R, D]: the first of two in the low half."""
    q = np.asarray(q)
    out = np.stack((q & 15, q >> 4), axis=-1).reshape(q.shape[0], -1)
    return out[:, :D]


def mxfp4_pack(codes):
    """Codes [R, D] to bytes [R, D / 2, rounded up]."""
    R, D = codes.shape
    c = np.zeros((R, D + D % 2), dtype=np.uint8)
    c[:, :D] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def mxfp4_doubt(x, near):
    """How far each value's rounding may move when x [R, D] is off by up to `near` [R, D]: 0 where
    it cannot change its value of the grid, else the step to the next one (at most 2), of a block
    whose exponent may be another one all of the block's values with twice the step."""
    x, near = np.asarray(x, dtype=np.float64), np.asarray(near, dtype=np.float64)
    b, n = np.abs(_blocks(x)), _blocks(near)
    e = mxfp4_exponents(x).astype(np.float64) - 127
    step = np.exp2(e)[..., None]
    borders = (GRID[1:] + GRID[:-1]) / 2
    hit = (np.abs(b[..., None] - borders * step[..., None]) <= n[..., None]).any(-1)
    out = np.where(hit, 2.0 * step, 0.0)
    # the largest may pass a power of two
    most = b.max(-1)
    low, high = np.maximum(most - n.max(-1), 0), most + n.max(-1)
    with np.errstate(divide="ignore"):
        moved = np.floor(np.log2(low)) != np.floor(np.log2(high))
    moved &= high > 2.0 ** -124
    out = np.where(moved[..., None], np.maximum(4.0 * step, 2.0 * b), out)
    return out.reshape(len(b), -1)[:, :x.shape[1]]


def swiglu_ffn_mxfp4(x, w_gate, w_up, w_down, unit):
    """One expert on rows x [R, D] (on the 4-bit grid) with weights [F, D], [F, D], [D, F] (what
    the 4-bit ones stand for): outputs [R, D], and how far they may be off when the first products
    are off by `unit` of their terms' magnitudes and the activation by (8 + |g|) 2^-22 of itself:
    as far as the activations' roundings to 4 bits may move."""
    g, u = x @ w_gate.T, x @ w_up.T
    act = silu(g) * u
    # |silu'| <= 1.1
    near = unit * (1.1 * (np.abs(x) @ np.abs(w_gate).T) * np.abs(u)
                   + np.abs(silu(g)) * (np.abs(x) @ np.abs(w_up).T))
    near += np.abs(act) * (8 + np.abs(g)) * 2.0 ** -22
    q = mxfp4_round(act)
    off = mxfp4_doubt(act, near) @ np.abs(w_down).T
    return q @ w_down.T, off + (len(w_down.T) + 32) * 2.0 ** -23 * (np.abs(q) @ np.abs(w_down).T)
