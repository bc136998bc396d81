"""CPU oracle for what stands around the expert layer: block norms with gate
and residual scale, the clipping of gradients by their global norm, 8-bit rows
and products.

TEST INFRASTRUCTURE ONLY (see the package docstring). Plain definitions in
float64; pins in tests/test_oracle_block.py (finite differences, closed forms,
whole-number cases).
"""

from __future__ import annotations

from typing import Dict, List, Sequence, Tuple

import numpy as np

from .llep import silu


def _f64(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def rms_norm(v, eps):
    """v / sqrt(mean(v^2) + eps) along the last axis."""
    v = _f64(v)
    return v / np.sqrt(np.mean(v * v, axis=-1, keepdims=True) + eps)


def block_norm(x, b, gate, w_post, w_pre, alpha, eps):
    """r = x + alpha * gate * (norm(b) * w_post), h = norm(r) * w_pre; b, gate, w_post and w_pre
    may be None (r = x; no gate; no norm of b; no h). gate broadcasts against [T, D]."""
    x, b, gate, w_post, w_pre = map(_f64, (x, b, gate, w_post, w_pre))
    r = x.copy()
    if b is not None:
        n = b if w_post is None else rms_norm(b, eps) * w_post
        r = r + alpha * (n if gate is None else gate * n)
    return r, None if w_pre is None else rms_norm(r, eps) * w_pre


def block_norm_backward(r, b, gate, w_post, w_pre, alpha, eps, d_r, d_h) -> Dict[str, np.ndarray]:
    """Gradients of block_norm by the chain rule, row by row, with each norm's
    Jacobian applied: d norm(v)_i / d v_j = (delta_ij - n_i n_j / D) / s,
    n = v / s, s = sqrt(mean(v^2) + eps)."""
    r, b, gate, w_post, w_pre, d_r, d_h = map(_f64, (r, b, gate, w_post, w_pre, d_r, d_h))
    T, D = d_r.shape

    def through(v, e):
        out = np.empty_like(v)
        for t in range(v.shape[0]):
            s = np.sqrt(np.mean(v[t] ** 2) + eps)
            n = v[t] / s
            out[t] = (e[t] - n * np.dot(n, e[t]) / D) / s
        return out

    out = {}
    total = d_r
    if w_pre is not None:
        out["dw_pre"] = np.sum(d_h * rms_norm(r, eps), axis=0)
        total = total + through(r, d_h * w_pre)
    out["dx"] = total
    if b is None:
        return out
    m = alpha * total * (1.0 if gate is None else gate)
    n = b if w_post is None else rms_norm(b, eps) * w_post
    if w_post is None:
        out["db"] = m * np.ones((T, D))
    else:
        out["dw_post"] = np.sum(m * rms_norm(b, eps), axis=0)
        out["db"] = through(b, m * w_post)
    if gate is not None:
        d_gate = alpha * total * n
        for axis in (0, 1):
            if gate.shape[axis] == 1:
                d_gate = d_gate.sum(axis=axis, keepdims=True)
        out["d_gate"] = d_gate
    return out


def quantize_rows(x) -> Tuple[np.ndarray, np.ndarray]:
    """8-bit rows in IEEE float32, step by step: scale = most * (1 / 127) and
    q = rint(x * (127 * (1 / most))) (ties to even) with most = max |x| of the row;
    rows below 2^-120 count as zero; rows that are not finite: scale NaN, q 0.
    Returns (q int8, scale float32)."""
    x = np.asarray(x, dtype=np.float32)
    q = np.zeros(x.shape, dtype=np.int8)
    scale = np.zeros(x.shape[0], dtype=np.float32)
    for t, row in enumerate(x):
        most = np.abs(row).max() if np.isfinite(row).all() else np.float32(np.nan)
        if np.isnan(most):
            scale[t] = np.nan
        elif most >= np.float32(2.0 ** -120):
            scale[t] = most * (np.float32(1) / np.float32(127))
            q[t] = np.rint(row * (np.float32(127) * (np.float32(1) / most))).astype(np.int8)
    return q, scale


def int8_product(x, x_scale, w, w_scale) -> np.ndarray:
    """x_scale[m] w_scale[n] sum_k x[m][k] w[n][k], the sum in whole numbers."""
    s = np.asarray(x, dtype=np.int64) @ np.asarray(w, dtype=np.int64).T
    return s.astype(np.float64) * _f64(x_scale)[:, None] * _f64(w_scale)[None, :]


def swiglu_ffn_int8(x, x_scale, w_gate, s_gate, w_up, s_up, w_down, s_down):
    """One expert on 8-bit rows (weights [F][D], [F][D], [D][F], rows = output
    channels): float64, the activation to 8 bits by row in between. Returns the
    outputs and the activations' row maxima."""
    g = int8_product(x, x_scale, w_gate, s_gate)
    a = silu(g) * int8_product(x, x_scale, w_up, s_up)
    most = np.abs(a).max(axis=1, keepdims=True, initial=0.0)
    step = np.where(most > 0, most / 127.0, 1.0)
    q = np.rint(a / step)
    w = _f64(w_down) * _f64(s_down)[:, None]
    return (q * step) @ w.T, most[:, 0]


def gradient_norm(grads: Sequence[np.ndarray]) -> float:
    """sqrt of the sum of squares over all elements of all tensors."""
    return float(np.sqrt(sum(float(np.sum(_f64(g) ** 2)) for g in grads)))


def clip_gradients(grads: Sequence[np.ndarray], max_norm: float) -> Tuple[float, List[np.ndarray]]:
    """The norm, and the gradients times min(1, max_norm / norm); as they are
    where the norm is not finite (in float32) or at most max_norm."""
    norm = gradient_norm(grads)
    clip = norm > max_norm and norm <= float(np.finfo(np.float32).max)
    factor = max_norm / norm if clip else 1.0
    return norm, [_f64(g) * factor for g in grads]
