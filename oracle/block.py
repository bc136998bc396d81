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
