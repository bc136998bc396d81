"""CPU oracle for the routing of tokens to experts and its gradient.

TEST INFRASTRUCTURE ONLY (see the package docstring). Plain definitions in
float64, a row at a time; pins in tests/test_oracle_route.py (worked rows,
finite differences, whole-number cases).
"""

from __future__ import annotations

import math

import numpy as np


def route_scores(row, score):
    """softmax or sigmoid of one row of logits; an expert with -inf has 0 (and a row of them)."""
    row = np.asarray(row, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-row))
        top = np.nanmax(row) if not np.all(np.isnan(row)) else 0.0
        e = np.exp(row - (top if top > -math.inf else 0.0))
        total = e.sum()
        return e / total if total != 0.0 else e


def choose(row, K, score="softmax", bias=None, groups=1, top_groups=1, group_score="max"):
    """The ids of one row: K of them, -1 where none is left."""
    row = np.asarray(row, dtype=np.float64)
    E = len(row)
    if bias is not None or (group_score == "top2" and top_groups < groups):
        key = route_scores(row, score) + (0.0 if bias is None else np.asarray(bias, np.float64))
    else:
        key = row
    # one that may be taken: (key, expert)
    left = [(float(key[e]), e) for e in range(E) if row[e] > -math.inf and key[e] > -math.inf]
    if top_groups < groups:
        size = E // groups
        of = [sorted((k for k, e in left if e // size == g), reverse=True) for g in range(groups)]
        value = [(sum(ks[:2]) if group_score == "top2" else ks[0]) if ks else -math.inf
                 for ks in of]
        kept = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
        left = [(k, e) for k, e in left if e // size in kept]
    left.sort(key=lambda ke: (-ke[0], ke[1]))
    ids = [e for _, e in left[:K]]
    return ids + [-1] * (K - len(ids))


def gates_of(row, ids, score="softmax", renormalize=True, scale=1.0):
    """The gates of these experts of one row."""
    row = np.asarray(row, dtype=np.float64)
    if not renormalize:
        s = route_scores(row, score)
        return [scale * float(s[e]) if e >= 0 else 0.0 for e in ids]
    # log scores: no sum of them vanishes
    if score == "softmax":
        logs = {e: float(row[e]) for e in ids if e >= 0}
    else:
        logs = {e: -float(np.logaddexp(0.0, -row[e])) for e in ids if e >= 0}
    if not logs:
        return [0.0] * len(ids)
    top = max(logs.values())
    total = sum(math.exp(logs[e] - top) for e in ids if e >= 0)
    return [scale * math.exp(logs[e] - top) / total if e >= 0 else 0.0 for e in ids]


def route(logits, K, score="softmax", bias=None, groups=1, top_groups=1, group_score="max",
          renormalize=True, scale=1.0):
    """(ids [T, K], gates [T, K]) of logits [T, E]."""
    ids = [choose(r, K, score, bias, groups, top_groups, group_score) for r in logits]
    gates = [gates_of(r, i, score, renormalize, scale) for r, i in zip(logits, ids)]
    T = len(ids)
    return (np.array(ids, dtype=np.int64).reshape(T, K),
            np.array(gates, dtype=np.float64).reshape(T, K))


def route_backward(logits, ids, d_gates, score="softmax", renormalize=True, scale=1.0):
    """d_logits through the Jacobian of each row's gates (ids fixed, -1: none)."""
    logits = np.asarray(logits, dtype=np.float64)
    out = np.zeros_like(logits)
    for t, row in enumerate(logits):
        pairs = [(e, float(d)) for e, d in zip(ids[t], d_gates[t]) if 0 <= e < len(row)]
        named = [e for e, _ in pairs]
        if not named:
            continue
        g = gates_of(row, named, score, renormalize, scale)
        s = route_scores(row, score)
        for (k, (_, d)), e in zip(enumerate(pairs), named):
            # d g_k / d l, row by row of the Jacobian
            jac = np.zeros(len(row))
            if score == "softmax":
                jac[e] += g[k]
                if renormalize:
                    for j, f in enumerate(named):
                        jac[f] -= g[k] * g[j] / scale
                else:
                    jac -= g[k] * s
            else:
                jac[e] += g[k] * (1.0 - s[e])
                if renormalize:
                    for j, f in enumerate(named):
                        jac[f] -= g[k] * g[j] / scale * (1.0 - s[f])
            out[t] += d * jac
    return out
