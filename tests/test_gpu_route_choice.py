"""The choice of experts where keys lie closer than the kernels' sorted keys tell
apart: group sums whose two keys cancel, keys hidden behind equal ones, scores that
are nothing next to each other; against the oracle's float64 keys, ids exactly, in
few and in many rows (64 and 16 lanes a row).

Ids are compared exactly although a score of the kernel and one of the oracle may
differ by a step or two of float64: the logits here are such that no key lies within
two steps of a score of a border between two roundings (test_logits_are_off_the_borders
computes that in 60 digits), or such that the scores' differences are far above them."""

from decimal import Decimal, getcontext

import numpy as np
import pytest

import oracle
from gpu_util import device

gpu = pytest.mark.gpu

# sigmoids of these have no key within two steps under the biases of CANCEL
FEW = (-1.5, -1.0, 0.0, 1.0, 1.5)
CANCEL = (16.0, 64.0, 1000.0)


@pytest.fixture(scope="module")
def dev():
    return device()


def _same_ids(dev, l, K, bias=None, rows=None, dtype="float32", **how):
    """llep_route's ids of logits [T, E] against the oracle's (of `rows` of them)."""
    import torch
    from paper_2601_17111_amd import binding as B
    x = torch.from_numpy(np.ascontiguousarray(l, dtype=np.float32)).to(getattr(torch, dtype)).to(dev)
    T, E = x.shape
    b = None if bias is None else torch.from_numpy(np.asarray(bias, dtype=np.float32)).to(dev)
    ids = torch.full((T, K), 77, dtype=torch.int32, device=dev)
    gates = torch.empty((T, K), device=dev)
    B.llep_route(B.make_route(T, K, E, **how), x, b, ids, gates)
    rows = np.arange(T) if rows is None else rows
    want, _ = oracle.route(x.float().cpu().numpy()[rows], K, bias=None if b is None else b.cpu().numpy(),
                           **how)
    got = ids.cpu().numpy()[rows]
    bad = np.nonzero((got != want).any(1))[0]
    assert len(bad) == 0, (rows[bad[:3]], got[bad[:3]], want[bad[:3]], len(bad))


def test_logits_are_off_the_borders():
    getcontext().prec = 60
    for l in FEW:
        s = 1 / (1 + (-Decimal(l)).exp())
        step = Decimal(float(np.spacing(float(s))))
        for bias in CANCEL:
            for b in (bias, -bias):
                key = s + Decimal(b)
                k = float(key)
                half = Decimal(float(np.spacing(abs(k)))) / 2
                border = min(abs(key - Decimal(k) - half), abs(key - Decimal(k) + half))
                assert border > 2 * step, (l, b)


@gpu
def test_group_sums_that_cancel(dev):
    """Two keys of 64 and -65 whose sum decides: its cut is that of the keys."""
    l = np.array([[0.0, 4e-13, 4 * 2.0 ** -37 - 4e-13, 0.0]])
    how = dict(score="sigmoid", groups=2, top_groups=1, group_score="top2")
    for T in (1, 60, 1100):
        _same_ids(dev, np.repeat(l, T, 0), 2, [64.0, -65.0, 64.0, -65.0], **how)


@gpu
@pytest.mark.parametrize("T", [700, 1100])
@pytest.mark.parametrize("E,G,top", [(32, 16, 5), (32, 16, 8), (64, 8, 3), (256, 8, 4)])
@pytest.mark.parametrize("size", CANCEL)
def test_groups_of_large_biases_of_both_signs(dev, T, E, G, top, size):
    """Few different logits, whose sums differ by the roundings of the keys alone."""
    g = np.random.default_rng(int(size) + E + top)
    rows = np.unique(np.concatenate([np.arange(0, T, 2 if E < 100 else 12), [T - 1]]))
    for _ in range(2):
        _same_ids(dev, g.choice(FEW, (T, E)), 4, g.choice([-size, size], E), rows, score="sigmoid",
                  groups=G, top_groups=top, group_score="top2")


@gpu
@pytest.mark.parametrize("T", [700, 1100])
@pytest.mark.parametrize("size,around", [(64.0, -22.0), (1e3, -22.0), (1e11, 0.0), (1e12, 0.0)])
def test_groups_whose_two_best_cancel(dev, T, size, around):
    """Every group's best expert is raised by as much as its second is lowered."""
    E, G = 64, 8
    g = np.random.default_rng(int(size) % 97)
    rows = np.arange(0, T, 2)
    for _ in range(2):
        b = np.full(E, -3 * size)
        for e in range(0, E, E // G):
            at = e + g.permutation(E // G)[:2]
            b[at] = size, -size
        _same_ids(dev, around + g.normal(size=(T, E)), 2, b, rows, score="sigmoid", groups=G, top_groups=4,
                  group_score="top2")


# saturated sigmoids: 1 - s is 9.4e-14 for 30, 7.7e-14 for 30.2, less apart than a cut key's
# step of 5.7e-14 and far more than a step of float64 (1.1e-16)
HIDDEN = [
    # the last of the chosen, one that is equal to it, and behind both a larger one
    (1, [30, 30, 30.2, 0, 1, 2, 3, 4], None),
    (1, [0, 30, 1, 30, 30, 2, 30, 30.25], None),
    (3, [3, 2, 30, 1, 30, 0, 0.5, 30.2], [1, 1, 0, 0, 0, 0, 0, 0]),
    (4, [3, 2, 30, 1, 30, 30.2, 30, 30.2], [1, 1, 0, 0, 0, 0, 0, 0]),
    # the same, below zero
    (2, [1, 30, 30, 30.2, 0, 0, 0, 0], [4, -3, -3, -3, -9, -9, -9, -9]),
]


@gpu
@pytest.mark.parametrize("K,row,bias", HIDDEN)
def test_a_key_hidden_behind_an_equal_one(dev, K, row, bias):
    """Among rows of which the same is true, in whatever order of the experts, and others."""
    E = len(row)
    g = np.random.default_rng(K)
    for T in (1, 60, 1100):
        for wide in (E, 40, 200):
            l = np.full((T, wide), -4.0) + 0.25 * (np.arange(wide) % 7)
            l[:, wide - E:] = row
            if T > 1:
                l[1::3] += g.normal(size=l[1::3].shape)
            b = np.zeros(wide) if bias is None else np.r_[np.full(wide - E, -9.0), bias]
            rows = np.unique(np.r_[np.arange(0, T, 17), T - 1])
            for dtype in ("float32", "bfloat16"):
                _same_ids(dev, l, K, b, rows, dtype, score="sigmoid")


# groups whose best ones are equal, and of one of them another that is larger by less than a cut key
# tells (30 against 30.2; 26 against 26 + 2^-7: 1 - s is 5.1e-12, its difference 4.0e-14)
HIDDEN_GROUPS = [
    ("max", 2, [30, 20, 0, 0, 30, 30.2, 0, 0], True, 1),
    ("max", 2, [30, 1, 30, 2, 30, 30, 30.2, 20], True, 1),
    ("top2", 2, [30, 26, 0, 1, 30, 26, 26 + 2.0 ** -7, 1], False, 1),
    ("top2", 2, [30, 26, 0, 1, 30, 26, 26 + 2.0 ** -7, 1], True, 1),
    ("top2", 2, [30, 26, 0, 1, 0, 1, 2, 3, 26, 30, 1, 26 + 2.0 ** -7, 4, 3, 2, 1], False, 1),
]


@gpu
@pytest.mark.parametrize("by,K,row,bias,top", HIDDEN_GROUPS)
def test_a_group_that_is_larger_by_a_hidden_key(dev, by, K, row, bias, top):
    E, size = len(row), 4
    for T in (1, 60, 1100):
        for groups in (E // size, 8, 16):
            l = np.full((T, groups * size), -4.0) + 0.25 * (np.arange(groups * size) % 7)
            l[:, groups * size - E:] = row
            for dtype in ("float32", "bfloat16"):
                _same_ids(dev, l, K, np.zeros(groups * size) if bias else None, None if T < 100 else
                          np.arange(0, T, 37), dtype, score="sigmoid", groups=groups, top_groups=top,
                          group_score=by)


@gpu
@pytest.mark.parametrize("low", [-1e3, -1e9, float(np.finfo(np.float32).min)])
def test_groups_of_nothing_but_scores_of_zero(dev, low):
    """Masks by a low finite value: groups of such experts are equal, also where -infinity leaves one
    of them a single expert."""
    inf = np.inf
    for T in (1, 60, 1100):
        for row in ([1.0, 2.0, low, -inf, low, low], [low, -inf, -inf, low, 1.0, 2.0],
                    [low, -inf, -inf, low, low, low]):
            _same_ids(dev, np.repeat([row], T, 0), 4, score="sigmoid", groups=3, top_groups=2,
                      group_score="top2")


@gpu
@pytest.mark.parametrize("by", ["max", "top2"])
def test_all_groups_are_no_groups(dev, by):
    """Sigmoids that are 1 in float64 tie as keys, their logits do not: the keys are the logits where
    every group remains, and the scores where one does not."""
    import torch
    l = np.repeat([[50.0, 60.0, 70.0, 80.0, 0.0, 90.0, 1.0, 2.0]], 3, 0)
    for top in (1, 2, 4):
        _same_ids(dev, l, 2, score="sigmoid", groups=4, top_groups=top, group_score=by)
    from paper_2601_17111_amd import binding as B
    x = torch.from_numpy(l).float().to(dev)
    ids = [torch.empty((3, 2), dtype=torch.int32, device=dev) for _ in range(3)]
    for i, (groups, top) in zip(ids, ((4, 4), (1, 1), (4, 3))):
        B.llep_route(B.make_route(3, 2, 8, "sigmoid", groups, top, by), x, None, i,
                     torch.empty((3, 2), device=dev))
    assert ids[0].tolist() == ids[1].tolist() == [[5, 3]] * 3
    # (the groups' scores are 2, 2, 1.5 and about 1.6 in float64, or 60, 80, 90 and 2)
    assert ids[2].tolist() == ([[0, 1]] if by == "top2" else [[5, 3]]) * 3
