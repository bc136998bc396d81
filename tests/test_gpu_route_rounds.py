"""Routing of many rows by rounds (more than 8 experts a token, or more groups than a
row's 16 lanes), in each of its widths and with each number of groups a lane holds, and
batches on both sides of the numbers of rows at which a row's lanes change; against the
oracle on a sample of rows: ids exactly, gates within 64 u and, below 2^-126, 1.5 steps
of 2^-149 times the factor and half a step (u = 2^-24, counted in test_gpu_route.py)."""

import math

import numpy as np
import pytest

import oracle
from gpu_util import device

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF = math.inf


@pytest.fixture(scope="module")
def dev():
    return device()


def _logits(seed, T, E, masked=0.05):
    import torch
    g = torch.Generator().manual_seed(seed)
    l = (torch.randn(T, E, generator=g) * 1.5).clamp(-8, 8)
    l[torch.rand(T, E, generator=g) < masked] = -INF
    l[torch.rand(T, generator=g) < masked] = -INF
    return l, torch.randn(E, generator=g) * 0.1


def _route(x, K, b, how):
    import torch
    from paper_2601_17111_amd import binding as B
    T, E = x.shape
    ids = torch.full((T, K), 77, dtype=torch.int32, device=x.device)
    gates = torch.full((T, K), -7.0, device=x.device)
    B.llep_route(B.make_route(T, K, E, **how), x, b, ids, gates)
    torch.cuda.synchronize()
    return ids, gates


def _check(x, K, b, how, at, ids, gates):
    want_ids, want = oracle.route(x.float().cpu().numpy()[at], K, bias=None if b is None else b.cpu().numpy(),
                                  **how)
    assert np.array_equal(ids.cpu().numpy()[at], want_ids)
    near = 64 * U * np.abs(want) + 2.0 ** -149 * (1.5 * how.get("scale", 1.0) + 0.5)
    assert np.all(np.abs(gates.double().cpu().numpy()[at] - want) <= near)


def _kernel(call):
    import torch
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as seen:
        call()
        torch.cuda.synchronize()
    names = [e.name for e in seen.events() if "route_" in e.name]
    assert len(names) == 1, names
    return names[0]


@pytest.mark.parametrize("T,E,G,top,K,per", [
    (2300, 20, 1, 1, 12, 2), (2101, 40, 1, 1, 9, 4), (2200, 100, 1, 1, 16, 8), (2500, 200, 1, 1, 10, 16),
    (2100, 500, 1, 1, 13, 32), (2300, 30, 5, 3, 11, 2), (2200, 128, 8, 4, 12, 8), (2050, 240, 10, 3, 9, 16),
    (2300, 60, 20, 7, 7, 4), (2100, 64, 64, 9, 8, 4), (2100, 28, 28, 12, 6, 2), (2100, 512, 64, 20, 12, 32),
    (2100, 510, 51, 20, 8, 32), (2049, 165, 33, 5, 16, 16),
])
def test_rounds_of_many_rows(dev, T, E, G, top, K, per):
    import torch
    l, bias = _logits(T + E + K, T, E)
    at = np.unique(np.r_[np.arange(0, T, 41), np.arange(T - 9, T)])
    names = set()
    for dtype in (torch.float32, torch.bfloat16):
        x = l.to(dtype).to(dev)
        for b in (None, bias.to(dev)):
            for by in ("max", "top2") if G > 1 else ("max",):
                for score, renormalize in (("softmax", True), ("softmax", False), ("sigmoid", True)):
                    how = dict(score=score, renormalize=renormalize, scale=2.5, groups=G, top_groups=top,
                               group_score=by)
                    ids, gates = _route(x, K, b, how)
                    _check(x, K, b, how, at, ids, gates)
                names.add(_kernel(lambda: _route(x, K, b, how)))
    assert len(names) == 4 and all("route_rounds_kernel" in n and f", {per}, 16, " in n for n in names), names


@pytest.mark.parametrize("E,K", [(32, 4), (100, 8), (128, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_few_and_many_rows(dev, E, K, score, renormalize):
    """Rows have the same ids on both sides of 1024 rows (64 and 16 lanes a row, with a bias) and of
    12288 (16 and 4, without one); their gates are those of their logits, whatever the order in which
    so many lanes add a row up."""
    import torch
    how = dict(score=score, renormalize=renormalize)
    l, bias = _logits(E + K, 12400, E)
    for b, sizes in ((bias.to(dev), (50, 1024, 1025, 3000)), (None, (50, 4000, 12287, 12288, 12400))):
        x = l.to(dev)
        first = None
        for T in sizes:
            ids, gates = _route(x[:T], K, b, how)
            at = np.unique(np.r_[np.arange(50), np.arange(0, T, 211), T - 1])
            _check(x[:T], K, b, how, at, ids, gates)
            first = ids[:50] if first is None else first
            assert torch.equal(ids[:50], first)
