"""llep_gradient_norm and llep_clip_gradients on the GPU against the oracle:
empty lists and tensors, one element to several pieces and launches, odd
counts, starts off 16-byte boundaries, both types mixed, in place and out of
place, norms at and below the limit, infinities and NaN, sums that leave the
range of 32 bits; the same bits every time; refusals.

Tolerances: the norm is summed in 64 bits and rounded to 32 once (2^-24, twice
allowed); a clipped value is one product of 32 bits with a factor rounded once
(2^-23 in all, twice allowed), a bfloat16 one rounded once more (2^-8)."""

import numpy as np
import pytest

import oracle
from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _tensors(dev, spec, seed=0, scale=0.1):
    """spec: (elements, type, elements by which it starts off an aligned address)."""
    import torch
    g = torch.Generator().manual_seed(seed)
    out = []
    for n, dtype, off in spec:
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        flat = torch.empty(n + off, dtype=dt, device=dev)
        flat[off:].copy_((torch.randn(n, generator=g) * scale).to(dt))
        out.append(flat[off:])
    return out


def _run(B, grads, max_norm, out, dev):
    import torch
    norm = torch.full((1,), -1.0, device=dev)
    ws = torch.empty(B.llep_clip_gradients_workspace_bytes(), dtype=torch.uint8, device=dev)
    ws.fill_(0xff)
    alone = torch.full((1,), -1.0, device=dev)
    B.llep_gradient_norm(grads, alone, ws)
    ws.fill_(0xff)
    B.llep_clip_gradients(grads, max_norm, norm, ws, out=out)
    torch.cuda.synchronize()
    assert torch.equal(norm, alone) or (torch.isnan(norm).all() and torch.isnan(alone).all())
    return float(norm)


MIXED = [(n, "bf16" if i % 3 == 0 else "f32", i % 4)
         for i, n in enumerate([1, 7, 8, 9, 0, 64, 1000, 16383, 16384, 16385, 40000])]


@pytest.mark.parametrize("spec", [
    [(1, "f32", 0)], [(1, "bf16", 1)], [(0, "f32", 0)], [], MIXED,
    [(100003, "f32", 0)], [(100003, "bf16", 0)], [(100001, "f32", 1)], [(100001, "bf16", 3)],
    MIXED * 30,                      # more tensors than one launch takes
    [(20_000_000, "f32", 0)],        # more pieces than workgroups
    [(5, "f32", 0)] * 96, [(5, "f32", 0)] * 97,
], ids=lambda s: f"{len(s)}x{sum(n for n, _, _ in s)}")
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(dev, spec, in_place):
    import torch
    from paper_2601_17111_amd import binding as B
    grads = _tensors(dev, spec)
    host = [g.double().cpu().numpy() for g in grads]
    exact = oracle.gradient_norm(host)
    for max_norm in (0.25 * exact, 2.0 * exact + 1.0):
        mine = [g.clone() if g.storage_offset() == 0 else
                torch.empty(g.numel() + g.storage_offset(), dtype=g.dtype, device=dev)
                [g.storage_offset():].copy_(g) for g in grads]
        out = mine if in_place else [torch.full_like(g, 7.0) for g in mine]
        norm = _run(B, mine, max_norm, None if in_place else out, dev)
        assert abs(norm - exact) <= 2.0 ** -23 * exact
        want_norm, want = oracle.clip_gradients(host, max_norm)
        for g, o, w in zip(mine, out, want):
            tol = 2.0 ** -22 + (2.0 ** -8 if o.dtype == torch.bfloat16 else 0.0)
            got = o.double().cpu().numpy()
            assert (np.abs(got - w) <= tol * np.abs(w) + 1e-44).all()
            if max_norm > exact:
                assert torch.equal(o, g)


def test_same_bits(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    grads = _tensors(dev, MIXED * 3, seed=5)
    first = None
    for _ in range(3):
        out = [torch.empty_like(g) for g in grads]
        norm = _run(B, grads, 0.1, out, dev)
        if first is None:
            first = (norm, out)
        assert norm == first[0] and all(torch.equal(a, b) for a, b in zip(out, first[1]))


def test_range_and_not_finite(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    # squares of 1e30 leave the range of 32 bits, their norm does not
    g = [torch.full((1000,), 1e30, device=dev), torch.full((9,), 1e-30, device=dev)]
    out = [torch.empty_like(t) for t in g]
    norm = _run(B, g, 1.0, out, dev)
    assert norm == pytest.approx(1e30 * np.sqrt(1000.0), rel=1e-6)
    assert float(out[0][0]) == pytest.approx(1.0 / np.sqrt(1000.0), rel=1e-6)
    # the type's largest value everywhere: the norm is infinite in 32 bits
    top = torch.full((64,), torch.finfo(torch.float32).max, device=dev)
    for bad in (top, torch.tensor([1.0, float("inf")], device=dev),
                torch.tensor([float("nan"), 2.0, -float("inf")], device=dev)):
        g = [bad, torch.full((33,), 3.0, device=dev)]
        for out in ([torch.zeros_like(t) for t in g], None):
            want = [t.clone() for t in g]
            norm = _run(B, g, 1.0, out, dev)
            assert np.isnan(norm) if torch.isnan(bad).any() else norm == np.inf
            for o, w in zip(g if out is None else out, want):
                assert torch.equal(torch.nan_to_num(o, 5.0), torch.nan_to_num(w, 5.0))
    # limits of 0 and infinity, and gradients of zero
    g = [torch.full((5,), 2.0, device=dev)]
    out = [torch.empty_like(g[0])]
    _run(B, g, 0.0, out, dev)
    assert not out[0].any()
    _run(B, g, float("inf"), out, dev)
    assert torch.equal(out[0], g[0])
    assert _run(B, [torch.zeros(5, device=dev)], 0.0, None, dev) == 0.0


def test_another_stream_and_graph(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    grads = _tensors(dev, MIXED, seed=2)
    out = [torch.empty_like(g) for g in grads]
    norm = torch.zeros(1, device=dev)
    ws = torch.empty(B.llep_clip_gradients_workspace_bytes(), dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.llep_clip_gradients(grads, 0.5, norm, ws, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.llep_clip_gradients(grads, 0.5, norm, ws, out=out)
    for k in range(3):
        for g in grads:
            g.add_(0.01 * k)
        want = [torch.empty_like(g) for g in grads]
        want_norm = torch.zeros(1, device=dev)
        B.llep_clip_gradients(grads, 0.5, want_norm, torch.empty_like(ws), out=want)
        for o in out:
            o.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want_norm)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    g = torch.ones(8, device=dev)
    norm = torch.zeros(1, device=dev)
    ws = torch.empty(B.llep_clip_gradients_workspace_bytes(), dtype=torch.uint8, device=dev)
    B.llep_clip_gradients([g], 1.0, norm, ws)
    for bad in (-1.0, float("nan")):
        with pytest.raises(B.LLEPError) as ei:
            B.llep_clip_gradients([g], bad, norm, ws)
        assert ei.value.code == B.LLEP_E_ARG
    with pytest.raises(B.LLEPError) as ei:
        B.llep_gradient_norm([g], norm, ws[:8])
    assert ei.value.code == B.LLEP_E_WORKSPACE
    with pytest.raises(TypeError):
        B.llep_gradient_norm([g.half()], norm, ws)
    with pytest.raises(TypeError):
        B.llep_clip_gradients([g], 1.0, norm, ws, out=[g.bfloat16()])
    with pytest.raises(ValueError):
        B.llep_clip_gradients([g], 1.0, norm, ws, out=[])
    with pytest.raises(ValueError):
        B.llep_gradient_norm([torch.ones((4, 4), device=dev).t()], norm, ws)
    with pytest.raises(ValueError):
        B.llep_gradient_norm([torch.ones(4)], norm, ws)
