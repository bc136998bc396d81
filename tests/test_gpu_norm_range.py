"""The backward of the block norm where values are far from 1, or not finite.

Rows of 1e15 and of 1e-15 (eps = 0) have gradients of 1e-15 to 1e30, all of
them in the range of 32 bits; the cube of a row's factor, 1e45, is not.
Tolerance: as for rows near 1 (2e-5 of the largest output, a bfloat16 one 2^-8
of its value more), for every row by itself."""

import numpy as np
import pytest

import oracle
from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _np(t):
    return t.double().cpu().numpy()


# whole rows (one vector a thread; two, for long float32 rows), odd rows, and
# whole rows that start off 16-byte boundaries
@pytest.mark.parametrize("D,off", [(64, 0), (2880, 0), (4104, 0), (33, 0), (64, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_and_small_rows(dev, dtype, D, off):
    import torch
    from paper_2601_17111_amd import binding as B
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(D)
    size = torch.tensor([1e15, 1e-15, 1.0, 1e-15, 1e15, 1.0]).view(-1, 1)
    T = len(size)

    def t(v):
        flat = torch.empty(v.numel() + off, dtype=dt, device=dev)
        flat[off:].view(v.shape).copy_(v)
        return flat[off:].view(v.shape)
    r = t(torch.randn((T, D), generator=g) * size)
    b = t(torch.randn((T, D), generator=g) * size)
    w_post, w_pre = (t(torch.randn(D, generator=g) * 0.2 + 1) for _ in range(2))
    d_r, d_h = t(torch.zeros((T, D))), t(torch.randn((T, D), generator=g))
    dx, db = t(torch.zeros((T, D))), t(torch.zeros((T, D)))
    dpost, dpre = torch.empty(D, device=dev), torch.empty(D, device=dev)
    ws = torch.empty(B.llep_block_norm_backward_workspace_bytes(T, D), dtype=torch.uint8,
                     device=dev)
    B.llep_block_norm_backward(r, b, None, w_post, w_pre, 0.5, 0.0, d_r, d_h, dx, db, None, dpost,
                               dpre, ws)
    torch.cuda.synchronize()
    want = oracle.block_norm_backward(_np(r), _np(b), None, _np(w_post), _np(w_pre), 0.5, 0.0,
                                      _np(d_r), _np(d_h))
    for name, got in (("dx", dx), ("db", db)):
        w = want[name]
        tol = 2e-5 * np.abs(w).max(axis=1, keepdims=True)
        if dtype == "bf16":
            tol = tol + 2.0 ** -8 * np.abs(w)
        off_by = np.abs(_np(got) - w) - tol
        assert not np.isnan(off_by).any() and off_by.max() <= 0, name
    terms = np.abs(_np(d_h) * oracle.rms_norm(_np(r), 0.0)).sum(0)
    assert (np.abs(_np(dpre) - want["dw_pre"]) <= 2e-5 * terms).all()
    terms = np.abs(0.5 * want["dx"] * oracle.rms_norm(_np(b), 0.0)).sum(0)
    assert (np.abs(_np(dpost) - want["dw_post"]) <= 2e-5 * terms).all()


@pytest.mark.parametrize("D", [64, 33])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_outputs_not_finite_without_their_norm(dev, gate, D):
    """Without w_post, db = alpha gate dx has nothing of b: an infinity or a NaN there (of a place
    that the next step masks, say) reaches neither db nor dx."""
    import torch
    from paper_2601_17111_amd import binding as B
    T = 3
    g = torch.Generator().manual_seed(D)
    b = torch.randn((T, D), generator=g).to(dev)
    b[0, 3], b[1, 0], b[2, D - 1] = float("inf"), -float("inf"), float("nan")
    shape = {"none": None, "channel": (1, D), "token": (T, 1), "full": (T, D)}[gate]
    gt = None if shape is None else torch.randn(shape, generator=g).to(dev)
    d_r = torch.randn((T, D), generator=g).to(dev)
    dx, db = torch.empty_like(b), torch.empty_like(b)
    d_gate = None if gt is None else torch.empty_like(gt)
    ws = torch.empty(B.llep_block_norm_backward_workspace_bytes(T, D), dtype=torch.uint8,
                     device=dev)
    B.llep_block_norm_backward(None, b, gt, None, None, 0.5, 1e-5, d_r, None, dx, db, d_gate, None,
                               None, ws, gate_shape=dict(none=0, channel=1, token=2, full=3)[gate])
    torch.cuda.synchronize()
    assert torch.equal(dx, d_r)
    want = 0.5 * d_r * (1.0 if gt is None else gt)
    assert bool(((db - want).abs() <= 2.0 ** -22 * want.abs()).all())
