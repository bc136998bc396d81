"""Rows of several wavefronts, several to a workgroup: more rows than workgroups
at D > 512, all of them random, so that what a row leaves in registers or LDS,
or a next row requested too early, would show in its neighbours. Norm forward
and backward, the norm's 8-bit rows, and rows to 8 bits, against the oracle on
every row, with the tolerances of the tests on few rows: column sums run over
at most T / workgroups + 1024 / 16 + 16 terms in a chain, fewer than 100 here."""

import numpy as np
import pytest

import oracle
from gpu_util import device
from test_gpu_int8 import _rows
from test_gpu_norm import ALPHA, EPS, _check_both

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


@pytest.mark.parametrize("T,D,gate,dtype,off", [
    (1777, 2048, "full", "f32", 0), (1100, 2880, "channel", "bf16", 0),
    (1100, 2880, "token", "bf16", 0), (1100, 2880, "full", "bf16", 0),
    (600, 7168, "channel", "f32", 0),      # two vectors a thread in the backward
    (600, 7168, "token", "f32", 0), (900, 7168, "channel", "bf16", 0),
    (2500, 520, "none", "f32", 0), (1500, 1025, "channel", "bf16", 0),
    (600, 2879, "channel", "bf16", 0), (600, 2879, "full", "f32", 0),
    (700, 2880, "token", "bf16", 1),       # whole rows off 16-byte boundaries
])
def test_norm(dev, T, D, gate, dtype, off):
    _check_both(dev, T, D, gate, True, True, True, _dt(dtype), T + D, off)


@pytest.mark.parametrize("T,D,off", [(1100, 2880, 0), (600, 7168, 0), (600, 2879, 0),
                                     (700, 2880, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_without_a_block(dev, T, D, off, dtype):
    _check_both(dev, T, D, "none", False, True, False, _dt(dtype), T, off)


@pytest.mark.parametrize("T,D", [(1100, 2880), (600, 7168), (1100, 2879)])
@pytest.mark.parametrize("block", [False, True])
def test_norm_to_8_bit_rows(dev, T, D, block):
    """Every row's bytes stand for its h: half a step, and what 32-bit sums leave."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = torch.Generator().manual_seed(D)
    x = (torch.randn((T, D), generator=g) * 2).to(dev).bfloat16()
    b = torch.randn((T, D), generator=g).to(dev).bfloat16() if block else None
    wp = (torch.randn(D, generator=g) * 0.2 + 1).to(dev).bfloat16() if block else None
    w = (torch.randn(D, generator=g) * 0.2 + 1).to(dev).bfloat16()
    n = B.llep_int8_row_bytes(D)
    q = torch.full((T, n), 55, dtype=torch.int8, device=dev)
    s = torch.empty(T, device=dev)
    B.llep_block_norm(x, b, None, wp, w, ALPHA, EPS, None, None, q, s)
    torch.cuda.synchronize()
    f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    _, want = oracle.block_norm(f(x), f(b), None, f(wp), f(w), ALPHA, EPS)
    assert not q[:, D:].any()
    sc = f(s)[:, None]
    most = np.abs(want).max(axis=1, keepdims=True)
    assert (np.abs(sc * 127 - most) <= 1e-5 * most).all()
    assert (np.abs(f(q[:, :D]) * sc - want) <= 0.5 * sc * (1 + 1e-4) + 1e-5 * most).all()


@pytest.mark.parametrize("R,D,dtype", [
    (5000, 2880, "bf16"), (5000, 2880, "f32"), (3500, 2879, "bf16"), (3500, 1003, "f32"),
    (2500, 7168, "bf16"), (2500, 9001, "bf16"), (2500, 9008, "f32"),
])
def test_rows_to_8_bits(dev, R, D, dtype):
    import torch
    g = torch.Generator().manual_seed(R + D)
    x = (torch.randn((R, D), generator=g) * torch.rand((R, 1), generator=g) * 3).to(_dt(dtype))
    q, s = _rows(dev, x)
    want_q, want_s = oracle.quantize_rows(x.float().numpy())
    assert np.array_equal(q[:, :D].cpu().numpy(), want_q)
    assert not q[:, D:].any()
    assert np.array_equal(s.cpu().numpy(), want_s)
