"""llep_block_norm and its backward on the GPU against the oracle: every gate
shape, with and without each part, rows of one element up to the largest, odd
rows and rows that start off 16-byte boundaries, one row to more rows than
workgroups, in place, on another stream; 8-bit rows; refusals.

Tolerances. A float32 output is a few products of a sum over D <= 8192 terms,
added per thread (at most 32) and over the threads by halves (10 levels), so
its relative error is below 50 * 2^-24 = 3e-6 of the largest magnitude that
enters it; 2e-5 of the largest output is allowed for sums of several such
terms. Column sums run over at most T / 1024 + 1024 / 16 + 16 terms in a
chain: below 100 * 2^-24 = 6e-6 of the sum of their magnitudes; 2e-5 of that.
A bfloat16 output is rounded once: 2^-8 of its value more (half an ulp is
2^-9)."""

import numpy as np
import pytest

import oracle
from gpu_util import device

pytestmark = pytest.mark.gpu

EPS, ALPHA = 1e-5, 0.5


@pytest.fixture(scope="module")
def dev():
    return device()


def _close(what, got, want, dtype, size=None):
    import torch
    got = got.double().cpu().numpy()
    want = np.asarray(want)
    assert got.shape == want.shape, what
    size = np.abs(want).max(initial=0.0) if size is None else size
    tol = 2e-5 * size + (np.abs(want) * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    worst = (np.abs(got - want) - tol).max(initial=-1.0)
    assert worst <= 0, f"{what}: over the tolerance by {worst:.3e}"


def _make(dev, T, D, gate, post, pre, block, dtype, seed, off=0):
    """Inputs; off: elements by which every array starts past an aligned address."""
    import torch
    g = torch.Generator().manual_seed(seed)

    def t(*shape, scale=1.0, mean=0.0):
        n = int(np.prod(shape))
        flat = torch.empty(n + off, dtype=dtype, device=dev)
        v = flat[off:].view(*shape)
        v.copy_((torch.randn(shape, generator=g) * scale + mean).to(dtype))
        return v
    shape = {"none": None, "channel": (1, D), "token": (T, 1), "full": (T, D)}[gate]
    return dict(x=t(T, D, scale=1.5), b=t(T, D) if block else None,
                gate=None if shape is None else t(*shape, scale=0.5, mean=0.5),
                w_post=t(D, scale=0.2, mean=1.0) if post else None,
                w_pre=t(D, scale=0.2, mean=1.0) if pre else None,
                d_r=t(T, D), d_h=t(T, D) if pre else None, empty=lambda: t(T, D))


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _check_both(dev, T, D, gate, post, pre, block, dtype, seed=0, off=0):
    import torch
    from paper_2601_17111_amd import binding as B
    i = _make(dev, T, D, gate, post, pre, block, dtype, seed, off)
    r, h = i["empty"](), i["empty"]() if pre else None
    codes = dict(none=0, channel=1, token=2, full=3)
    args = [i[k] for k in ("b", "gate", "w_post", "w_pre")]
    B.llep_block_norm(i["x"], *args, ALPHA, EPS, r, h, gate_shape=codes[gate])
    want_r, want_h = oracle.block_norm(*map(_np, [i["x"], *args]), ALPHA, EPS)
    _close("r", r, want_r, dtype)
    if pre:
        _close("h", h, want_h, dtype)
    dx, db = i["empty"](), i["empty"]() if block else None
    f32 = dict(dtype=torch.float32, device=dev)
    d_gate = None if i["gate"] is None else torch.full(i["gate"].shape, float("nan"), **f32)
    dw_post = torch.full((D,), float("nan"), **f32) if post else None
    dw_pre = torch.full((D,), float("nan"), **f32) if pre else None
    ws = torch.empty(max(16, B.llep_block_norm_backward_workspace_bytes(T, D)), dtype=torch.uint8,
                     device=dev)
    ws.fill_(0xff)
    B.llep_block_norm_backward(r, *args, ALPHA, EPS, i["d_r"], i["d_h"], dx, db, d_gate, dw_post,
                               dw_pre, ws, gate_shape=codes[gate])
    torch.cuda.synchronize()
    want = oracle.block_norm_backward(_np(r), *map(_np, args), ALPHA, EPS, _np(i["d_r"]),
                                      _np(i["d_h"]))
    _close("dx", dx, want["dx"], dtype)
    if block:
        _close("db", db, want["db"], dtype)
    nb = None if not block else (_np(i["b"]) if not post else oracle.rms_norm(_np(i["b"]), EPS))
    gt = 1.0 if i["gate"] is None else _np(i["gate"])
    if pre:
        size = np.abs(_np(i["d_h"]) * oracle.rms_norm(_np(r), EPS)).sum(0)
        _close("dw_pre", dw_pre, want["dw_pre"], torch.float32, size + 1e-30)
    if post:
        size = np.abs(ALPHA * want["dx"] * gt * nb).sum(0)
        _close("dw_post", dw_post, want["dw_post"], torch.float32, size + 1e-30)
    if i["gate"] is not None:
        terms = np.abs(ALPHA * want["dx"] * nb * (1.0 if not post else _np(i["w_post"])))
        axes = tuple(a for a in (0, 1) if i["gate"].shape[a] == 1)
        size = terms.sum(axis=axes, keepdims=True) if gate in ("channel", "token") else terms.max()
        _close("d_gate", d_gate, want["d_gate"], torch.float32, size + 1e-30)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False), (False, False)])
def test_parts(dev, dtype, gate, post, pre):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for T, D, off in [(1, 8, 0), (5, 72, 0), (3, 33, 0), (7, 64, 1)]:
        _check_both(dev, T, D, gate, post, pre, True, dt, T + D, off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D,off", [
    (1, 1, 0), (2, 7, 0), (1, 255, 0), (3, 512, 0), (3, 520, 0), (2, 1024, 0), (2, 1025, 0),
    (2, 2048, 0), (2, 2056, 0), (2, 2880, 0), (2, 2880, 3), (2, 3001, 0), (2, 4096, 0),
    (2, 4104, 0), (2, 7168, 0), (1, 8191, 0), (2, 8192, 0), (1, 8192, 1),
])
def test_row_lengths(dev, dtype, T, D, off):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    _check_both(dev, T, D, "channel", True, True, True, dt, D, off)
    _check_both(dev, T, D, "none", False, True, False, dt, D, off)


@pytest.mark.parametrize("T", [63, 1023, 1024, 1025, 4099])
def test_many_rows(dev, T):
    import torch
    _check_both(dev, T, 24, "channel", True, True, True, torch.float32, T)
    _check_both(dev, T, 16, "token", True, True, True, torch.bfloat16, T)


def test_no_rows(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    D = 40
    e = torch.empty((0, D), device=dev)
    w = torch.ones(D, device=dev)
    g = torch.ones((1, D), device=dev)
    B.llep_block_norm(e, e, g, w, w, ALPHA, EPS, e, e)
    dg, dw, dv = (torch.full(s, 7.0, device=dev) for s in ((1, D), (D,), (D,)))
    ws = torch.empty(16, dtype=torch.uint8, device=dev)
    B.llep_block_norm_backward(e, e, g, w, w, ALPHA, EPS, e, e, e, e, dg, dw, dv, ws)
    torch.cuda.synchronize()
    assert not dg.any() and not dw.any() and not dv.any()


def test_zero_rows_and_large_values(dev):
    """A row of zeros has finite outputs; values near the type's ends keep
    theirs as the definition in 32 bits has them."""
    import torch
    from paper_2601_17111_amd import binding as B
    for D in (64, 33):
        x = torch.zeros((2, D), device=dev)
        b = torch.zeros((2, D), device=dev)
        x[1], b[1] = 1e15, 1e-15
        w = torch.ones(D, device=dev)
        r, h = torch.empty_like(x), torch.empty_like(x)
        B.llep_block_norm(x, b, None, w, w, 1.0, EPS, r, h)
        want_r, want_h = oracle.block_norm(*map(_np, [x, b]), None, _np(w), _np(w), 1.0, EPS)
        _close("r", r, want_r, torch.float32)
        _close("h", h, want_h, torch.float32)
        # a NaN stays in its own row
        x[0, D // 2] = float("nan")
        B.llep_block_norm(x, b, None, w, w, 1.0, EPS, r, h)
        assert torch.isnan(h[0]).all() and not torch.isnan(h[1]).any()
        assert torch.isnan(r[0]).sum() == 1


@pytest.mark.parametrize("D,off", [(512, 0), (2880, 0), (77, 0), (4104, 0), (2880, 1)])
def test_in_place_and_streams(dev, D, off):
    import torch
    from paper_2601_17111_amd import binding as B
    i = _make(dev, 9, D, "channel", True, True, True, torch.bfloat16, 3, off)
    args = [i[k] for k in ("gate", "w_post", "w_pre")]
    r, h = i["empty"](), i["empty"]()
    B.llep_block_norm(i["x"], i["b"], *args, ALPHA, EPS, r, h)
    x, b = i["empty"](), i["empty"]()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x.copy_(i["x"])
        b.copy_(i["b"])
        B.llep_block_norm(x, b, *args, ALPHA, EPS, x, b)
    side.synchronize()
    assert torch.equal(x, r) and torch.equal(b, h)
    # the backward with dx over d_r and db over d_h, and twice the same bits
    ws = torch.empty(B.llep_block_norm_backward_workspace_bytes(9, D), dtype=torch.uint8,
                     device=dev)
    f = lambda *s: torch.empty(s, dtype=torch.float32, device=dev)  # noqa: E731
    outs = []
    for alias in (False, True, True):
        d_r, d_h = i["empty"](), i["empty"]()
        d_r.copy_(i["d_r"])
        d_h.copy_(i["d_h"])
        dx, db = (d_r, d_h) if alias else (i["empty"](), i["empty"]())
        o = [dx, db, f(1, D), f(D), f(D)]
        B.llep_block_norm_backward(r, i["b"], *args, ALPHA, EPS, d_r, d_h, *o, ws)
        torch.cuda.synchronize()
        outs.append(o)
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_refusals(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    x = torch.zeros((4, 16), device=dev)
    w = torch.ones(16, device=dev)
    ok = dict(x=x, b=x.clone(), gate=None, w_post=w, w_pre=w, alpha=1.0, eps=EPS, r=x.clone(),
              h=x.clone())
    B.llep_block_norm(**ok)
    for bad, err in [
        (dict(b=None), B.LLEPError),                       # w_post without b
        (dict(w_pre=None), B.LLEPError),                   # h without w_pre
        (dict(r=None, h=None), B.LLEPError),               # nothing to write
        (dict(eps=-1.0), B.LLEPError),
        (dict(eps=float("nan")), B.LLEPError),
        (dict(b=x[:3]), ValueError),
        (dict(x=x.t()), ValueError),
        (dict(w_pre=w.bfloat16()), TypeError),
        (dict(x=x.half()), TypeError),
        (dict(gate=torch.ones((4, 2), device=dev)), ValueError),
        (dict(r=torch.zeros((4, 32), device=dev)[:, ::2]), ValueError),
        (dict(h=torch.zeros((4, 16))), ValueError),        # not on a GPU
    ]:
        with pytest.raises(err):
            B.llep_block_norm(**{**ok, **bad})
    big = torch.zeros((1, 8193), device=dev)
    with pytest.raises(B.LLEPError) as ei:
        B.llep_block_norm(big, None, None, None, torch.ones(8193, device=dev), 1.0, EPS, None, big)
    assert ei.value.code == B.LLEP_E_ARG
    f = torch.zeros(16, device=dev)
    ws = torch.empty(16, dtype=torch.uint8, device=dev)
    with pytest.raises(B.LLEPError) as ei:
        B.llep_block_norm_backward(x, x, None, w, w, 1.0, EPS, x, x, x.clone(), x.clone(), None,
                                   f, f.clone(), ws)
    assert ei.value.code == B.LLEP_E_WORKSPACE
    ws = torch.empty(B.llep_block_norm_backward_workspace_bytes(4, 16), dtype=torch.uint8,
                     device=dev)
    with pytest.raises(B.LLEPError):  # w_post without dw_post
        B.llep_block_norm_backward(x, x, None, w, w, 1.0, EPS, x, x, x.clone(), x.clone(), None,
                                   None, f, ws)
