"""ExpertBlock: norms, experts, gate, residual and clipping run together, in
training (float32 and bf16) and in serving with 8-bit experts, against the
oracle's definitions put together the same way; the norm's 8-bit rows; and the
norm's gradients against central differences.

Tolerances, on the largest entry: float32 1e-4 (the float32 layer keeps 1e-5
of its own outputs, and the norms after it divide by values near 1); bf16 5e-2
(2e-2 for the layer, whose inputs and outputs are rounded to bf16 and pass
through three norms); 8 bits as for the layer on its own, 6% of the 2-norm."""

import numpy as np
import pytest

import oracle
from gpu_util import device

pytestmark = pytest.mark.gpu

EPS, ALPHA = 1e-5, 0.5


@pytest.fixture(scope="module")
def dev():
    return device()


class Case:
    def __init__(self, dev, T, dtype, gate, seed=0, K=2, E=8, P=4, D=64, F=128):
        import torch
        from paper_2601_17111_amd import binding as B
        from paper_2601_17111_amd.block import ExpertBlock
        from paper_2601_17111_amd.layer import LLEPLayer
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        g = torch.Generator().manual_seed(seed)

        def t(*shape, scale=1.0, mean=0.0):
            return (torch.randn(shape, generator=g) * scale + mean).to(dev).to(self.dt)
        self.T, self.K, self.E, self.D, self.F = T, K, E, D, F
        self.x = t(T, D)
        self.w = [t(E, D, F, scale=0.2), t(E, D, F, scale=0.2), t(E, F, D, scale=0.2)]
        self.ids = torch.randint(0, E, (T, K), generator=g).to(torch.int32).to(dev)
        self.gates = torch.softmax(torch.randn((T, K), generator=g), -1).to(dev)
        shape = {"none": None, "channel": (1, D), "token": (T, 1), "full": (T, D)}[gate]
        self.gate = None if shape is None else t(*shape, scale=0.3, mean=0.5)
        self.w_pre, self.w_post, self.w_next = (t(D, scale=0.2, mean=1.0) for _ in range(3))
        self.d_r, self.d_h = t(T, D), t(T, D)
        layer = LLEPLayer(T, K, E, P, D, F, -(-T * K * 5 // (4 * P)), self.dt, dev)
        self.block = ExpertBlock(layer, self.w_pre, self.w_post, self.gate, self.w_next, ALPHA, EPS)
        self.packed = B.llep_pack_weights(*self.w)
        self.packed_t = B.llep_pack_weights_backward(*self.w)

    def f64(self, t):
        return None if t is None else t.double().cpu().numpy()

    def oracle_forward(self):
        _, h = oracle.block_norm(self.f64(self.x), None, None, None, self.f64(self.w_pre), ALPHA,
                                 EPS)
        W = [self.f64(w) for w in self.w]
        ids, gates = self.ids.cpu().numpy(), self.gates.cpu().numpy()
        y = oracle.moe_output(h, ids, gates, lambda e: (W[0][e], W[1][e], W[2][e]))
        r, hn = oracle.block_norm(self.f64(self.x), y, self.f64(self.gate), self.f64(self.w_post),
                                  self.f64(self.w_next), ALPHA, EPS)
        return h, y, r, hn

    def oracle_backward(self):
        h, y, r, _ = self.oracle_forward()
        a = oracle.block_norm_backward(r, y, self.f64(self.gate), self.f64(self.w_post),
                                       self.f64(self.w_next), ALPHA, EPS, self.f64(self.d_r),
                                       self.f64(self.d_h))
        W = [self.f64(w) for w in self.w]
        dh, d_gates, dW = oracle.moe_backward(
            h, self.ids.cpu().numpy(), self.gates.cpu().numpy(),
            lambda e: (W[0][e], W[1][e], W[2][e]), a["db"], self.E)
        b = oracle.block_norm_backward(self.f64(self.x), None, None, None, self.f64(self.w_pre),
                                       ALPHA, EPS, a["dx"], dh)
        grads = {k: np.zeros(tuple(w.shape)) for k, w in zip(("w_gate", "w_up", "w_down"), self.w)}
        for e, parts in dW.items():
            for k, p in zip(("w_gate", "w_up", "w_down"), parts):
                grads[k][e] = p
        grads["w_pre"], grads["w_post"], grads["w_next"] = b["dw_pre"], a["dw_post"], a["dw_pre"]
        if self.gate is not None:
            grads["gate"] = a["d_gate"]
        return b["dx"], d_gates, grads


def _near(what, got, want, tol):
    got = got.double().cpu().numpy()
    err = np.abs(got - want).max() / np.abs(want).max()
    print(f"[{what}] {err:.2e}", flush=True)
    assert got.shape == want.shape and err <= tol, what


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 5e-2)])
@pytest.mark.parametrize("T,gate", [(1, "channel"), (37, "token"), (300, "full"), (300, "none")])
def test_training_step(dev, T, gate, dtype, tol):
    import torch
    c = Case(dev, T, dtype, gate, seed=T)
    r, h_next = c.block.forward(c.ids, c.gates, c.x, *c.packed)
    dx, d_gates, grads = c.block.backward(c.x, c.d_r, c.d_h, c.gates, c.packed[0], *c.packed_t)
    torch.cuda.synchronize()
    _, _, want_r, want_h = c.oracle_forward()
    _near("r", r, want_r, tol)
    _near("h_next", h_next, want_h, tol)
    want_dx, want_dg, want = c.oracle_backward()
    _near("dx", dx, want_dx, tol)
    _near("d_gates", d_gates, want_dg, tol)
    assert set(grads) == set(want)
    for k in want:
        _near(k, grads[k], want[k], tol)
    # the gradients of the whole block clipped by their norm
    before = [g.double().cpu().numpy() for g in grads.values()]
    exact = oracle.gradient_norm(before)
    norm = c.block.clip(grads, 0.5 * exact)
    torch.cuda.synchronize()
    assert abs(float(norm) - exact) <= 2.0 ** -23 * exact
    for g, b in zip(grads.values(), before):
        assert np.allclose(g.double().cpu().numpy(), 0.5 * b, rtol=1e-6, atol=0)


@pytest.mark.parametrize("T", [1, 37, 500])
def test_serving_with_8_bit_experts(dev, T):
    import torch
    from paper_2601_17111_amd.layer import Int8Experts
    c = Case(dev, T, "bf16", "channel", seed=T + 1)
    _, _, want_r, want_h = c.oracle_forward()
    r, h = c.block.forward_int8(c.ids, c.gates, c.x, Int8Experts.from_weights(*c.w))
    torch.cuda.synchronize()
    for what, got, want in (("r", r, want_r), ("h_next", h, want_h)):
        err = np.linalg.norm(c.f64(got) - want) / np.linalg.norm(want)
        print(f"[{what} T={T}] {err:.3e}", flush=True)
        assert err <= 0.06


@pytest.mark.parametrize("D,off", [(64, 0), (512, 0), (520, 0), (2880, 0), (7168, 0), (100, 0),
                                   (2001, 0), (512, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_to_8_bit_rows(dev, D, off, dtype):
    """The norm's 8-bit rows stand for its h: within half a step and what 32-bit sums leave."""
    import torch
    from paper_2601_17111_amd import binding as B
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    T = 6
    g = torch.Generator().manual_seed(D)
    flat = torch.empty(T * D + off, dtype=dt, device=dev)
    x = flat[off:].view(T, D)
    x.copy_(torch.randn((T, D), generator=g) * 2)
    x[2] = 0
    x[3, D // 2] = float("inf")
    w = (torch.randn(D, generator=g) * 0.2 + 1).to(dev).to(dt)
    n = B.llep_int8_row_bytes(D)
    q = torch.full((T, n), 55, dtype=torch.int8, device=dev)
    s = torch.empty(T, device=dev)
    h = torch.empty_like(x)
    B.llep_block_norm(x, None, None, None, w, 1.0, EPS, None, h, q, s)
    alone_q, alone_s = torch.empty_like(q), torch.empty_like(s)
    B.llep_block_norm(x, None, None, None, w, 1.0, EPS, None, None, alone_q, alone_s)
    torch.cuda.synchronize()
    assert torch.equal(q, alone_q) and torch.equal(torch.nan_to_num(s, 3.0),
                                                   torch.nan_to_num(alone_s, 3.0))
    assert not q[:, D:].any() and not q[2].any() and float(s[2]) == 0
    assert torch.isnan(s[3]) and not q[3].any()
    rows = [0, 1, 4, 5]
    _, want = oracle.block_norm(x[rows].double().cpu().numpy(), None, None, None,
                                w.double().cpu().numpy(), 1.0, EPS)
    sc = s[rows].double().cpu().numpy()[:, None]
    most = np.abs(want).max(axis=1, keepdims=True)
    assert (np.abs(sc * 127 - most) <= 1e-5 * most).all()
    got = q[rows, :D].double().cpu().numpy() * sc
    assert (np.abs(got - want) <= 0.5 * sc * (1 + 1e-4) + 1e-5 * most).all()


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("D", [64, 37])
def test_norm_gradients_against_differences(dev, gate, D):
    """The gradients on the GPU (float32), along random directions, against central differences of
    the definition in 64 bits: differences of step h are off by h^2 / 6 times a third derivative,
    below 1e-7 here; the gradients by 1e-5 of their size."""
    import torch
    from paper_2601_17111_amd import binding as B
    T = 9
    g = np.random.default_rng(D)
    shape = {"none": None, "channel": (1, D), "token": (T, 1), "full": (T, D)}[gate]
    host = [g.standard_normal((T, D)), g.standard_normal((T, D)),
            None if shape is None else g.standard_normal(shape) * 0.3 + 0.5,
            g.standard_normal(D) * 0.2 + 1, g.standard_normal(D) * 0.2 + 1]
    host = [None if a is None else a.astype(np.float32).astype(np.float64) for a in host]
    d_r, d_h = (g.standard_normal((T, D)).astype(np.float32) for _ in range(2))

    def loss(a):
        r, h = oracle.block_norm(*a, ALPHA, EPS)
        return np.sum(r * d_r) + np.sum(h * d_h)

    t = [None if a is None else torch.from_numpy(a.astype(np.float32)).to(dev) for a in host]
    r = torch.empty_like(t[0])
    h = torch.empty_like(r)
    B.llep_block_norm(*t, ALPHA, EPS, r, h)
    f = lambda a: None if a is None else torch.empty(a.shape, device=dev)  # noqa: E731
    dx, db, dg, dpost, dpre = (f(a) for a in t)
    ws = torch.empty(B.llep_block_norm_backward_workspace_bytes(T, D), dtype=torch.uint8,
                     device=dev)
    B.llep_block_norm_backward(r, *t[1:], ALPHA, EPS, torch.from_numpy(d_r).to(dev),
                               torch.from_numpy(d_h).to(dev), dx, db, dg, dpost, dpre, ws)
    torch.cuda.synchronize()
    for i, grad in enumerate((dx, db, dg, dpost, dpre)):
        if grad is None:
            continue
        gr = grad.double().cpu().numpy()
        for k in range(3):
            v = g.standard_normal(host[i].shape)
            two = []
            for step in (1e-4, -1e-4):
                moved = list(host)
                moved[i] = host[i] + step * v
                two.append(loss(moved))
            want = (two[0] - two[1]) / 2e-4
            assert abs(np.sum(gr * v) - want) <= 1e-5 * np.sum(np.abs(gr * v)) + 1e-5, (i, k)


def test_serving_in_a_graph(dev):
    """Norm, 8-bit experts, norm and gate, and an 8-bit projection, captured once and replayed with
    other inputs in between: every replay as the eager calls."""
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts
    for T in (3, 700):
        c = Case(dev, T, "bf16", "channel", seed=T + 2)
        experts = Int8Experts.from_weights(*c.w)
        wq = torch.randint(-127, 128, (96, c.D), device=dev, dtype=torch.int8)
        ws = torch.rand(96, device=dev)
        packed = B.llep_pack_matrix_int8(wq)
        q = torch.empty((T, c.D), dtype=torch.int8, device=dev)
        s = torch.empty(T, device=dev)
        out = torch.empty((T, 96), device=dev)

        def step(x):
            r, h = c.block.forward_int8(c.ids, c.gates, x, experts)
            B.llep_quantize_rows(h, q, s)
            B.llep_int8_matmul(q, s, packed, ws, out, c.D)
            return r
        x = c.x.clone()
        step(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(x)
        for k in range(3):
            x.copy_(c.x * (1 + 0.1 * k))
            graph.replay()
            torch.cuda.synchronize()
            got = (c.block.r.clone(), out.clone())
            want_r = step(x.clone()).clone()
            torch.cuda.synchronize()
            assert torch.equal(got[0], want_r) and torch.equal(got[1], out)


def test_misuse_is_refused(dev):
    """What would read past a tensor, or another call's rows, raises."""
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts
    T, D = 5, 64
    x = torch.zeros((T, D), device=dev)
    w = torch.ones(D, device=dev)
    for gate, shape in [(torch.ones((1, D), device=dev), B.LLEP_GATE_FULL),
                        (torch.ones((1, D), device=dev), B.LLEP_GATE_TOKEN),
                        (torch.ones((T, 1), device=dev), B.LLEP_GATE_CHANNEL),
                        (torch.ones((T, D), device=dev), B.LLEP_GATE_NONE),
                        (torch.ones((T, D), device=dev), 9), (None, B.LLEP_GATE_FULL)]:
        with pytest.raises(ValueError):
            B.llep_block_norm(x, x.clone(), gate, w, w, 1.0, EPS, x.clone(), gate_shape=shape)
    g = torch.ones(8, device=dev)
    norm = torch.zeros(1, device=dev)
    n = B.llep_clip_gradients_workspace_bytes()
    for ws in (torch.zeros(n, dtype=torch.uint8), torch.zeros((n, 2), dtype=torch.uint8,
                                                              device=dev)[:, 0]):
        with pytest.raises(ValueError):
            B.llep_gradient_norm([g], norm, ws)
    with pytest.raises(B.LLEPError) as ei:
        B.llep_gradient_norm([g], norm, None)
    assert ei.value.code == B.LLEP_E_WORKSPACE
    c = Case(dev, 8, "bf16", "none")
    experts = Int8Experts.from_weights(*c.w)
    c.block.forward_int8(c.ids, c.gates, c.x, experts)
    with pytest.raises(RuntimeError):
        c.block.backward(c.x, c.d_r, c.d_h, c.gates, c.packed[0], *c.packed_t)
    with pytest.raises(ValueError):
        c.block.layer.forward_int8(c.ids, c.gates, c.x[:, :32].contiguous(), experts)
    with pytest.raises(ValueError):  # 8-bit rows of another width
        c.block.layer.forward_int8(c.ids, c.gates, torch.zeros((8, 128), dtype=torch.int8,
                                                               device=dev), experts, -1, None,
                                   torch.zeros(8, device=dev))
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    c.block.backward(c.x, c.d_r, c.d_h, c.gates, c.packed[0], *c.packed_t)
    torch.cuda.synchronize()
