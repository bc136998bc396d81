"""The expert layer on 4-bit weights against the oracle: the grouped FFN through
the stream and both heights of tiles, on all devices and on each; LLEPLayer and
ExpertBlock; Router and layer together, in serving and in training.

Tolerance of the grouped FFN: the first products may be off by (D + 32) 2^-23 of
their terms' magnitudes, the activation by (8 + |g|) 2^-22 of itself more (the
exponential's argument is rounded in units of |g|, the rest are a few roundings).
Where that reaches a border between two values of the 4-bit grid, or a block's
next power of two, the output may move by that step times the weight (as computed
by the oracle, element by element); the second product adds (F + 32) 2^-23 of its
terms, a bfloat16 output 2^-8 of its value."""

import math

import numpy as np
import pytest

import oracle
from gpu_util import device, run_plan
from test_gpu_block import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _experts(g, dev, E, D, F):
    """Weights of 4 bits on the GPU, and what they stand for."""
    import torch
    from paper_2601_17111_amd.layer import Mxfp4Experts
    args, values = [], []
    for N, K in ((F, D), (F, D), (D, F)):
        codes = g.integers(0, 16, (E * N, K)).astype(np.uint8)
        e = g.integers(117, 122, (E * N, K // 32)).astype(np.uint8)
        args += [torch.from_numpy(a.reshape(E, N, -1)).to(dev) for a in (oracle.mxfp4_pack(codes), e)]
        values.append(oracle.mxfp4_decode(codes, e).reshape(E, N, K))
    return Mxfp4Experts(*args), values


def _layer(dev, T, K, E, P, D, F, hot, seed):
    """Routing with a share `hot` of the pairs on expert 0, 4-bit rows in plan order."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(seed)
    ids = np.where(g.random((T, K)) < hot, 0, g.integers(0, E, (T, K))).astype(np.int32)
    cap = max(1, -(-T * K * 11 // (10 * P)))
    _, info, (params, bufs, ids_t) = run_plan(ids, E, P, cap, dev=dev)
    x = torch.from_numpy(g.normal(size=(T, D)).astype(np.float32)).to(dev)
    nq, ns = B.llep_mxfp4_row_bytes(D), B.llep_mxfp4_scale_bytes(D)
    rows = torch.empty((T, nq + ns), dtype=torch.uint8, device=dev)
    B.llep_quantize_rows_mxfp4(x, rows[:, :nq], rows[:, nq:])
    xv = oracle.mxfp4_round(x.cpu().numpy())
    experts, w = _experts(g, dev, E, D, F)
    _, row_pair = oracle.permute(
        ids.reshape(-1).tolist(), oracle.plan(ids.reshape(-1).tolist(), E, P, cap), E)
    row_pair = np.asarray(row_pair, dtype=np.int64)
    return locals()


def _run(L, device, dtype):
    """Outputs, and the heights of tiles that the call's list of tiles can be of (its length is at
    the start of the workspace)."""
    import torch
    from paper_2601_17111_amd import binding as B
    dev, D, F = L["dev"], L["D"], L["F"]
    xp = L["rows"][torch.from_numpy(L["row_pair"] // L["K"]).to(dev)]
    out = torch.full((len(xp), D), float("nan"), dtype=dtype, device=dev)
    ws = torch.empty(B.llep_grouped_ffn_mxfp4_workspace_bytes(L["params"], F), dtype=torch.uint8,
                     device=dev)
    ws.fill_(0xff)
    B.llep_grouped_ffn_mxfp4(L["params"], L["bufs"], device, xp, L["experts"].gate_up,
                             L["experts"].down, D, F, out, ws)
    torch.cuda.synchronize()
    n = int(ws[:4].view(torch.int32)[0])
    gb, groups = L["bufs"].group_begin.cpu().tolist(), L["bufs"].groups.cpu().tolist()
    groups = groups[gb[max(device, 0)]:gb[-1 if device < 0 else device + 1]]
    return out, {h for h in (16, 128, 256) if n == sum(-(-m[3] // h) for m in groups)}, groups


def _check(L, out, rows):
    ids = L["ids"].reshape(-1)[L["row_pair"]]
    got = out.double().cpu().numpy()
    for e in np.unique(ids[rows]):
        r = rows[ids[rows] == e]
        want, off = oracle.swiglu_ffn_mxfp4(L["xv"][L["row_pair"][r] // L["K"]], L["w"][0][e],
                                            L["w"][1][e], L["w"][2][e], (L["D"] + 32) * 2.0 ** -23)
        if out.element_size() == 2:
            off = off + 2.0 ** -8 * (np.abs(want) + off)
        assert (np.abs(got[r] - want) <= off).all(), e


@pytest.mark.parametrize("T,K,E,P,D,F,hot,height", [
    (1, 1, 1, 1, 64, 64, 0.0, 16), (1, 4, 8, 4, 128, 192, 0.0, 16), (3, 2, 8, 4, 192, 64, 0.5, 16),
    (20, 4, 16, 4, 256, 320, 0.7, 16), (40, 8, 16, 8, 320, 384, 0.3, 16),
    (70, 2, 4, 1, 448, 128, 0.9, 16), (300, 4, 8, 4, 128, 192, 0.6, 16), (700, 2, 4, 2, 576, 320, 0.8, 16),
    (1100, 1, 2, 1, 64, 64, 0.5, 16), (515, 4, 64, 8, 256, 64, 0.95, 16),
    (600, 2, 4, 2, 1088, 1216, 0.3, 128), (600, 2, 4, 2, 1088, 1216, 0.95, 128),
    (515, 8, 64, 8, 704, 576, 0.6, 128), (2000, 2, 128, 8, 704, 576, 0.2, 256), (1800, 2, 128, 8, 704, 576, 0.2, 128),
    (1201, 1, 2, 1, 1216, 1088, 0.5, 128), (1400, 8, 4, 4, 320, 192, 0.4, 128),
    (1050, 2, 8, 4, 320, 4160, 0.5, 256), (975, 4, 16, 4, 1344, 2112, 0.3, 256),
    (975, 4, 16, 2, 1344, 2112, 0.97, 256), (4000, 4, 32, 4, 192, 1088, 0.5, 256),
])
def test_grouped_ffn(dev, T, K, E, P, D, F, hot, height):
    import torch
    L = _layer(dev, T, K, E, P, D, F, hot, T + E)
    R = T * K
    narrow, forms, groups = _run(L, -1, torch.bfloat16)
    assert height in forms
    edges = [r for _, _, start, n in groups for r in (start, start + n - 1)]
    rows = np.unique(np.concatenate([edges, np.linspace(0, R - 1, min(R, 120))]).astype(int))
    wide, forms, _ = _run(L, -1, torch.float32)
    assert height in forms and not torch.isnan(wide).any()
    assert torch.equal(wide.bfloat16(), narrow)
    _check(L, wide, rows)
    _check(L, narrow, rows)
    for dtype, all_rows in ((torch.bfloat16, narrow), (torch.float32, wide)):
        for d in range(P):  # its rows alone are written, with the same bits
            part, forms, groups = _run(L, d, dtype)
            mine = np.zeros(R, dtype=bool)
            for _, _, start, n in groups:
                mine[start:start + n] = True
            assert not mine.any() or height in forms
            m = torch.from_numpy(mine).to(dev)
            assert torch.equal(part[m], all_rows[m]) and torch.isnan(part[~m]).all()


@pytest.mark.parametrize("T", [1, 37, 900])
def test_layer(dev, T):
    """LLEPLayer.forward_mxfp4 and ExpertBlock.forward_mxfp4: outputs of all pairs, a bad id and a
    pair without an expert left out. The sum of K products in 32 bits adds K 2^-23 of its terms."""
    import torch
    from paper_2601_17111_amd.block import ExpertBlock
    from paper_2601_17111_amd.layer import LLEPLayer
    K, E, P, D, F = 4, 16, 4, 320, 192
    g = np.random.default_rng(T)
    ids = np.where(g.random((T, K)) < 0.4, 0, g.integers(0, E, (T, K))).astype(np.int32)
    ids[0, 0], ids[T // 2, 1] = E, -1
    gates = g.uniform(0, 1, (T, K)).astype(np.float32)
    experts, w = _experts(g, dev, E, D, F)
    layer = LLEPLayer(T, K, E, P, D, F, -(-T * K * 11 // (10 * P)), torch.bfloat16, dev)
    on = [torch.from_numpy(a).to(dev) for a in (ids, gates)]
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.from_numpy(g.normal(size=(T, D))).to(dtype).to(dev)
        y = layer.forward_mxfp4(*on, x, experts).double().cpu().numpy()
        xv = oracle.mxfp4_round(x.double().cpu().numpy())
        want, off = np.zeros((T, D)), np.zeros((T, D))
        for t, k in np.ndindex(T, K):
            if 0 <= ids[t, k] < E and (T < 100 or t % 29 == 0 or t > T - 4):
                e = ids[t, k]
                o, d = oracle.swiglu_ffn_mxfp4(xv[t:t + 1], *(m[e] for m in w), (D + 32) * 2.0 ** -23)
                want[t] += gates[t, k] * o[0]
                off[t] += gates[t, k] * (d[0] + K * 2.0 ** -23 * (np.abs(o[0]) + d[0]))
        off += 2.0 ** -8 * (np.abs(want) + off)
        at = [t for t in range(T) if T < 100 or t % 29 == 0 or t > T - 4]
        assert (np.abs(y[at] - want[at]) <= off[at]).all()
        if dtype == torch.bfloat16:
            # the block's parts one after another
            from paper_2601_17111_amd import binding as B
            v = [torch.rand(D, device=dev).bfloat16() for _ in range(3)]
            block = ExpertBlock(layer, *v[:2], w_next=v[2], alpha=0.5)
            r, h = block.forward_mxfp4(*on, x, experts)
            hx, r2, h2 = (torch.empty_like(x) for _ in range(3))
            B.llep_block_norm(x, None, None, None, v[0], 0.5, block.eps, None, hx)
            B.llep_block_norm(x, layer.forward_mxfp4(*on, hx, experts), None, v[1], v[2], 0.5,
                              block.eps, r2, h2)
            assert torch.equal(r, r2) and torch.equal(h, h2)


@pytest.mark.parametrize("T", [6, 90, 1500])
def test_tokens_that_are_not_finite(dev, T):
    """A token with a NaN or an infinity is NaN, the others are as without it; in the stream and in
    tiles."""
    import torch
    from paper_2601_17111_amd.layer import LLEPLayer
    K, E, P, D, F = 2, 4, 2, 704, 640
    g = np.random.default_rng(T)
    experts, _ = _experts(g, dev, E, D, F)
    ids = torch.from_numpy(g.integers(0, E, (T, K)).astype(np.int32)).to(dev)
    gates = torch.from_numpy(g.uniform(0.1, 1, (T, K)).astype(np.float32)).to(dev)
    x = torch.from_numpy(g.normal(size=(T, D))).to(dev).bfloat16()
    layer = LLEPLayer(T, K, E, P, D, F, -(-T * K * 11 // (10 * P)), torch.bfloat16, dev)
    want = layer.forward_mxfp4(ids, gates, x, experts).clone()
    bad = x.clone()
    bad[1, 3], bad[T - 1, D - 1], bad[T // 2, 40] = math.nan, math.inf, -math.inf
    got = layer.forward_mxfp4(ids, gates, bad, experts)
    rows = torch.zeros(T, dtype=torch.bool, device=dev)
    rows[[1, T // 2, T - 1]] = True
    assert bool(torch.isnan(got[rows]).all()) and torch.equal(got[~rows], want[~rows])


def test_experts_from_weights(dev):
    """from_weights packs the 4-bit rows of the transposed weights."""
    import torch
    from paper_2601_17111_amd.layer import Mxfp4Experts
    E, D, F = 3, 192, 128
    g = torch.Generator().manual_seed(1)
    w = [torch.randn(s, generator=g) * 0.05 for s in ((E, D, F), (E, D, F), (E, F, D))]
    got = Mxfp4Experts.from_weights(*[t.bfloat16().to(dev) for t in w])
    args = []
    for t in w:
        rows = t.bfloat16().double().transpose(1, 2).numpy()
        flat = rows.reshape(-1, rows.shape[2])
        e = oracle.mxfp4_exponents(flat)
        args += [torch.from_numpy(a.reshape(E, rows.shape[1], -1)).to(dev)
                 for a in (oracle.mxfp4_pack(oracle.mxfp4_codes(flat, e)), e)]
    want = Mxfp4Experts(*args)
    assert torch.equal(got.gate_up, want.gate_up) and torch.equal(got.down, want.down)


def test_router_and_layer_serving(dev):
    """Router -> forward_mxfp4, eager, captured and replayed with other tokens, padded rows among
    them, and with a second captured layer that has its own buffers."""
    import torch
    from paper_2601_17111_amd.layer import LLEPLayer, Router
    T, K, E, P, D, F = 50, 4, 16, 4, 320, 192
    g = np.random.default_rng(3)
    experts, _ = _experts(g, dev, E, D, F)
    bias = torch.randn(E, device=dev) * 0.1
    xs = [torch.randn(T, D, device=dev).bfloat16() for _ in range(3)]
    ls = [torch.randn(T, E, device=dev) for _ in range(3)]
    ls[1][40:] = -math.inf  # a padded batch
    make = lambda: (Router(T, K, E, "sigmoid", bias, 4, 2, "top2", scale=2.5),
                    LLEPLayer(T, K, E, P, D, F, -(-T * K * 11 // (10 * P)), torch.bfloat16, dev))
    router, layer = make()

    def call(router, layer, l, x):
        ids, gates = router.forward(l)
        return layer.forward_mxfp4(ids, gates, x, experts)
    want = [call(router, layer, l, x).clone() for l, x in zip(ls, xs)]
    assert not bool(want[1][40:].any()) and all(bool(torch.isfinite(w).all()) for w in want)
    l, x = ls[0].clone(), xs[0].clone()
    graphs = []
    for r, y in (make(), (router, layer)):
        call(r, y, l, x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(r, y, l, x)
        graphs.append((graph, y))
    for i in (1, 2, 0, 1):
        l.copy_(ls[i])
        x.copy_(xs[i])
        for graph, y in graphs:
            y.y.fill_(0)
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y.y, want[i]) for _, y in graphs)


def test_router_and_block_training(dev):
    """Router -> ExpertBlock.forward -> backward -> Router.backward: the gradient of the router's
    logits is the oracle's of the gates' gradients, which the block's own tests hold."""
    import torch
    from paper_2601_17111_amd.layer import Router
    for score in ("softmax", "sigmoid"):
        c = Case(dev, 37, "bf16", "channel", seed=3)
        E, K, T = c.block.layer.E, c.block.layer.K, c.T
        l = torch.randn(T, E, device=dev)
        router = Router(T, K, E, score)
        ids, gates = router.forward(l)
        c.block.forward(ids, gates, c.x, *c.packed)
        _, d_gates, _ = c.block.backward(c.x, c.d_r, c.d_h, gates, c.packed[0], *c.packed_t)
        dl = router.backward(l, d_gates)
        want = oracle.route_backward(l.double().cpu().numpy(), ids.tolist(), d_gates.tolist(), score)
        near = (200 + 2 * K) * 2.0 ** -24 * float(d_gates.abs().max()) * (1 + K)
        assert bool(torch.isfinite(dl).all()) and float(dl.abs().max()) > 0
        assert (np.abs(dl.double().cpu().numpy() - want) <= near).all()


def test_allocations_are_the_streams_own(dev):
    """What calls with stream= allocate is that stream's."""
    import torch
    from paper_2601_17111_amd.layer import Mxfp4Experts, Router
    from test_gpu_stream_buffers import _stream_of, _tensors
    c = Case(dev, 37, "bf16", "channel", seed=3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    layer = c.block.layer
    router = Router(c.T, layer.K, layer.E)
    l = torch.randn(c.T, layer.E, device=dev)
    side.wait_stream(torch.cuda.current_stream())
    here = {**_tensors(layer), **_tensors(router), **_tensors(c.block)}
    experts = Mxfp4Experts.from_weights(*c.w, stream=side)
    ids, gates = router.forward(l, side)
    layer.forward_mxfp4(ids, gates, c.x, experts, stream=side)
    c.block.forward_mxfp4(ids, gates, c.x, experts, stream=side)
    router.backward(l, gates, side)
    side.synchronize()
    made = {**_tensors(layer), **_tensors(router), **_tensors(c.block), **_tensors(experts)}
    made = {k: t for k, t in made.items() if k not in here}
    assert len(made) >= 7
    for k, t in made.items():
        assert _stream_of(t) == side.cuda_stream, k


def test_no_tokens(dev):
    import torch
    from paper_2601_17111_amd.layer import LLEPLayer
    experts, _ = _experts(np.random.default_rng(0), dev, 4, 64, 64)
    layer = LLEPLayer(0, 2, 4, 2, 64, 64, 1, torch.bfloat16, dev)
    y = layer.forward_mxfp4(torch.empty((0, 2), dtype=torch.int32, device=dev),
                            torch.empty((0, 2), device=dev),
                            torch.empty((0, 64), dtype=torch.bfloat16, device=dev), experts)
    torch.cuda.synchronize()
    assert y.shape == (0, 64)


def test_refused_calls_change_nothing(dev):
    """Between a training forward and its backward; and a backward after a serving call is refused."""
    import torch
    from paper_2601_17111_amd.layer import Mxfp4Experts
    c = Case(dev, 37, "bf16", "channel", seed=3)
    layer = c.block.layer
    experts = Mxfp4Experts.from_weights(*c.w)
    other = Mxfp4Experts.from_weights(*[w[:4].contiguous() for w in c.w])

    def back():
        dx, d_gates, grads = c.block.backward(c.x, c.d_r, c.d_h, c.gates, c.packed[0], *c.packed_t)
        torch.cuda.synchronize()
        return [t.clone() for t in (dx, d_gates, *grads.values())]
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    want = back()
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    for args, err in [((c.ids, c.gates, c.x[:, :32].contiguous(), experts), ValueError),
                      ((c.ids, c.gates, c.x[:5], experts), ValueError),
                      ((c.ids, c.gates, c.x.half(), experts), TypeError),
                      ((c.ids, c.gates, c.x.cpu(), experts), ValueError),
                      ((c.ids, c.gates, c.x.t().contiguous().t(), experts), ValueError),
                      ((c.ids.long(), c.gates, c.x, experts), TypeError),
                      ((c.ids[:5], c.gates, c.x, experts), ValueError),
                      ((c.ids, c.gates.bfloat16(), c.x, experts), TypeError),
                      ((c.ids, c.gates, c.x, other), ValueError),
                      ((c.ids, c.gates, c.x, experts, layer.P), ValueError),
                      ((c.ids, c.gates, c.x, experts, -2), ValueError)]:
        with pytest.raises(err):
            layer.forward_mxfp4(*args)
    with pytest.raises(ValueError):
        c.block.forward_mxfp4(c.ids, c.gates, c.x, other)
    assert all(torch.equal(a, b) for a, b in zip(back(), want))
    c.block.forward_mxfp4(c.ids, c.gates, c.x, experts)
    with pytest.raises(RuntimeError):
        back()
    f32 = Case(dev, 5, "f32", "channel", seed=3)
    with pytest.raises(TypeError):
        f32.block.layer.forward_mxfp4(f32.ids, f32.gates, f32.x, Mxfp4Experts.from_weights(*f32.w))


def test_experts_that_do_not_fit_are_refused(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Mxfp4Experts
    z = lambda *s: torch.zeros(s, dtype=torch.uint8, device=dev)
    gate, gs, down, ds = z(2, 128, 32), z(2, 128, 2), z(2, 64, 64), z(2, 64, 4)
    Mxfp4Experts(gate, gs, gate, gs, down, ds)
    for args, err in [((gate, gs, gate, gs, z(2, 128, 64), z(2, 128, 4)), ValueError),
                      ((gate, gs, z(2, 64, 32), z(2, 64, 2), down, ds), ValueError),
                      ((gate, gs[:, :, :1].contiguous(), gate, gs[:, :, :1].contiguous(), down, ds),
                       ValueError),
                      ((gate[0], gs[0], gate[0], gs[0], down[0], ds[0]), ValueError),
                      ((z(2, 96, 48), z(2, 96, 3), z(2, 96, 48), z(2, 96, 3), z(2, 96, 48), z(2, 96, 3)),
                       ValueError),
                      ((gate, gs, gate, gs, down, ds[:, :, :3].contiguous()), ValueError),
                      ((gate.char(), gs, gate.char(), gs, down, ds), TypeError)]:
        with pytest.raises(err):
            Mxfp4Experts(*args)
    L = _layer(dev, 4, 1, 2, 1, 64, 64, 0.0, 0)
    e, x = L["experts"], L["rows"]
    out = torch.empty((4, 64), dtype=torch.bfloat16, device=dev)
    args = (L["params"], L["bufs"])
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    B.llep_grouped_ffn_mxfp4(*args, -1, x, e.gate_up, e.down, 64, 64, out, ws)
    for bad, err in [
        (lambda: B.llep_grouped_ffn_mxfp4(*args, 1, x, e.gate_up, e.down, 64, 64, out, ws), B.LLEPError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x, e.gate_up, e.down, 64, 64, out, ws[:16]),
         B.LLEPError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x, e.gate_up, e.down, 64, 64, out, ws[16:]),
         B.LLEPError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x[:3], e.gate_up, e.down, 64, 64, out, ws),
         ValueError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x, e.gate_up, e.down, 64, 192, out, ws), ValueError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x, e.gate_up[:1], e.down, 64, 64, out, ws),
         ValueError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x, e.gate_up, e.down, 64, 64, out.half(), ws),
         TypeError),
        (lambda: B.llep_grouped_ffn_mxfp4(*args, -1, x[:, :64].contiguous(), e.gate_up, e.down, 64, 64,
                                          out, ws), ValueError),
    ]:
        with pytest.raises(err):
            bad()
    torch.cuda.synchronize()
