"""8-bit rows, products and the expert layer on 8-bit weights against the
oracle: rows bit for bit; products over lengths from one to the largest k, odd
sizes, one row to several tiles; the same bits from every kernel; the grouped
FFN through the weight stream and the tiles, on one device's groups and on
all; refusals.

Tolerances. A product is an exact sum, rounded to 32 bits, times two scales:
three roundings, 2^-22 of the value allowed; a bfloat16 one is rounded once
more (2^-8 allowed). The grouped FFN's activations carry errors of 32-bit
arithmetic (below 2e-6 of the value), so that of a row's F values about F 127
4e-6 (0.2 at F = 384) lie near enough to a tie to round to the other side, each
worth one step of the row's activation scale times the largest weight; five
such steps are allowed, and 2e-5 of the largest output."""

import numpy as np
import pytest

import oracle
from gpu_util import device, run_plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _rows(dev, x, off=0):
    """llep_quantize_rows of a float tensor on the host."""
    import torch
    from paper_2601_17111_amd import binding as B
    flat = torch.empty(x.numel() + off, dtype=x.dtype, device=dev)
    xd = flat[off:].view(x.shape)
    xd.copy_(x)
    q = torch.full((x.shape[0], B.llep_int8_row_bytes(x.shape[1])), 77, dtype=torch.int8,
                   device=dev)
    s = torch.full((x.shape[0],), -1.0, device=dev)
    B.llep_quantize_rows(xd, q, s)
    torch.cuda.synchronize()
    return q, s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,D,off", [
    (0, 5, 0), (1, 1, 0), (3, 8, 0), (5, 63, 0), (4, 64, 1), (2, 1000, 0), (3, 1001, 0),
    (3, 2048, 0), (2, 2880, 0), (2, 2880, 1), (2, 4104, 0), (2, 7168, 0), (2, 8200, 0),
    (1, 9001, 0), (1, 65536, 0), (1, 65535, 0), (1027, 72, 0),
])
def test_rows(dev, dtype, R, D, off):
    import torch
    g = torch.Generator().manual_seed(R + D)
    x = torch.randn((R, D), generator=g) * 3
    if R > 2:
        x[1] = 0
        x[2] *= 1e-20
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, s = _rows(dev, x, off)
    want_q, want_s = oracle.quantize_rows(x.float().numpy())
    assert np.array_equal(q[:, :D].cpu().numpy(), want_q)
    assert not q[:, D:].any()
    assert np.array_equal(s.cpu().numpy(), want_s)


@pytest.mark.parametrize("D", [8, 37, 4096, 9001])
def test_rows_not_finite_and_tiny(dev, D):
    import torch
    x = torch.ones((7, D))
    x[0, D - 1] = float("nan")
    x[1, 0] = float("inf")
    x[2, D // 2] = -float("inf")
    x[3] = 1e-37
    x[4] = torch.finfo(torch.float32).max
    x[5] = 2.0 ** -120
    x[6, 0] = -float("nan")
    q, s = _rows(dev, x)
    want_q, want_s = oracle.quantize_rows(x.numpy())
    assert np.array_equal(q[:, :D].cpu().numpy(), want_q)
    assert np.array_equal(s.cpu().numpy(), want_s, equal_nan=True)


def _matrix(g, N, K):
    return (g.integers(-127, 128, (N, K)).astype(np.int8),
            (g.uniform(0.5, 1.5, N) * 0.01).astype(np.float32))


def _product(dev, q, s, w, ws, K, dtype):
    import torch
    from paper_2601_17111_amd import binding as B
    M, N = q.shape[0], w.shape[0]
    out = torch.full((M, N), float("nan"), dtype=dtype, device=dev)
    work = torch.empty(B.llep_int8_matmul_workspace_bytes(M, N, K), dtype=torch.uint8, device=dev)
    work.fill_(0xff)
    packed = B.llep_pack_matrix_int8(torch.from_numpy(w).to(dev))
    B.llep_int8_matmul(q, s, packed, torch.from_numpy(ws).to(dev), out, K, work)
    torch.cuda.synchronize()
    return out


def _bytes(dev, q):
    """Whole numbers as the padded rows that llep_int8_matmul takes."""
    import torch
    M, K = q.shape
    out = torch.zeros((M, -(-K // 64) * 64), dtype=torch.int8)
    out[:, :K] = torch.from_numpy(q)
    return out.to(dev)


def _check_product(dev, M, N, K, dtype, seed=0):
    import torch
    g = np.random.default_rng(seed)
    q = g.integers(-127, 128, (M, K)).astype(np.int8)
    s = (g.uniform(0.5, 1.5, M) * 0.01).astype(np.float32)
    w, ws = _matrix(g, N, K)
    out = _product(dev, _bytes(dev, q), torch.from_numpy(s).to(dev), w, ws, K, dtype)
    # whole-number products in float64: exact below 2^53
    want = (q.astype(np.float64) @ w.astype(np.float64).T) * s[:, None].astype(np.float64) \
        * ws[None, :].astype(np.float64)
    tol = (2.0 ** -22 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * np.abs(want)
    err = np.abs(out.double().cpu().numpy() - want) - tol
    assert not np.isnan(err).any() and err.max(initial=-1.0) <= 0, (M, N, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [
    (0, 8, 8), (1, 1, 1), (1, 16, 64), (1, 2880, 2880), (2, 3, 65), (3, 17, 63), (15, 64, 128),
    (16, 65, 130), (17, 100, 192), (31, 257, 1003), (33, 48, 1000), (63, 193, 64), (64, 256, 320),
    (65, 16, 64), (65, 255, 100), (100, 1, 200), (129, 512, 448), (255, 384, 512), (256, 192, 64),
    (257, 600, 300), (333, 2881, 1003), (513, 264, 192), (1000, 130, 5000), (2, 40, 65536),
    (70, 20, 65536), (1500, 1200, 256), (4, 5000, 257),
])
def test_product(dev, dtype, M, N, K):
    import torch
    _check_product(dev, M, N, K, torch.bfloat16 if dtype == "bf16" else torch.float32, M + N + K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K", [
    # 128-row tiles: one to three slices of k and more, a last tile of few rows
    # or columns, odd rows and columns, fewer tiles than workgroups and more
    (1800, 1800, 64), (1793, 1801, 130), (130, 30001, 70), (1500, 3001, 501), (2050, 1288, 1300),
    (2500, 4104, 200),
    # 256-row tiles
    (3000, 3001, 700), (3001, 5000, 1000),
])
def test_product_of_many_rows(dev, dtype, M, N, K):
    import torch
    _check_product(dev, M, N, K, torch.bfloat16 if dtype == "bf16" else torch.float32, M + N + K)


@pytest.mark.parametrize("M", [1, 16, 20, 64, 65, 300])
def test_largest_sums(dev, M):
    """Every product 127 * -127 over the largest k: whole numbers near 2^30."""
    import torch
    K, N = 65536, 33
    q = np.full((M, K), 127, dtype=np.int8)
    w = np.full((N, K), -127, dtype=np.int8)
    one = torch.ones(M, device=dev)
    out = _product(dev, _bytes(dev, q), one, w, np.ones(N, dtype=np.float32), K, torch.float32)
    assert (out == float(-127 * 127 * K)).all()


def test_same_bits_for_any_number_of_rows(dev):
    """A row's product does not depend on the rows beside it, so on the kernel that ran."""
    import torch
    g = np.random.default_rng(1)
    M, N, K = 700, 530, 1100
    q = _bytes(dev, g.integers(-127, 128, (M, K)).astype(np.int8))
    s = torch.rand(M, device=dev) + 0.1
    w, ws = _matrix(g, N, K)
    for dtype in (torch.bfloat16, torch.float32):
        whole = _product(dev, q, s, w, ws, K, dtype)
        for m in (1, 5, 16, 17, 32, 33, 64, 65, 100, 128, 129, 256, 257, 400, 512, 513):
            assert torch.equal(_product(dev, q[:m], s[:m], w, ws, K, dtype), whole[:m]), m


def test_scales_not_finite(dev):
    """A row that was not finite gives NaN in its own outputs alone."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(2)
    for M in (5, 300):
        x = torch.randn((M, 128))
        x[3, 7] = float("nan")
        q, s = _rows(dev, x)
        w, ws = _matrix(g, 64, 128)
        out = _product(dev, q, s, w, ws, 128, torch.float32)
        bad = torch.isnan(out)
        assert bad[3].all() and int(bad.sum()) == 64


def _layer(dev, T, K, E, P, D, F, hot, seed):
    """Routing with a share `hot` of the pairs on expert 0, 8-bit weights, rows in plan order."""
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts
    g = np.random.default_rng(seed)
    ids = np.where(g.random((T, K)) < hot, 0, g.integers(0, E, (T, K))).astype(np.int32)
    cap = max(1, -(-T * K * 11 // (10 * P)))
    _, info, (params, bufs, ids_t) = run_plan(ids, E, P, cap, dev=dev)
    x = g.integers(-127, 128, (T, D)).astype(np.int8)
    s = (g.uniform(0.5, 1.5, T) * 0.02).astype(np.float32)
    w = [g.integers(-127, 128, sh).astype(np.int8) for sh in ((E, F, D), (E, F, D), (E, D, F))]
    sc = [(g.uniform(0.5, 1.5, sh) * 0.0003).astype(np.float32) for sh in ((E, F), (E, F), (E, D))]
    experts = Int8Experts(*[torch.from_numpy(a).to(dev) for pair in zip(w, sc) for a in pair])
    pair_row, row_pair = oracle.permute(
        ids.reshape(-1).tolist(), oracle.plan(ids.reshape(-1).tolist(), E, P, cap), E)
    row_pair = np.asarray(row_pair, dtype=np.int64)
    return locals()


def _ffn(L, device, by_row=False):
    import torch
    from paper_2601_17111_amd import binding as B
    dev, e = L["dev"], L["experts"]
    tok = L["row_pair"] // L["K"]
    xp = torch.from_numpy(L["x"][tok]).to(dev)
    rp = torch.from_numpy(L["row_pair"].astype(np.int32)).to(dev)
    s = torch.from_numpy(L["s"][tok] if by_row else L["s"]).to(dev)
    out = torch.full((len(tok), L["D"]), float("nan"), dtype=torch.bfloat16, device=dev)
    ws = torch.empty(B.llep_grouped_ffn_int8_workspace_bytes(L["params"], L["F"]),
                     dtype=torch.uint8, device=dev)
    ws.fill_(0xff)
    B.llep_grouped_ffn_int8(L["params"], L["bufs"], device, xp, s, None if by_row else rp,
                            e.gate_up, e.gate_scale, e.up_scale, e.down, e.down_scale, out, ws)
    torch.cuda.synchronize()
    return out


def _check_ffn(L, out, rows):
    ids = L["ids"].reshape(-1)[L["row_pair"]]
    got = out.double().cpu().numpy()
    for e in np.unique(ids[rows]):
        r = rows[ids[rows] == e]
        tok = L["row_pair"][r] // L["K"]
        want, most = oracle.swiglu_ffn_int8(
            L["x"][tok], L["s"][tok], L["w"][0][e], L["sc"][0][e], L["w"][1][e], L["sc"][1][e],
            L["w"][2][e], L["sc"][2][e])
        biggest = 127 * L["sc"][2][e].max()
        tol = (5 * most[:, None] / 127 * biggest + 2.0 ** -8 * np.abs(want)
               + 2e-5 * np.abs(want).max())
        assert (np.abs(got[r] - want) <= tol).all(), e


@pytest.mark.parametrize("T,K,E,P,D,F,hot", [
    (1, 1, 1, 1, 64, 64, 0.0), (1, 4, 8, 4, 128, 192, 0.0), (3, 2, 8, 4, 192, 64, 0.5),
    (20, 4, 16, 4, 256, 320, 0.7), (40, 8, 16, 8, 320, 384, 0.3), (70, 2, 4, 1, 448, 128, 0.9),
    (130, 2, 16, 4, 192, 256, 0.6),                    # the stream, pieces of 64 rows
    (300, 4, 8, 4, 128, 192, 0.6),                     # tiles
    (700, 2, 4, 2, 576, 320, 0.8),                     # tiles of 192 columns for D
    (1100, 1, 2, 1, 64, 64, 0.5), (515, 4, 64, 8, 256, 64, 0.95),
])
def test_grouped_ffn(dev, T, K, E, P, D, F, hot):
    import torch
    L = _layer(dev, T, K, E, P, D, F, hot, T + E)
    R = T * K
    rows = np.unique(np.linspace(0, R - 1, min(R, 160)).astype(int))
    out = _ffn(L, -1)
    assert not torch.isnan(out).any()
    _check_ffn(L, out, rows)
    assert torch.equal(_ffn(L, -1, by_row=True), out)
    # one device's groups: its rows alone are written, with the same bits
    gb = L["bufs"].group_begin.cpu().tolist()
    groups = L["bufs"].groups.cpu().tolist()
    for d in range(P):
        part = _ffn(L, d)
        mine = np.zeros(R, dtype=bool)
        for _, _, start, n in groups[gb[d]:gb[d + 1]]:
            mine[start:start + n] = True
        m = torch.from_numpy(mine).to(dev)
        assert torch.equal(part[m], out[m]) and torch.isnan(part[~m]).all()


def test_grouped_ffn_sizes_of_calls_agree(dev):
    """The stream's pieces of 16 and 64 rows and the tiles give a token's rows the same bits."""
    import torch
    L = _layer(dev, 400, 2, 8, 2, 192, 320, 0.5, 11)
    whole = _ffn(L, -1).cpu()
    of = {int(p): i for i, p in enumerate(L["row_pair"])}
    for t in (1, 9, 60, 95, 100):
        S = dict(L)
        ids = L["ids"][:t]
        _, _, (params, bufs, _) = run_plan(ids, 8, 2, t + 1, dev=dev)
        _, rp = oracle.permute(ids.reshape(-1).tolist(),
                               oracle.plan(ids.reshape(-1).tolist(), 8, 2, t + 1), 8)
        S.update(params=params, bufs=bufs, row_pair=np.asarray(rp, dtype=np.int64), ids=ids)
        got = _ffn(S, -1).cpu()
        assert torch.equal(got, whole[[of[int(p)] for p in S["row_pair"]]]), t


@pytest.mark.parametrize("T,K,E,P,D,F,hot", [
    (1, 4, 8, 4, 128, 192, 0.0), (20, 4, 16, 4, 256, 320, 0.7), (130, 2, 16, 4, 192, 256, 0.6),
    (300, 4, 8, 4, 128, 192, 0.6), (700, 2, 4, 2, 576, 320, 0.8), (1100, 1, 2, 1, 64, 64, 0.5),
    (2100, 2, 4, 2, 320, 1088, 0.5),
])
def test_grouped_ffn_float32_outputs(dev, T, K, E, P, D, F, hot):
    """Float32 outputs are the values that the bfloat16 ones are rounded from, and
    llep_combine_to_bf16 sums them with one rounding (float32 sums of K products:
    K 2^-23 of their magnitudes)."""
    import torch
    from paper_2601_17111_amd import binding as B
    L = _layer(dev, T, K, E, P, D, F, hot, 3 * T + E)
    narrow = _ffn(L, -1)
    e = L["experts"]
    tok = L["row_pair"] // K
    wide = torch.full((T * K, D), float("nan"), device=dev)
    ws = torch.empty(B.llep_grouped_ffn_int8_workspace_bytes(L["params"], F), dtype=torch.uint8,
                     device=dev)
    B.llep_grouped_ffn_int8(L["params"], L["bufs"], -1, torch.from_numpy(L["x"][tok]).to(dev),
                            torch.from_numpy(L["s"]).to(dev),
                            torch.from_numpy(L["row_pair"].astype(np.int32)).to(dev), e.gate_up,
                            e.gate_scale, e.up_scale, e.down, e.down_scale, wide, ws)
    gates = np.random.default_rng(T).uniform(0, 1, (T, K)).astype(np.float32)
    pair_row = torch.from_numpy(np.asarray(L["pair_row"], dtype=np.int32)).to(dev)
    y = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
    B.llep_combine_to_bf16(L["params"], wide, pair_row, torch.from_numpy(gates).to(dev), y)
    torch.cuda.synchronize()
    assert torch.equal(wide.bfloat16(), narrow)
    rows = wide.double().cpu().numpy()[np.asarray(L["pair_row"])].reshape(T, K, D)
    terms = rows * gates[:, :, None]
    want = terms.sum(1)
    tol = 2.0 ** -8 * np.abs(want) + K * 2.0 ** -23 * np.abs(terms).sum(1)
    assert (np.abs(y.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("T,hot", [(2, 0.0), (30, 0.7), (40, 0.6)])
def test_grouped_ffn_of_large_weights(dev, T, hot):
    """Weights of more than half the cache, which rows that have them to themselves read past it:
    row tiles of 16 and of 32 rows, experts of one tile and a hot one of several; 24 rows checked
    (the tolerance of above: five steps, F = 2048 having about one of them expected)."""
    import torch
    L = _layer(dev, T, 4, 16, 4, 2880, 2048, hot, T)
    R = T * 4
    assert 3 * min(R, 16) * 2880 * 2048 > 128 << 20
    out = _ffn(L, -1)
    assert not torch.isnan(out).any()
    _check_ffn(L, out, np.unique(np.linspace(0, R - 1, min(R, 24)).astype(int)))
    assert torch.equal(_ffn(L, -1, by_row=True), out)


def test_product_of_a_large_matrix(dev):
    """A matrix of more than half the cache by a few rows: the same bits as by more rows."""
    import torch
    g = torch.Generator(device=dev).manual_seed(4)
    N, K, M = 70001, 2048, 40
    w = torch.randint(-127, 128, (N, K), generator=g, device=dev, dtype=torch.int8)
    q = torch.randint(-127, 128, (M, K), generator=g, device=dev, dtype=torch.int8)
    s = torch.rand(M, generator=g, device=dev) + 0.5
    ws = (torch.rand(N, generator=g, device=dev) + 0.5).cpu().numpy()
    from paper_2601_17111_amd import binding as B
    packed, wsd = B.llep_pack_matrix_int8(w), torch.from_numpy(ws).to(dev)
    outs = []
    for m in (40, 16, 3):
        out = torch.full((m, N), float("nan"), device=dev)
        B.llep_int8_matmul(q[:m], s[:m], packed, wsd, out, K)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(outs[0][:16], outs[1]) and torch.equal(outs[0][:3], outs[2])
    cols = np.linspace(0, N - 1, 300).astype(int)
    want = oracle.int8_product(q.cpu().numpy(), s.cpu().numpy(), w.cpu().numpy()[cols], ws[cols])
    got = outs[0].double().cpu().numpy()[:, cols]
    assert (np.abs(got - want) <= 2.0 ** -22 * np.abs(want)).all()


@pytest.mark.parametrize("T,hot", [(1, 0.0), (37, 0.5), (600, 0.7)])
def test_layer_near_the_bf16_layer(dev, T, hot):
    """LLEPLayer.forward_int8 with experts from bf16 weights: near forward(), as
    far as 8 bits go (each of the three roundings to 8 bits has steps of
    most / 127, errors of rms 0.29 steps, most about 4 times the rms of the
    values: 0.9% of the rms each; inputs, gate and up weights, activations and
    down weights together about 2.5%; 6% allowed), and a bad id's pair is left
    out as there."""
    import torch
    from paper_2601_17111_amd.layer import Int8Experts, LLEPLayer
    K, E, P, D, F = 4, 16, 4, 320, 192
    g = torch.Generator().manual_seed(T)
    ids = torch.where(torch.rand((T, K), generator=g) < hot, 0,
                      torch.randint(0, E, (T, K), generator=g)).to(torch.int32)
    ids[0, 0] = E  # out of range
    ids = ids.to(dev)
    gates = torch.softmax(torch.randn((T, K), generator=g), -1).to(dev)
    x = torch.randn((T, D), generator=g).to(dev).bfloat16()
    w = [(torch.randn(s, generator=g) * 0.05).to(dev).bfloat16()
         for s in ((E, D, F), (E, D, F), (E, F, D))]
    from paper_2601_17111_amd import binding as B
    layer = LLEPLayer(T, K, E, P, D, F, -(-T * K * 11 // (10 * P)), torch.bfloat16, dev)
    want = layer.forward(ids, gates, x, *B.llep_pack_weights(*w)).float().clone()
    got = layer.forward_int8(ids, gates, x, Int8Experts.from_weights(*w)).float()
    torch.cuda.synchronize()
    err = float((got - want).norm() / want.norm())
    print(f"[int8 layer T={T}] relative difference {err:.3e}", flush=True)
    assert err <= 0.06


def test_refusals(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts, LLEPLayer
    x = torch.zeros((4, 100), device=dev)
    q = torch.zeros((4, 128), dtype=torch.int8, device=dev)
    s = torch.zeros(4, device=dev)
    B.llep_quantize_rows(x, q, s)
    for bad, err in [
        (lambda: B.llep_quantize_rows(x, q[:, :64].contiguous(), s), B.LLEPError),
        (lambda: B.llep_quantize_rows(x, torch.zeros((4, 104), dtype=torch.int8, device=dev), s),
         B.LLEPError),
        (lambda: B.llep_quantize_rows(x.half(), q, s), TypeError),
        (lambda: B.llep_quantize_rows(x, q, s[:3]), ValueError),
        (lambda: B.llep_quantize_rows(x.t(), q, s), ValueError),
        (lambda: B.llep_int8_row_bytes(0), B.LLEPError),
        (lambda: B.llep_int8_row_bytes(65537), B.LLEPError),
    ]:
        with pytest.raises(err):
            bad()
    w = torch.zeros((48, 100), dtype=torch.int8, device=dev)
    packed = B.llep_pack_matrix_int8(w)
    ws, out = torch.zeros(48, device=dev), torch.zeros((4, 48), device=dev)
    B.llep_int8_matmul(q, s, packed, ws, out, 100)
    for bad, err in [
        (lambda: B.llep_int8_matmul(q, s, packed, ws, out, 200), ValueError),  # another matrix
        (lambda: B.llep_int8_matmul(q, s, packed, ws[:40], out, 100), ValueError),
        (lambda: B.llep_int8_matmul(q[:, :64].contiguous(), s, packed, ws, out, 100), B.LLEPError),
        (lambda: B.llep_int8_matmul(q, s, packed, ws, out.half(), 100), TypeError),
        (lambda: B.llep_pack_matrix_int8(w, w[:32].contiguous()), ValueError),
        (lambda: B.llep_pack_matrix_int8(w, w), B.LLEPError),  # gate and up: N % 32
        (lambda: B.llep_pack_matrix_int8(w.float()), TypeError),
        (lambda: B.llep_pack_matrix_int8(w[0]), ValueError),
    ]:
        with pytest.raises(err):
            bad()
    layer = LLEPLayer(4, 1, 2, 1, 64, 64, 4, torch.float32, dev)
    e = Int8Experts(*[torch.zeros(sh, dtype=t, device=dev) for sh, t in (
        ((2, 64, 64), torch.int8), ((2, 64), torch.float32)) * 3])
    ids = torch.zeros((4, 1), dtype=torch.int32, device=dev)
    with pytest.raises(TypeError):
        layer.forward_int8(ids, torch.ones((4, 1), device=dev), torch.zeros((4, 64), device=dev), e)
    L = _layer(dev, 4, 1, 2, 1, 64, 64, 0.0, 0)
    z = torch.zeros((4, 64), dtype=torch.int8, device=dev)
    o = torch.zeros((4, 64), dtype=torch.bfloat16, device=dev)
    f = L["experts"]
    args = (L["params"], L["bufs"])
    tail = (f.gate_up, f.gate_scale, f.up_scale, f.down, f.down_scale, o)
    with pytest.raises(B.LLEPError) as ei:
        B.llep_grouped_ffn_int8(*args, -1, z, s, None, *tail, torch.empty(16, device=dev))
    assert ei.value.code == B.LLEP_E_WORKSPACE
    big = torch.empty(1 << 20, dtype=torch.uint8, device=dev)
    with pytest.raises(B.LLEPError):
        B.llep_grouped_ffn_int8(*args, 1, z, s, None, *tail, big)
    with pytest.raises(ValueError):
        B.llep_grouped_ffn_int8(*args, -1, z, s[:3], None, *tail, big)
    B.llep_grouped_ffn_int8(*args, -1, z, s, None, *tail, big)
    torch.cuda.synchronize()
