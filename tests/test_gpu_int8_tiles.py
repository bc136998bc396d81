"""8-bit products through the tiles of 128 and of 256 rows, dense and grouped,
each call checked to be on the form that it names: the grouped FFN against the
oracle (first and last rows of every group among them), on all devices and on
each, scales by token and by row, bfloat16 and float32 outputs; the same bits as
the weight stream gives; dense products of the same rows by the stream and both
tile heights bit for bit, with the largest sums and with scales that are not
finite.

Tolerance of the grouped FFN: of a row's F activations about L = F 127 4e-6 lie
near enough to a tie to round to the other side (as in the tests of the
stream); L + 6 sqrt(L) + 5 of them are allowed for, each worth one step of the
row's activation scale times the largest weight, and 2e-5 of the largest output;
bfloat16 outputs 2^-8 of their value more. Dense products: three roundings,
2^-22 of the value."""

import math

import numpy as np
import pytest

import oracle
from gpu_util import device, run_plan
from test_gpu_int8 import _bytes, _layer, _matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


# ---- grouped ----------------------------------------------------------------

def _groups(L, device):
    gb, groups = L["bufs"].group_begin.cpu().tolist(), L["bufs"].groups.cpu().tolist()
    lo, hi = (0, gb[-1]) if device < 0 else (gb[device], gb[device + 1])
    return groups[lo:hi]


def _run(L, device, dtype, by_row=False):
    """Outputs, and the row heights of tiles that the call's list of tiles can be of (its length
    is at the start of the workspace)."""
    import torch
    from paper_2601_17111_amd import binding as B
    dev, e = L["dev"], L["experts"]
    tok = L["row_pair"] // L["K"]
    xp = torch.from_numpy(L["x"][tok]).to(dev)
    rp = torch.from_numpy(L["row_pair"].astype(np.int32)).to(dev)
    s = torch.from_numpy(L["s"][tok] if by_row else L["s"]).to(dev)
    out = torch.full((len(tok), L["D"]), float("nan"), dtype=dtype, device=dev)
    ws = torch.empty(B.llep_grouped_ffn_int8_workspace_bytes(L["params"], L["F"]),
                     dtype=torch.uint8, device=dev)
    ws.fill_(0xff)
    B.llep_grouped_ffn_int8(L["params"], L["bufs"], device, xp, s, None if by_row else rp,
                            e.gate_up, e.gate_scale, e.up_scale, e.down, e.down_scale, out, ws)
    torch.cuda.synchronize()
    n = int(ws[:4].view(torch.int32)[0])
    sizes = [g[3] for g in _groups(L, device)]
    return out, {h for h in (16, 32, 64, 128, 256) if n == sum(-(-m // h) for m in sizes)}


def _check(L, out, rows):
    lam = L["F"] * 127 * 4e-6
    steps = lam + 6 * math.sqrt(lam) + 5
    ids = L["ids"].reshape(-1)[L["row_pair"]]
    got = out.double().cpu().numpy()
    for e in np.unique(ids[rows]):
        r = rows[ids[rows] == e]
        tok = L["row_pair"][r] // L["K"]
        want, most = oracle.swiglu_ffn_int8(
            L["x"][tok], L["s"][tok], L["w"][0][e], L["sc"][0][e], L["w"][1][e], L["sc"][1][e],
            L["w"][2][e], L["sc"][2][e])
        tol = (steps * most[:, None] / 127 * 127 * L["sc"][2][e].max()
               + 2e-5 * np.abs(want).max())
        if out.element_size() == 2:
            tol = tol + 2.0 ** -8 * np.abs(want)
        assert (np.abs(got[r] - want) <= tol).all(), e


@pytest.mark.parametrize("T,K,E,P,D,F,hot,height", [
    (600, 2, 4, 2, 1088, 1216, 0.3, 128), (600, 2, 4, 2, 1088, 1216, 0.95, 128),
    (515, 8, 64, 8, 704, 576, 0.6, 128), (2000, 2, 128, 8, 704, 576, 0.2, 128),
    (1201, 1, 2, 1, 1216, 1088, 0.5, 128),
    (1050, 2, 8, 4, 320, 4160, 0.5, 256), (975, 4, 16, 4, 1344, 2112, 0.3, 256),
    (975, 4, 16, 2, 1344, 2112, 0.97, 256),
])
def test_grouped_tiles(dev, T, K, E, P, D, F, hot, height):
    import torch
    L = _layer(dev, T, K, E, P, D, F, hot, T + E)
    R = T * K
    edges = [r for _, _, start, n in _groups(L, -1) for r in (start, start + n - 1)]
    rows = np.unique(np.concatenate([edges, np.linspace(0, R - 1, 120)]).astype(int))
    narrow, forms = _run(L, -1, torch.bfloat16)
    assert forms == {height}
    wide, forms = _run(L, -1, torch.float32)
    assert forms == {height}
    assert not torch.isnan(wide).any() and torch.equal(wide.bfloat16(), narrow)
    _check(L, wide, rows)
    _check(L, narrow, rows)
    for dtype, all_rows in ((torch.bfloat16, narrow), (torch.float32, wide)):
        assert torch.equal(_run(L, -1, dtype, by_row=True)[0], all_rows)
        for d in range(P):  # its rows alone are written, with the same bits
            part, forms = _run(L, d, dtype, by_row=d % 2 == 1)
            mine = np.zeros(R, dtype=bool)
            for _, _, start, n in _groups(L, d):
                mine[start:start + n] = True
            assert not mine.any() or height in forms
            m = torch.from_numpy(mine).to(dev)
            assert torch.equal(part[m], all_rows[m]) and torch.isnan(part[~m]).all()
    # the same tokens in calls that the weight stream takes
    of = {int(p): i for i, p in enumerate(L["row_pair"])}
    for t, stream in ((max(1, 5 * E // K), 16), (max(1, 16 * E // K), 32)):
        S = dict(L)
        ids = L["ids"][:t]
        cap = t * K + 1
        _, _, (params, bufs, _) = run_plan(ids, E, P, cap, dev=dev)
        flat = ids.reshape(-1).tolist()
        _, rp = oracle.permute(flat, oracle.plan(flat, E, P, cap), E)
        S.update(params=params, bufs=bufs, row_pair=np.asarray(rp, dtype=np.int64), ids=ids)
        for dtype, all_rows in ((torch.bfloat16, narrow), (torch.float32, wide)):
            got, forms = _run(S, -1, dtype)
            assert stream in forms
            assert torch.equal(got, all_rows[[of[int(p)] for p in S["row_pair"]]])


# ---- dense ------------------------------------------------------------------

def _product(q, s, packed, ws, out, K, form):
    """llep_int8_matmul, and that its kernel is of the form named."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    from paper_2601_17111_amd import binding as B
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as seen:
        B.llep_int8_matmul(q, s, packed, ws, out, K)
        torch.cuda.synchronize()
    names = [e.name for e in seen.events() if "int8_" in e.name]
    assert len(names) == 1 and form in names[0], names
    return out


TILES_128, TILES_256, STREAM = ("int8_tiles_kernel<128, 128", "int8_tiles_kernel<256, 256",
                                "int8_stream_kernel")


# the least rows of the three forms, by the estimates of the call's time
@pytest.mark.parametrize("N,K,m128,m256", [(2050, 1300, 2050, 7100), (5001, 1003, 1200, 3001),
                                           (7168, 2048, 700, 4100)])
def test_same_bits_from_every_kernel(dev, N, K, m128, m256):
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(N)
    q = torch.randint(-127, 128, (m256, -(-K // 64) * 64), device=dev, dtype=torch.int8,
                      generator=torch.Generator(device=dev).manual_seed(N))
    q[:, K:] = 0
    s = torch.rand(m256, device=dev) + 0.1
    s[5] = float("nan")  # a row that was not finite
    w, ws = _matrix(g, N, K)
    packed, wsd = B.llep_pack_matrix_int8(torch.from_numpy(w).to(dev)), torch.from_numpy(ws).to(dev)
    for dtype in (torch.float32, torch.bfloat16):
        outs = {}
        for m, form in ((m256, TILES_256), (m128, TILES_128), (100, STREAM), (17, STREAM),
                        (9, STREAM)):
            out = torch.full((m, N), 7.0, dtype=dtype, device=dev)
            outs[m] = _product(q[:m], s[:m], packed, wsd, out, K, form)
        whole = outs[m256]
        assert bool(torch.isnan(whole[5]).all()) and int(torch.isnan(whole).sum()) == N
        for m, out in outs.items():
            assert torch.equal(torch.nan_to_num(out, 3.0), torch.nan_to_num(whole[:m], 3.0)), m
        rows = np.unique(np.concatenate([[0, 4, 6, m128 - 1, m256 - 1],
                                         np.linspace(7, m256 - 1, 60)]).astype(int))
        want = oracle.int8_product(q[rows, :K].cpu().numpy(), s[rows].cpu().numpy(), w, ws)
        got = whole[rows].double().cpu().numpy()
        tol = 2.0 ** -22 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
        assert (np.abs(got - want) <= tol * np.abs(want)).all()


@pytest.mark.parametrize("M,N,form", [(1650, 1660, TILES_128), (4100, 4100, TILES_256)])
def test_largest_sums(dev, M, N, form):
    """Every product 127 * -127 over the largest k, whole numbers near 2^30, through the tiles."""
    import torch
    from paper_2601_17111_amd import binding as B
    K = 65536
    q = torch.full((M, K), 127, dtype=torch.int8, device=dev)
    packed = B.llep_pack_matrix_int8(torch.full((N, K), -127, dtype=torch.int8, device=dev))
    out = torch.full((M, N), 7.0, device=dev)
    _product(q, torch.ones(M, device=dev), packed, torch.ones(N, device=dev), out, K, form)
    assert bool((out == float(-127 * 127 * K)).all())
