"""4-bit rows, packed weights and products against the oracle.

Rows are compared value by value and exponent by exponent: their rounding is
defined to the bit. Products of whole numbers whose sums stay below 2^24 units
are exact in 32 bits in any order, so float32 outputs have to be equal and
bfloat16 ones their rounding. Of other products every value of k may cost one
rounding, or cutting, of the sum of the magnitudes: (K + 32) 2^-23 of it (32: the
joins of parts of k), and half a step, 2^-8, of a bfloat16 result."""

import math

import numpy as np
import pytest

import oracle
from gpu_util import device

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def dev():
    return device()


def _sizes(D):
    from paper_2601_17111_amd import binding as B
    return B.llep_mxfp4_row_bytes(D), B.llep_mxfp4_scale_bytes(D)


# ---- rows -------------------------------------------------------------------

def _quantize(dev, x):
    import torch
    from paper_2601_17111_amd import binding as B
    R, D = x.shape
    nq, ns = _sizes(D)
    q = torch.full((R, nq), 0xee, dtype=torch.uint8, device=dev)
    s = torch.full((R, ns), 0xee, dtype=torch.uint8, device=dev)
    B.llep_quantize_rows_mxfp4(x, q, s)
    torch.cuda.synchronize()
    return q, s


def _check_rows(dev, x):
    """x on the GPU: its 4-bit rows, and what they stand for, against the oracle."""
    import torch
    from paper_2601_17111_amd import binding as B
    R, D = x.shape
    q, s = _quantize(dev, x)
    values = x.double().cpu().numpy()
    e = oracle.mxfp4_exponents(values)
    nb = -(-D // 32)
    got = s.cpu().numpy()
    assert np.array_equal(got[:, :nb], e)
    assert (got[:, nb:] != 255).all()
    codes = oracle.mxfp4_unpack(q.cpu().numpy(), 2 * q.shape[1])
    assert (codes[:, D:] == 0).all()
    want = oracle.mxfp4_decode(oracle.mxfp4_codes(values, e), e)
    have = oracle.mxfp4_decode(codes[:, :D], got)
    assert np.array_equal(have, want, equal_nan=True)
    out = torch.full((R, D), 7.0, dtype=x.dtype, device=dev)
    B.llep_dequantize_rows_mxfp4(q, s, out)
    assert np.array_equal(out.double().cpu().numpy(), have, equal_nan=True)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("R,D", [(1, 1), (3, 2), (2, 7), (1, 31), (5, 32), (2, 33), (7, 64), (3, 127),
                                 (4, 128), (2, 129), (3, 504), (2, 512), (3, 513), (70, 1003),
                                 (33, 2880), (1, 65536), (2, 65529)])
def test_rows(dev, R, D, dtype):
    import torch
    g = torch.Generator().manual_seed(R * D)
    x = torch.randn(R, D, generator=g) * torch.exp2(torch.randint(-9, 9, (R, D), generator=g).float())
    _check_rows(dev, x.to(getattr(torch, dtype)).to(dev))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_ties_and_borders(dev, dtype):
    """Every midpoint of the grid and its neighbours, at several powers of two, both signs."""
    import torch
    t = getattr(torch, dtype)
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0])
    step = torch.finfo(t).eps
    near = torch.cat([mid, mid * (1 + step), mid * (1 - step / 2), torch.tensor([4.0, 0.0, -0.0, 6.0])])
    rows = []
    for power in (-120, -60, -3, 0, 5, 100, 125):
        for sign in (1, -1):
            row = torch.zeros(64)
            row[:len(near)] = near * sign * 2.0 ** power
            row[40] = 4.0 * 2.0 ** power
            row[32:40] = near[:8] * sign * 2.0 ** power
            rows.append(row)
    _check_rows(dev, torch.stack(rows).to(t).to(dev))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_smallest_and_largest(dev, dtype):
    import torch
    t = getattr(torch, dtype)
    big, tiny = torch.finfo(t).max, torch.finfo(t).tiny
    x = torch.zeros(8, 96)
    x[0, 3], x[0, 70] = big, -big
    x[1, :4] = torch.tensor([tiny, -tiny, tiny * 3, tiny * 0.5])
    x[2, 5] = tiny * 2.0 ** -5
    x[3] = tiny * torch.arange(96) / 8
    x[4, 10], x[4, 11] = INF, 1.0
    x[5, 33] = NAN
    x[6, 95], x[6, 1] = -INF, NAN
    x[7] = -0.0
    _check_rows(dev, x.to(t).to(dev))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_every_byte_and_exponent(dev, dtype):
    """All 256 bytes under all 256 exponents; values beyond the type's range are infinite."""
    import torch
    from paper_2601_17111_amd import binding as B
    q = torch.arange(256, dtype=torch.uint8).repeat(256, 1)
    s = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 16)
    out = torch.empty((256, 512), dtype=getattr(torch, dtype), device=dev)
    B.llep_dequantize_rows_mxfp4(q.to(dev), s.to(dev), out)
    want = oracle.mxfp4_decode(oracle.mxfp4_unpack(q.numpy(), 512), s.numpy())
    want[np.abs(want) >= 2.0 ** 128] *= INF
    assert np.array_equal(out.double().cpu().numpy(), want, equal_nan=True)


def test_rows_apart_and_unaligned(dev):
    """Values and exponents side by side in wider rows, whose other bytes stay; inputs and outputs
    that start at any element."""
    import torch
    from paper_2601_17111_amd import binding as B
    for D, dtype, off in ((100, torch.float32, 1), (96, torch.bfloat16, 3), (1003, torch.bfloat16, 1),
                          (512, torch.float32, 0)):
        R, (nq, ns) = 9, _sizes(D)
        flat = torch.randn(R * D + 8, device=dev).to(dtype)
        x = flat[off:off + R * D].view(R, D)
        wide = torch.full((R, nq + ns + 32), 0x5a, dtype=torch.uint8, device=dev)
        q, s = wide[:, :nq], wide[:, nq + 16:nq + 16 + ns]
        B.llep_quantize_rows_mxfp4(x, q, s)
        q2, s2 = _quantize(dev, x.clone())
        assert torch.equal(q, q2) and torch.equal(s, s2)
        assert bool((wide[:, nq:nq + 16] == 0x5a).all()) and bool((wide[:, -16:] == 0x5a).all())
        out = torch.full((R * D + 8,), 3.0, dtype=dtype, device=dev)
        B.llep_dequantize_rows_mxfp4(q, s, out[off:off + R * D].view(R, D))
        want = torch.empty((R, D), dtype=dtype, device=dev)
        B.llep_dequantize_rows_mxfp4(q2, s2, want)
        assert torch.equal(out[off:off + R * D].view(R, D), want)
        assert out[:off].tolist() == [3.0] * off and bool((out[off + R * D:] == 3.0).all())


def test_no_rows(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    q = torch.empty((0, 64), dtype=torch.uint8, device=dev)
    s = torch.empty((0, 16), dtype=torch.uint8, device=dev)
    x = torch.empty((0, 100), device=dev)
    B.llep_quantize_rows_mxfp4(x, q, s)
    B.llep_dequantize_rows_mxfp4(q, s, x)
    w = B.llep_pack_matrix_mxfp4(torch.zeros((8, 50), dtype=torch.uint8, device=dev),
                                 torch.full((8, 4), 127, dtype=torch.uint8, device=dev))
    B.llep_mxfp4_matmul(q, s, w, torch.empty((0, 8), device=dev), 100)
    torch.cuda.synchronize()


# ---- products ---------------------------------------------------------------

def _random_rows(g, R, K, lo, hi):
    """Codes and exponents as 4-bit rows, and the values that they stand for."""
    codes = g.integers(0, 16, (R, K)).astype(np.uint8)
    e = g.integers(lo, hi, (R, -(-K // 32))).astype(np.uint8)
    return codes, e, oracle.mxfp4_decode(codes, e)


def _as_rows(dev, codes, e, pad_exponent=127):
    import torch
    nq, ns = _sizes(codes.shape[1])
    q = torch.zeros((len(codes), nq), dtype=torch.uint8)
    b = oracle.mxfp4_pack(codes)
    q[:, :b.shape[1]] = torch.from_numpy(b)
    s = torch.full((len(codes), ns), pad_exponent, dtype=torch.uint8)
    s[:, :e.shape[1]] = torch.from_numpy(e)
    return q.to(dev), s.to(dev)


def _pack(dev, codes, e):
    import torch
    from paper_2601_17111_amd import binding as B
    return B.llep_pack_matrix_mxfp4(torch.from_numpy(oracle.mxfp4_pack(codes)).to(dev),
                                    torch.from_numpy(e).to(dev), K=codes.shape[1])


def _check_product(dev, M, N, K, seed, lo=126, hi=129):
    """float32 and bfloat16 outputs of whole numbers (of 2^-4: 6 * 6 * 4 K of them stay below
    2^24 up to K = 7000)."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(seed)
    xc, xe, xv = _random_rows(g, M, K, lo, hi)
    wc, we, wv = _random_rows(g, N, K, lo, hi)
    q, s = _as_rows(dev, xc, xe, seed % 255)
    w = _pack(dev, wc, we)
    want = torch.from_numpy(xv).to(dev) @ torch.from_numpy(wv).to(dev).t()
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M + 1, N), NAN, dtype=dtype, device=dev)
        B.llep_mxfp4_matmul(q, s, w, out[:M], K)
        torch.cuda.synchronize()
        assert torch.equal(out[:M], want.to(dtype)), (M, N, K, dtype)
        assert bool(torch.isnan(out[M]).all())


@pytest.mark.parametrize("M,N,K", [
    (1, 1, 1), (1, 2880, 2880), (2, 3, 65), (3, 17, 63), (15, 64, 128), (16, 65, 130), (1, 7168, 2048),
    (17, 100, 192), (31, 257, 1003), (33, 48, 1000), (63, 193, 64), (64, 256, 320), (17, 4200, 130),
    (65, 16, 64), (65, 255, 100), (100, 1, 200), (129, 512, 448), (255, 384, 512), (256, 192, 64),
    (257, 600, 300), (333, 2881, 1003), (513, 264, 192), (1000, 130, 5000), (130, 4100, 4096),
    (256, 4096, 4096), (4, 5000, 257), (8, 40, 6999),
])
def test_products(dev, M, N, K):
    _check_product(dev, M, N, K, M + N + K)


@pytest.mark.parametrize("M,N,K", [
    # 128-row tiles: one to six slices of k and more, a last tile of few rows or
    # columns, odd rows and columns, fewer tiles than workgroups and more
    (1800, 1800, 64), (1793, 1801, 130), (130, 30001, 70), (1500, 3001, 501), (2050, 1288, 640),
    (2500, 4104, 200), (1024, 1024, 768), (1025, 2050, 1300), (600, 5000, 3001),
    # 256-row tiles, several of them for a workgroup, and those that are just not
    (8192, 4096, 128), (8200, 4097, 257), (6001, 5008, 500), (3000, 7001, 1000), (4100, 4100, 2890),
    (16385, 2056, 400), (16400, 6208, 130), (8190, 8185, 333), (7937, 8200, 1500), (4090, 4090, 2890),
    (12200, 5377, 1000), (8100, 8100, 64),
])
def test_products_of_many_rows(dev, M, N, K):
    _check_product(dev, M, N, K, M + N + K)


@pytest.mark.parametrize("M,N,K,form", [
    (1, 7168, 2048, "stream_kernel<1, 1, 8"), (16, 300, 65, "stream_kernel<1, 1, 8"),
    (17, 768, 2048, "stream_kernel<2, 1, 16"), (64, 2048, 7168, "stream_kernel<2, 1, 16"),
    (64, 7168, 2048, "stream_kernel<2, 2, 8"), (33, 20000, 130, "tiles_kernel<128"), (40, 7168, 1000, "stream_kernel<2, 2, 8"),
    (256, 4096, 4096, "stream_kernel<4, 4, 8"), (200, 4200, 5000, "tiles_kernel<128"), (200, 4000, 5000, "stream_kernel<4, 4, 8"),
    (1024, 7168, 2048, "tiles_kernel<128"), (2050, 1288, 640, "tiles_kernel<128"),
    (8192, 4096, 128, "tiles_kernel<256"), (4100, 4100, 2890, "tiles_kernel<128"),
    (4090, 4090, 2890, "tiles_kernel<256"), (8190, 8185, 333, "tiles_kernel<256"),
])
def test_forms(dev, M, N, K, form):
    """Each of the ways that a product can take, by the name of its kernel, gives whole numbers."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as seen:
        _check_product(dev, M, N, K, M + N + K)
        torch.cuda.synchronize()
    names = {e.key for e in seen.key_averages() if "llep::mx_" in e.key and "pack" not in e.key}
    assert names and all(form in n for n in names), names


@pytest.mark.parametrize("M,N,K", [(5, 300, 1000), (40, 200, 2880), (700, 1500, 2880), (2900, 3000, 300)])
def test_products_of_many_exponents(dev, M, N, K):
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(M)
    xc, xe, xv = _random_rows(g, M, K, 90, 150)
    wc, we, wv = _random_rows(g, N, K, 110, 140)
    q, s = _as_rows(dev, xc, xe)
    w = _pack(dev, wc, we)
    xv, wv = torch.from_numpy(xv).to(dev), torch.from_numpy(wv).to(dev)
    want, near = xv @ wv.t(), (K + 32) * 2.0 ** -23 * (xv.abs() @ wv.abs().t())
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.empty((M, N), dtype=dtype, device=dev)
        B.llep_mxfp4_matmul(q, s, w, out, K)
        tol = near + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
        assert bool(((out.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("M,N", [(4, 70), (40, 300), (100, 300), (1500, 1500), (4100, 4100), (4090, 4090)])
def test_blocks_of_nan(dev, M, N):
    """An exponent of 255 makes the rows that have it NaN, and no others."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(N)
    K = 400
    xc, xe, _ = _random_rows(g, M, K, 126, 129)
    wc, we, _ = _random_rows(g, N, K, 126, 129)
    xe[1, 12], we[N - 1, 0] = 255, 255  # (the last block, of 16 values, and the first)
    xc[1] = 0  # zeros times NaN
    q, s = _as_rows(dev, xc, xe)
    out = torch.empty((M, N), device=dev)
    B.llep_mxfp4_matmul(q, s, _pack(dev, wc, we), out, K)
    bad = torch.isnan(out)
    assert bool(bad[1].all()) and bool(bad[:, N - 1].all())
    assert int(bad.sum()) == M + N - 1


def test_extreme_exponents(dev):
    """Blocks of 2^-127 and of 2^127 whose products are ordinary numbers."""
    import torch
    from paper_2601_17111_amd import binding as B
    K, N = 128, 32
    for M in (3, 40, 1500):
        xc = np.full((M, K), 2, dtype=np.uint8)  # ones
        wc = np.full((N, K), 5, dtype=np.uint8)  # threes
        xe = np.full((M, 4), 254, dtype=np.uint8)
        we = np.zeros((N, 4), dtype=np.uint8)
        q, s = _as_rows(dev, xc, xe)
        out = torch.empty((M, N), device=dev)
        B.llep_mxfp4_matmul(q, s, _pack(dev, wc, we), out, K)
        assert bool((out == 3.0 * K).all())


def test_rows_of_a_product_lie_apart(dev):
    """Operand rows in a wider buffer, in all forms; whatever is between them."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(5)
    K, N = 700, 1800
    for M in (3, 30, 200, 1800, 8190):
        xc, xe, xv = _random_rows(g, M, K, 126, 129)
        wc, we, wv = _random_rows(g, N, K, 126, 129)
        q, s = _as_rows(dev, xc, xe)
        wide = torch.randint(0, 256, (M, q.shape[1] + s.shape[1] + 48), dtype=torch.uint8, device=dev)
        wide[:, 16:16 + q.shape[1]] = q
        wide[:, -16 - s.shape[1]:-16] = s
        out = torch.empty((M, N), device=dev)
        B.llep_mxfp4_matmul(wide[:, 16:16 + q.shape[1]], wide[:, -16 - s.shape[1]:-16],
                            _pack(dev, wc, we), out, K)
        want = torch.from_numpy(xv).to(dev) @ torch.from_numpy(wv).to(dev).t()
        assert torch.equal(out, want.float())


def test_outputs_past_32_bits(dev):
    """More than 2^31 outputs, and more than 4 GiB of them: the last rows and columns."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(6)
    M, N, K = 70000, 32784, 64
    xc, xe, xv = _random_rows(g, M, K, 126, 129)
    wc, we, wv = _random_rows(g, N, K, 126, 129)
    q, s = _as_rows(dev, xc, xe)
    out = torch.zeros((M, N), dtype=torch.bfloat16, device=dev)
    assert out.numel() > 2 ** 31
    B.llep_mxfp4_matmul(q, s, _pack(dev, wc, we), out, K)
    xv, wv = torch.from_numpy(xv).to(dev), torch.from_numpy(wv).to(dev)
    for a, b in ((0, 300), (M // 2, M // 2 + 300), (M - 300, M)):
        assert torch.equal(out[a:b], (xv[a:b] @ wv.t()).bfloat16())


@pytest.mark.parametrize("dtype,R", [("float32", 50001), ("bfloat16", 50001), ("bfloat16", 190001)])
def test_rows_of_more_than_the_cache(dev, dtype, R):
    """Values, and 4-bit rows, of more than 256 MB: the same as those of smaller calls."""
    import torch
    from paper_2601_17111_amd import binding as B
    D = 2888
    x = torch.randn(R, D, device=dev).to(getattr(torch, dtype))
    assert x.numel() * x.element_size() > 256 << 20
    q, s = _quantize(dev, x)
    out = torch.empty_like(x)
    B.llep_dequantize_rows_mxfp4(q, s, out)
    for a, b in ((0, 7000), (25000, 32000), (43000, R)):
        q1, s1 = _quantize(dev, x[a:b].clone())
        assert torch.equal(q[a:b], q1) and torch.equal(s[a:b], s1)
        part = torch.empty_like(x[a:b])
        B.llep_dequantize_rows_mxfp4(q1, s1, part)
        assert torch.equal(out[a:b], part)


def test_packed_gate_and_up_rows(dev):
    """Gate and up rows together: 32 of the first, then the matching 32 of the second."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(7)
    N, K = 96, 200
    parts = [_random_rows(g, N, K, 126, 129) for _ in range(2)]
    args = [torch.from_numpy(a).to(dev) for c, e, _ in parts for a in (oracle.mxfp4_pack(c), e)]
    both = B.llep_pack_matrix_mxfp4(*args, K=K)
    order = np.concatenate([np.arange(i, i + 32) + N * h for i in range(0, N, 32) for h in (0, 1)])
    wc, we = (np.concatenate([p[i] for p in parts])[order] for i in (0, 1))
    assert torch.equal(both, _pack(dev, wc, we))


@pytest.mark.parametrize("E,N,K,extra", [(3, 40, 70, 5), (2, 16, 256, 16), (1, 33, 31, 3)])
def test_packing_rows_longer_than_needed(dev, E, N, K, extra):
    """What lies behind a row's values and exponents is not read as such."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(8)
    c, e, _ = _random_rows(g, E * N, K, 100, 150)
    b = oracle.mxfp4_pack(c)
    dense = B.llep_pack_matrix_mxfp4(torch.from_numpy(b.reshape(E, N, -1)).to(dev),
                                     torch.from_numpy(e.reshape(E, N, -1)).to(dev), K=K)
    if K % 2:
        b[:, -1] |= 0xf0  # the half of a byte that no value has
    longer = [np.concatenate([a, np.full((len(a), extra), 255, dtype=np.uint8)], 1)
              .reshape(E, N, -1) for a in (b, e)]
    assert torch.equal(B.llep_pack_matrix_mxfp4(*(torch.from_numpy(a).to(dev) for a in longer), K=K),
                       dense)


def test_product_in_a_graph_and_on_a_stream(dev):
    """Rows and product captured and replayed with other activations, by a few and by many rows;
    and on a stream of its own."""
    import torch
    from paper_2601_17111_amd import binding as B
    g = np.random.default_rng(9)
    N, K = 1900, 300
    wc, we, _ = _random_rows(g, N, K, 118, 122)
    w = _pack(dev, wc, we)
    for M in (1, 25, 1900):
        xs = [torch.randn(M, K, device=dev) for _ in range(3)]
        nq, ns = _sizes(K)
        q = torch.empty((M, nq), dtype=torch.uint8, device=dev)
        s = torch.empty((M, ns), dtype=torch.uint8, device=dev)
        out = torch.empty((M, N), dtype=torch.bfloat16, device=dev)

        def call(x, stream=None):
            B.llep_quantize_rows_mxfp4(x, q, s, stream)
            B.llep_mxfp4_matmul(q, s, w, out, K, stream)
        want = []
        for x in xs:
            call(x)
            want.append(out.clone())
        x = xs[0].clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(x)
        for i in (1, 2, 0, 1):
            x.copy_(xs[i])
            out.fill_(0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(xs[2], side)
        side.synchronize()
        assert torch.equal(out, want[2])


def test_refusals(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    u8 = dict(dtype=torch.uint8, device=dev)
    x = torch.zeros((4, 100), device=dev)
    q, s = torch.zeros((4, 64), **u8), torch.zeros((4, 16), **u8)
    w, ws = torch.zeros((48, 50), **u8), torch.full((48, 4), 127, **u8)
    packed = B.llep_pack_matrix_mxfp4(w, ws)
    out = torch.zeros((4, 48), device=dev)
    B.llep_quantize_rows_mxfp4(x, q, s)
    B.llep_mxfp4_matmul(q, s, packed, out, 100)
    wide = torch.zeros((4, 72), **u8)
    for bad, err in [
        (lambda: B.llep_quantize_rows_mxfp4(x.half(), q, s), TypeError),
        (lambda: B.llep_quantize_rows_mxfp4(x.t(), q, s), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x.cpu(), q, s), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x, q[:3], s), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x, q[:, :48], s), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x, q, s[:, :8]), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x, q.char(), s), TypeError),
        (lambda: B.llep_quantize_rows_mxfp4(x, wide[:, :64], s), B.LLEPError),   # 72 bytes apart
        (lambda: B.llep_quantize_rows_mxfp4(x, torch.zeros((4, 80), **u8)[:, 8:72], s), B.LLEPError),
        (lambda: B.llep_quantize_rows_mxfp4(x, torch.zeros((64, 4), **u8).t(), s), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x, q[:1].expand(4, 64), s), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(x[:1], torch.zeros((1, 128), **u8)[:, ::2], s[:1]), ValueError),
        (lambda: B.llep_quantize_rows_mxfp4(torch.zeros((4, 0), device=dev), q, s), B.LLEPError),
        (lambda: B.llep_dequantize_rows_mxfp4(q, s, x.half()), TypeError),
        (lambda: B.llep_dequantize_rows_mxfp4(q, s, torch.zeros((4, 200), device=dev)), ValueError),
        (lambda: B.llep_mxfp4_row_bytes(0), B.LLEPError),
        (lambda: B.llep_mxfp4_scale_bytes(65537), B.LLEPError),
        (lambda: B.llep_pack_matrix_mxfp4(w, ws[:, :3].contiguous()), ValueError),
        (lambda: B.llep_pack_matrix_mxfp4(w, ws, K=101), ValueError),
        (lambda: B.llep_pack_matrix_mxfp4(w, ws, K=0), B.LLEPError),
        (lambda: B.llep_pack_matrix_mxfp4(w, ws, w), ValueError),
        (lambda: B.llep_pack_matrix_mxfp4(w, ws, w, ws), B.LLEPError),           # N % 32
        (lambda: B.llep_pack_matrix_mxfp4(w.char(), ws), TypeError),
        (lambda: B.llep_pack_matrix_mxfp4(w[0], ws[0]), ValueError),
        (lambda: B.llep_pack_matrix_mxfp4(torch.zeros((0, 50), **u8), torch.zeros((0, 4), **u8)),
         B.LLEPError),
        (lambda: B.llep_mxfp4_matmul(q, s, packed, out, 200), ValueError),       # another matrix
        (lambda: B.llep_mxfp4_matmul(q, s, packed, out.half(), 100), TypeError),
        (lambda: B.llep_mxfp4_matmul(q[:3], s, packed, out, 100), ValueError),
        (lambda: B.llep_mxfp4_matmul(q, s, packed, torch.zeros((4, 30), device=dev), 100), ValueError),
        (lambda: B.llep_mxfp4_matmul(q, s, packed, torch.zeros(4 * 48 + 1, device=dev)[1:].view(4, 48),
                                     100), B.LLEPError),
    ]:
        with pytest.raises(err):
            bad()
    torch.cuda.synchronize()
