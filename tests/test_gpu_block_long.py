"""The calls around the block on tensors of more than 2^31 elements or bytes:
the last rows have the bits that a short call on those rows alone gives (a row's
result depends on no other row; sums over rows get zeros from all the others)."""

import pytest

from gpu_util import device

pytestmark = pytest.mark.gpu

TAIL = 3  # rows that hold values; the others are zeros


@pytest.fixture(scope="module")
def dev():
    return device()


def _tailed(dev, T, D, seed, dtype=None, rows=TAIL):
    """[T, D], zeros but for the last `rows` rows."""
    import torch
    g = torch.Generator(device=dev).manual_seed(seed)
    t = torch.zeros((T, D), dtype=dtype or torch.bfloat16, device=dev)
    t[-rows:] = torch.randn((rows, D), generator=g, device=dev).to(t.dtype)
    return t


def _weights(dev, D):
    return [_tailed(dev, 1, D, 2 + i, rows=1).view(D) for i in range(3)]


@pytest.mark.parametrize("D", [8192, 8191])  # whole vectors, and odd rows
def test_norm(dev, D):
    import torch
    from paper_2601_17111_amd import binding as B
    T = (1 << 31) // D + 100
    x, b = _tailed(dev, T, D, 0), _tailed(dev, T, D, 1)
    post, pre, gate = _weights(dev, D)

    def run(x, b):
        r, h = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        B.llep_block_norm(x, b, gate.view(1, D), post, pre, 0.5, 1e-5, r, h)
        return r, h

    r, h = run(x, b)
    r1, h1 = run(x[-TAIL:], b[-TAIL:])
    torch.cuda.synchronize()
    assert torch.equal(r[-TAIL:], r1) and torch.equal(h[-TAIL:], h1)
    assert bool(r1.any()) and not bool(r[:TAIL].any()) and not bool(h[-TAIL - 2:-TAIL].any())


@pytest.mark.parametrize("D", [8192, 8191])
def test_norm_backward(dev, D):
    """The gradients come from the last row alone, so every sum over rows is one
    value and zeros."""
    import torch
    from paper_2601_17111_amd import binding as B
    T = (1 << 31) // D + 100
    r, b = _tailed(dev, T, D, 0), _tailed(dev, T, D, 1)
    d_r, d_h = _tailed(dev, T, D, 5, rows=1), _tailed(dev, T, D, 6, rows=1)
    post, pre, gate = _weights(dev, D)

    def run(r, b, d_r, d_h):
        dx, db = torch.full_like(r, 7.0), torch.full_like(r, 7.0)
        sums = [torch.full(s, 7.0, device=dev) for s in ((1, D), (D,), (D,))]
        ws = torch.empty(B.llep_block_norm_backward_workspace_bytes(*r.shape), dtype=torch.uint8,
                         device=dev)
        B.llep_block_norm_backward(r, b, gate.view(1, D), post, pre, 0.5, 1e-5, d_r, d_h, dx, db,
                                   *sums, ws)
        return dx, db, sums

    dx, db, sums = run(r, b, d_r, d_h)
    dx1, db1, sums1 = run(*(t[-TAIL:] for t in (r, b, d_r, d_h)))
    torch.cuda.synchronize()
    assert torch.equal(dx[-TAIL:], dx1) and torch.equal(db[-TAIL:], db1)
    assert bool(dx1[-1].any()) and bool(db1[-1].any()) and not bool(dx[:TAIL].any())
    for got, want in zip(sums, sums1):
        assert torch.equal(got, want) and bool(want.any())


@pytest.mark.parametrize("D", [8192, 8191])
def test_rows_to_8_bits(dev, D):
    import torch
    from paper_2601_17111_amd import binding as B
    T = (1 << 31) // D + 100
    x = _tailed(dev, T, D, 0)

    def run(x):
        q = torch.full((x.shape[0], B.llep_int8_row_bytes(D)), 7, dtype=torch.int8, device=dev)
        s = torch.full((x.shape[0],), 7.0, device=dev)
        B.llep_quantize_rows(x, q, s)
        return q, s

    q, s = run(x)
    q1, s1 = run(x[-TAIL:])
    torch.cuda.synchronize()
    assert torch.equal(q[-TAIL:], q1) and torch.equal(s[-TAIL:], s1)
    assert bool(q1.any()) and not bool(q[:TAIL].any()) and not bool(s[:-TAIL].any())


@pytest.mark.parametrize("M,N,K", [(66000, 32800, 64),    # outputs past 2^31 elements
                                   (33000, 48, 65536)])   # rows past 2^31 bytes
def test_product(dev, M, N, K):
    import torch
    from paper_2601_17111_amd import binding as B
    g = torch.Generator(device=dev).manual_seed(K)
    assert max(M * N, M * K) > 1 << 31
    q = torch.zeros((M, K), dtype=torch.int8, device=dev)
    q[-TAIL:] = torch.randint(-127, 128, (TAIL, K), generator=g, device=dev, dtype=torch.int8)
    w = torch.randint(-127, 128, (N, K), generator=g, device=dev, dtype=torch.int8)
    s = torch.rand(M, generator=g, device=dev) + 0.5
    ws = torch.rand(N, generator=g, device=dev) + 0.5
    packed = B.llep_pack_matrix_int8(w)

    def run(q, s):
        out = torch.full((q.shape[0], N), float("nan"), dtype=torch.bfloat16, device=dev)
        B.llep_int8_matmul(q, s, packed, ws, out, K)
        return out

    out, out1 = run(q, s), run(q[-TAIL:], s[-TAIL:])
    torch.cuda.synchronize()
    assert torch.equal(out[-TAIL:], out1)
    assert bool(out1.any()) and not bool(out[:TAIL].any()) and not bool(out[-TAIL - 2:-TAIL].any())


def test_clip(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    n = (1 << 31) + 100003
    g = torch.Generator(device=dev).manual_seed(0)
    grad = torch.zeros(n, dtype=torch.bfloat16, device=dev)
    tail = torch.randn(1000, generator=g, device=dev).bfloat16()
    grad[-1000:] = tail

    def run(t):
        norm = torch.full((1,), -1.0, device=dev)
        ws = torch.empty(B.llep_clip_gradients_workspace_bytes(), dtype=torch.uint8, device=dev)
        B.llep_clip_gradients([t], 1.0, norm, ws)
        return norm

    norm, norm1 = run(grad), run(tail)
    torch.cuda.synchronize()
    # the sum of squares in 64 bits: another order, the same 32 bits but for a tie
    want = float(norm1)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want and want > 1.0
    # and so a factor of 32 bits, a product and a bfloat16 of it
    a, b = grad[-1000:].float(), tail.float()
    assert bool(((a - b).abs() <= 2.0 ** -7 * b.abs()).all()) and not bool(grad[:1000].any())
