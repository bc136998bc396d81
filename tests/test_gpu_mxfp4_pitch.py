"""4-bit rows that are far apart: parts of a buffer whose rows are as long as the calls
take them (LLEP_MAX_FFN_DIM bytes), and an only row of a longer one."""

import pytest

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _rows(n, width, pitch, dev):
    import torch
    return torch.full((n, pitch), 0xa5, dtype=torch.uint8, device=dev)[:, 32:32 + width]


@pytest.mark.parametrize("M", [5, 100, 700])
@pytest.mark.parametrize("N,K", [(48, 100), (300, 1000)])
def test_rows_as_far_apart_as_may_be(dev, M, N, K):
    import torch
    from paper_2601_17111_amd import binding as B
    far = B.LLEP_MAX_FFN_DIM
    g = torch.Generator().manual_seed(M)
    x = torch.randn((M, K), generator=g).to(dev)
    nq, ns = B.llep_mxfp4_row_bytes(K), B.llep_mxfp4_scale_bytes(K)
    w = torch.randint(0, 256, (N, nq), dtype=torch.uint8, generator=g).to(dev)
    ws = torch.randint(120, 130, (N, ns), dtype=torch.uint8, generator=g).to(dev)
    packed = B.llep_pack_matrix_mxfp4(w, ws, K=K)
    got = []
    for q_pitch, s_pitch in ((nq, ns), (far, far), (far, ns + 64)):
        if q_pitch == nq:
            q, s = (torch.empty((M, n), dtype=torch.uint8, device=dev) for n in (nq, ns))
        else:
            q, s = _rows(M, nq, q_pitch, dev), _rows(M, ns, s_pitch, dev)
        back, y = torch.empty_like(x), torch.empty((M, N), device=dev)
        B.llep_quantize_rows_mxfp4(x, q, s)
        B.llep_dequantize_rows_mxfp4(q, s, back)
        B.llep_mxfp4_matmul(q, s, packed, y, K)
        torch.cuda.synchronize()
        got.append([q, s, back, y])
        if q_pitch > nq:  # what lies around the rows is left as it is
            for t, n in ((q, nq), (s, ns)):
                whole = t._base
                assert bool((whole[:, :32] == 0xa5).all()) and bool((whole[:, 32 + n:] == 0xa5).all())
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_rows_further_apart_are_refused(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    x = torch.zeros((2, 100), device=dev)
    near = torch.zeros((2, 64), dtype=torch.uint8, device=dev)
    beyond = torch.zeros((2, B.LLEP_MAX_FFN_DIM + 16), dtype=torch.uint8, device=dev)[:, :64]
    packed = B.llep_pack_matrix_mxfp4(near, near, K=100)
    for q, s in ((beyond, near), (near, beyond)):
        for call in (lambda: B.llep_quantize_rows_mxfp4(x, q, s), lambda: B.llep_dequantize_rows_mxfp4(q, s, x),
                     lambda: B.llep_mxfp4_matmul(q, s, packed, torch.zeros((2, 2), device=dev), 100)):
            with pytest.raises(B.LLEPError):
                call()
    torch.cuda.synchronize()


def test_an_only_row_of_a_long_buffer(dev):
    """Its distance to a next one, which is not there, does not matter."""
    import torch
    from paper_2601_17111_amd import binding as B
    x = torch.randn((1, 100), generator=torch.Generator().manual_seed(1)).to(dev)
    got = []
    for width in (64, 100, 70000):
        buffers = [torch.full((1, width), 0xa5, dtype=torch.uint8, device=dev) for _ in "qs"]
        back = torch.empty_like(x)
        B.llep_quantize_rows_mxfp4(x, *buffers)
        B.llep_dequantize_rows_mxfp4(*buffers, back)
        torch.cuda.synchronize()
        got.append(back)
        assert bool((buffers[0][:, 64:] == 0xa5).all()) and bool((buffers[1][:, 16:] == 0xa5).all())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
