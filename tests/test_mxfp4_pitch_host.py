"""4-bit rows and weights whose sizes or distances do not fit the C calls' 32 bits are
refused by the binding, which would pass their lowest 32 bits on; tensors without
memory (device "meta") stand for such large ones."""

import pytest

torch = pytest.importorskip("torch")
B = pytest.importorskip("paper_2601_17111_amd.binding")


def _rows(n, width, pitch):
    t = torch.empty((n, width), dtype=torch.uint8, device="meta").as_strided((n, width), (pitch, 1))
    B._type_code(torch.empty(1))  # (the calls ask for the data's type first)
    return t, t.get_device()


def test_rows_further_apart_than_32_bits():
    for pitch in (1 << 31, (1 << 32) + 64, 1 << 33):
        t, dev = _rows(2, 64, pitch)
        with pytest.raises(ValueError, match="apart"):
            B._byte_rows("q", t, 2, 64, dev)
    for pitch in (64, 65536, (1 << 31) - 16):
        t, dev = _rows(2, 64, pitch)
        assert B._byte_rows("q", t, 2, 64, dev) == pitch


def test_the_distance_of_an_only_row_means_nothing():
    """Nor does its width, beyond the bytes that are used."""
    for n in (0, 1):
        for width, pitch in ((64, 64), (64, 1 << 33), (70000, 70000), (100, 7), ((1 << 32) + 16, 1 << 32)):
            t, dev = _rows(n, width, pitch)
            assert B._byte_rows("q", t, n, 64, dev) == 64
    t = torch.empty((1, 64), dtype=torch.uint8, device="meta").as_strided((1, 64), (128, 2))
    with pytest.raises(ValueError):
        B._byte_rows("q", t, 1, 64, t.get_device())


@pytest.mark.parametrize("shape,blocks,K", [
    ((4, (1 << 32) + 64), 4, 128), ((4, 1 << 31), 4, 128), ((4, 64), (1 << 32) + 4, 128),
    (((1 << 32) + 16, 1), 1, 2), (((1 << 32) + 1, 16, 1), 1, 2), ((4, 1 << 32), 1 << 28, (1 << 33) - 2)])
def test_weights_of_more_than_32_bits(shape, blocks, K):
    w = torch.empty(shape, dtype=torch.uint8, device="meta")
    scale = torch.empty((*shape[:-1], blocks), dtype=torch.uint8, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        B.llep_pack_matrix_mxfp4(w, scale, K=K)
