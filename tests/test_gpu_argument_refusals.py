"""Arguments of the calls around the block that do not fit are refused with an
error of the package, or by their shapes."""

import pytest

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.mark.parametrize("shape", [(0, 64, 64), (2, 0, 64), (2, 64, 0), (0, 64), (64, 0)])
def test_matrices_of_no_elements(dev, shape):
    import torch
    from paper_2601_17111_amd import binding as B
    with pytest.raises(B.LLEPError) as ei:
        B.llep_pack_matrix_int8(torch.empty(shape, dtype=torch.int8, device=dev))
    assert ei.value.code == B.LLEP_E_ARG


def test_clipped_outputs_of_another_shape(dev):
    """As many elements are not enough: a transposed output would hold other places' values."""
    import torch
    from paper_2601_17111_amd import binding as B
    norm = torch.zeros(1, device=dev)
    ws = torch.empty(B.llep_clip_gradients_workspace_bytes(), dtype=torch.uint8, device=dev)
    g = [torch.ones((4, 6), device=dev), torch.ones(8, device=dev)]
    B.llep_clip_gradients(g, 1.0, norm, ws, out=[torch.empty_like(t) for t in g])
    for out in ([torch.zeros((6, 4), device=dev), torch.zeros(8, device=dev)],
                [torch.zeros(24, device=dev), torch.zeros(8, device=dev)],
                [torch.zeros((4, 6), device=dev), torch.zeros((8, 1), device=dev)]):
        with pytest.raises(ValueError):
            B.llep_clip_gradients(g, 1.0, norm, ws, out=out)
        torch.cuda.synchronize()
        assert not any(bool(t.any()) for t in out)
