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
