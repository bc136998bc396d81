"""ExpertBlock without a GPU: what it refuses when it is made."""

import types

import pytest

B = pytest.importorskip("paper_2601_17111_amd.binding")


def _layer(D):
    import torch
    return types.SimpleNamespace(T=2, D=D, dtype=torch.bfloat16, device="cpu")


def test_rows_longer_than_the_norms_take():
    import torch
    from paper_2601_17111_amd.block import ExpertBlock
    w = torch.ones(8192, dtype=torch.bfloat16)
    ExpertBlock(_layer(8192), w, w, None, w)
    for D in (8256, 65536):
        w = torch.ones(D, dtype=torch.bfloat16)
        with pytest.raises(ValueError, match="8192"):
            ExpertBlock(_layer(D), w, w, None, w)
