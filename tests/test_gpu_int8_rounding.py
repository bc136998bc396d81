"""LLEPLayer.forward_int8 rounds a token's outputs once, whatever the batch: a
token has the same bits in a batch of any size as alone, and they are those of
llep_combine_to_bf16 on its experts' float32 outputs."""

import numpy as np
import pytest

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _weights(dev, E, D, F, seed):
    import torch
    from paper_2601_17111_amd.layer import Int8Experts
    g = torch.Generator().manual_seed(seed)
    w = [(torch.randn(s, generator=g) * 0.05).to(dev).bfloat16()
         for s in ((E, D, F), (E, D, F), (E, F, D))]
    return Int8Experts.from_weights(*w)


# rows of outputs: fewer than 2^21 elements, as many, and more; the last through
# tiles of 128 rows
@pytest.mark.parametrize("T,K,E,D,F", [(40, 4, 8, 1024, 128), (512, 4, 8, 1024, 128),
                                       (700, 4, 8, 1088, 192), (1201, 2, 4, 1088, 1216)])
def test_rounded_once_in_any_batch(dev, T, K, E, D, F):
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import LLEPLayer
    g = torch.Generator().manual_seed(T)
    ids = torch.randint(0, E, (T, K), generator=g).to(torch.int32).to(dev)
    gates = torch.softmax(torch.randn((T, K), generator=g), -1).to(dev)
    x = torch.randn((T, D), generator=g).to(dev).bfloat16()
    experts = _weights(dev, E, D, F, T)
    layer = LLEPLayer(T, K, E, 2, D, F, T * K, torch.bfloat16, dev)
    y = layer.forward_int8(ids, gates, x, experts).clone()
    alone = LLEPLayer(1, K, E, 2, D, F, K, torch.bfloat16, dev)
    for t in np.unique(np.linspace(0, T - 1, 12).astype(int)):
        one = alone.forward_int8(ids[t:t + 1], gates[t:t + 1], x[t:t + 1], experts)
        torch.cuda.synchronize()
        assert torch.equal(one[0], y[t]), t
    # from the experts' outputs in float32
    rows = torch.full((T * K, D), float("nan"), device=dev)
    ws = torch.empty(B.llep_grouped_ffn_int8_workspace_bytes(layer.params, F), dtype=torch.uint8,
                     device=dev)
    B.llep_grouped_ffn_int8(layer.params, layer.bufs, -1, layer.x_perm_q, layer.x_scale,
                            layer.row_pair, experts.gate_up, experts.gate_scale, experts.up_scale,
                            experts.down, experts.down_scale, rows, ws)
    want = torch.full((T, D), float("nan"), dtype=torch.bfloat16, device=dev)
    B.llep_combine_to_bf16(layer.params, rows, layer.pair_row, gates, want)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
