"""A batch of no tokens through the layer with 8-bit experts and through the
expert block: no error, outputs of no rows, weight gradients of zero."""

import pytest

from gpu_util import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_no_tokens(dev, gate):
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.block import ExpertBlock
    from paper_2601_17111_amd.layer import Int8Experts, LLEPLayer
    K, E, D, F = 2, 4, 64, 128
    bf = dict(dtype=torch.bfloat16, device=dev)
    w = [torch.ones(s, **bf) for s in ((E, D, F), (E, D, F), (E, F, D))]
    ids = torch.empty((0, K), dtype=torch.int32, device=dev)
    gates = torch.empty((0, K), device=dev)
    x = torch.empty((0, D), **bf)
    layer = LLEPLayer(0, K, E, 2, D, F, 1, torch.bfloat16, dev)
    experts = Int8Experts.from_weights(*w)
    assert layer.forward_int8(ids, gates, x, experts).shape == (0, D)
    assert layer.forward_int8(ids, gates, torch.empty((0, D), dtype=torch.int8, device=dev),
                              experts, x_scale=torch.empty(0, device=dev)).shape == (0, D)
    shape = {"none": None, "channel": (1, D), "token": (0, 1), "full": (0, D)}[gate]
    one = torch.ones(D, **bf)
    block = ExpertBlock(layer, one, one, None if shape is None else torch.ones(shape, **bf), one)
    r, h = block.forward_int8(ids, gates, x, experts)
    assert r.shape == h.shape == (0, D)
    packed, packed_t = B.llep_pack_weights(*w), B.llep_pack_weights_backward(*w)
    r, h = block.forward(ids, gates, x, *packed)
    assert r.shape == h.shape == (0, D)
    dx, d_gates, grads = block.backward(x, x, x, gates, packed[0], *packed_t)
    norm = block.clip(grads, 1.0)
    torch.cuda.synchronize()
    assert dx.shape == (0, D) and d_gates.shape == (0, K) and float(norm) == 0.0
    assert not any(bool(g.any()) for g in grads.values())
