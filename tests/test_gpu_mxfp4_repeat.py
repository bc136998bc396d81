"""The 4-bit expert layer repeats itself: the same bits in every pass, whatever its buffers
hold from before and whatever another layer has run in between."""

import numpy as np
import pytest

from gpu_util import device
from test_gpu_mxfp4_experts import _experts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,E,P,D,F,hot", [
    (5, 4, 16, 4, 320, 192, 0.5), (600, 2, 4, 2, 1088, 1216, 0.3), (975, 4, 16, 4, 1344, 2112, 0.3),
    (1531, 8, 128, 8, 2048, 768, 0.6)])
def test_same_bits_in_every_pass(T, K, E, P, D, F, hot):
    import torch
    from paper_2601_17111_amd.layer import LLEPLayer
    dev = device()
    g = np.random.default_rng(T)
    experts, _ = _experts(g, dev, E, D, F)
    ids = np.where(g.random((T, K)) < hot, 0, g.integers(0, E, (T, K))).astype(np.int32)
    ids = torch.from_numpy(ids).to(dev)
    gates = torch.from_numpy(g.uniform(0, 1, (T, K)).astype(np.float32)).to(dev)
    x = torch.from_numpy(g.normal(size=(T, D))).to(dev).bfloat16()
    layer, other = (LLEPLayer(T, K, E, P, D, F, -(-T * K * 11 // (10 * P)), torch.bfloat16, dev) for _ in "ab")
    want = layer.forward_mxfp4(ids, gates, x, experts).clone()
    for i in range(12):
        if i % 3 == 1:
            other.forward_mxfp4(ids, gates, -x, experts)
        if i % 3 == 2:
            for t in (layer.x_mx, layer.x_perm_mx, layer.mxfp4_workspace):
                t.fill_(255)
            layer.out_perm_mx.fill_(float("nan"))
            layer.y.fill_(float("nan"))
        assert torch.equal(layer.forward_mxfp4(ids, gates, x, experts), want), i
