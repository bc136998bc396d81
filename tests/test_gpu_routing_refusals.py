"""Routing tensors that a kernel would read past their end, or as another type,
are refused before anything is enqueued: token ids and gates of the layer with
8-bit experts and of the expert block, and what llep_combine_to_bf16 reads."""

import pytest

from gpu_util import device
from test_gpu_block import Case

pytestmark = pytest.mark.gpu

REFUSED = (TypeError, ValueError)


@pytest.fixture(scope="module")
def dev():
    return device()


def _bad_routing(ids, gates):
    """(ids, gates), one of them not what a layer of [T, K] pairs takes."""
    T, K = ids.shape
    for bad in (ids.long(), ids[:T - 1], ids.view(-1)[:T * K - 1], ids.cpu(), None,
                ids.repeat(1, 2)[:, :K], ids.t(), ids.float()):
        yield bad, gates
    for bad in (gates.bfloat16(), gates.double(), gates[:T - 1], gates[:, :1].contiguous(),
                gates.cpu(), None, gates.repeat(1, 2)[:, :K]):
        yield ids, bad


def test_layer_and_block(dev):
    import torch
    from paper_2601_17111_amd.layer import Int8Experts
    c = Case(dev, 37, "bf16", "channel", seed=3)
    experts = Int8Experts.from_weights(*c.w)
    layer = c.block.layer
    for ids, gates in _bad_routing(c.ids, c.gates):
        with pytest.raises(REFUSED):
            layer.forward_int8(ids, gates, c.x, experts)
        with pytest.raises(REFUSED):
            c.block.forward_int8(ids, gates, c.x, experts)
        with pytest.raises(REFUSED):
            c.block.forward(ids, gates, c.x, *c.packed)
    # one after another is as good as [T, K]
    y = layer.forward_int8(c.ids, c.gates, c.x, experts).clone()
    flat = layer.forward_int8(c.ids.view(-1), c.gates.view(-1), c.x, experts)
    torch.cuda.synchronize()
    assert torch.equal(y, flat)
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    for _, gates in _bad_routing(c.ids, c.gates):
        if gates is not c.gates:
            with pytest.raises(REFUSED):
                c.block.backward(c.x, c.d_r, c.d_h, gates, c.packed[0], *c.packed_t)


def test_combine(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    T, K, D = 9, 2, 64
    p = B.make_params(T, K, 4, 2, T * K)
    rows = torch.randn((T * K, D), device=dev)
    where = torch.randperm(T * K, device=dev).to(torch.int32)
    gates = torch.rand((T, K), device=dev)
    y = torch.empty((T, D), dtype=torch.bfloat16, device=dev)
    for pair_row in (where.long(), where[:T * K - 1], where.cpu(), None,
                     where.repeat_interleave(2)[::2]):
        with pytest.raises(REFUSED):
            B.llep_combine_to_bf16(p, rows, pair_row, gates, y)
    for bad in (gates.bfloat16(), gates[:T - 1], gates[:, :1].contiguous(), gates.cpu(),
                gates.repeat(1, 2)[:, :K]):
        with pytest.raises(REFUSED):
            B.llep_combine_to_bf16(p, rows, where, bad, y)
    # longer lists of rows, flat gates, and none of them (sums)
    long = torch.cat([where, where])
    want = torch.empty_like(y)
    B.llep_combine_to_bf16(p, rows, where, gates, want)
    B.llep_combine_to_bf16(p, rows, long, gates.view(-1), y)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    B.llep_combine_to_bf16(p, rows, where, None, y)
    torch.cuda.synchronize()
    assert torch.equal(y, rows[where.long()].view(T, K, D).sum(1).bfloat16())
