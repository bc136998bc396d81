"""A refused call changes nothing: between a training forward and its backward,
8-bit calls with arguments that do not fit raise and leave the backward as it
would have been; and a backward that has no forward of its own is refused
before it writes."""

import pytest

from gpu_util import device
from test_gpu_block import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _back(c):
    import torch
    dx, d_gates, grads = c.block.backward(c.x, c.d_r, c.d_h, c.gates, c.packed[0], *c.packed_t)
    torch.cuda.synchronize()
    return [t.clone() for t in (dx, d_gates, *grads.values())]


@pytest.mark.parametrize("first_use", [True, False])
def test_training_survives_refused_serving(dev, first_use):
    import torch
    from paper_2601_17111_amd.layer import Int8Experts
    c = Case(dev, 37, "bf16", "channel", seed=3)
    layer, T, D = c.block.layer, c.T, c.D
    experts = Int8Experts.from_weights(*c.w)
    if not first_use:
        c.block.forward_int8(c.ids, c.gates, c.x, experts)
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    want = _back(c)
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    other = Int8Experts.from_weights(*[w[:4].contiguous() for w in c.w])
    q = torch.zeros((T, D), dtype=torch.int8, device=dev)
    s = torch.zeros(T, device=dev)
    off = torch.zeros(T * D + 8, dtype=torch.int8, device=dev)[8:].view(T, D)
    for args, kw in [((c.ids, c.gates, c.x[:, :32].contiguous(), experts), {}),
                     ((c.ids, c.gates, c.x[:5], experts), {}),
                     ((c.ids, c.gates, c.x.half(), experts), {}),
                     ((c.ids, c.gates, c.x.t().contiguous().t(), experts), {}),
                     ((c.ids, c.gates, q, experts), {}),
                     ((c.ids, c.gates, c.x, experts), dict(x_scale=s)),
                     ((c.ids, c.gates, q, experts), dict(x_scale=s[:5])),
                     ((c.ids, c.gates, q, experts), dict(x_scale=s.bfloat16())),
                     ((c.ids, c.gates, off, experts), dict(x_scale=s)),
                     ((c.ids, c.gates, c.x, other), {}),
                     ((c.ids, c.gates, c.x, experts, c.block.layer.P), {}),
                     ((c.ids, c.gates, c.x, experts, -2), {})]:
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            layer.forward_int8(*args, **kw)
    got = _back(c)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_scales_of_another_type_are_refused_when_packed(dev):
    import torch
    from paper_2601_17111_amd.layer import Int8Experts
    z = [torch.zeros(sh, dtype=t, device=dev) for sh, t in (
        ((2, 64, 64), torch.int8), ((2, 64), torch.float32)) * 3]
    Int8Experts(*z)
    for i in (1, 3, 5):
        off = torch.zeros(2 * 64 + 1, device=dev)[1:].view(2, 64)
        for bad in (z[i].bfloat16(), z[i].cpu(), z[i].t().contiguous().t(), off):
            with pytest.raises((TypeError, ValueError)):
                Int8Experts(*z[:i], bad, *z[i + 1:])


@pytest.mark.parametrize("D,F", [(64, 96), (72, 64)])
def test_layer_of_other_sizes(dev, D, F):
    """Before the plan that a refused call would leave behind."""
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts, LLEPLayer
    layer = LLEPLayer(4, 1, 2, 1, D, F, 4, torch.bfloat16, dev)
    z = [torch.zeros(sh, dtype=t, device=dev) for n in ((2, F), (2, F), (2, D))
         for sh, t in (((*n, D + F - n[1]), torch.int8), (n, torch.float32))]
    ids = torch.zeros((4, 1), dtype=torch.int32, device=dev)
    layer.bufs.loads.fill_(77)
    try:
        experts = Int8Experts(*z)
    except B.LLEPError:
        return  # sizes that cannot be packed
    with pytest.raises(B.LLEPError) as ei:
        layer.forward_int8(ids, torch.ones((4, 1), device=dev),
                           torch.zeros((4, D), dtype=torch.bfloat16, device=dev), experts)
    assert ei.value.code == B.LLEP_E_ARG
    torch.cuda.synchronize()
    assert bool((layer.bufs.loads == 77).all())


def test_backward_without_its_forward_writes_nothing(dev):
    import torch
    from paper_2601_17111_amd.layer import Int8Experts
    c = Case(dev, 20, "bf16", "token", seed=4)
    c.block.forward(c.ids, c.gates, c.x, *c.packed)
    dx, d_gates, grads = c.block.backward(c.x, c.d_r, c.d_h, c.gates, c.packed[0], *c.packed_t)
    torch.cuda.synchronize()
    before = [t.clone() for t in (dx, d_gates, *grads.values())]
    c.block.forward_int8(c.ids, c.gates, c.x, Int8Experts.from_weights(*c.w))
    with pytest.raises(RuntimeError):
        c.block.backward(c.x, c.d_r * 2, c.d_h, c.gates, c.packed[0], *c.packed_t)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dx, d_gates, *grads.values()), before))
