"""Memory that a call with stream= allocates belongs to that stream: in the
current stream's pool it could still be in use by what is enqueued there."""

import pytest

from gpu_util import device
from test_gpu_block import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def _stream_of(t):
    """The stream that the allocator keeps t's memory for."""
    import torch
    at = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's memory")


def _tensors(o, skip=()):
    import torch
    out = {}
    for k, v in vars(o).items():
        if k in skip:
            continue
        for i, t in enumerate(v.values() if isinstance(v, dict) else [v]):
            if isinstance(t, torch.Tensor) and t.is_cuda and t.numel():
                out[f"{type(o).__name__}.{k}[{i}]"] = t
    return out


def test_allocations_are_the_streams_own(dev):
    import torch
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts
    c = Case(dev, 37, "bf16", "channel", seed=3)
    block, layer = c.block, c.block.layer
    q = [torch.ones(s, dtype=torch.int8, device=dev)
         for s in ((c.E, c.F, c.D), (c.E, c.F, c.D), (c.E, c.D, c.F))]
    sc = [torch.ones(s, device=dev) * 0.001 for s in ((c.E, c.F), (c.E, c.F), (c.E, c.D))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    here = {**_tensors(block), **_tensors(layer)}
    made = {}
    made["matrix"] = B.llep_pack_matrix_int8(q[0], stream=side)
    made["gate_up"], made["down"] = B.llep_pack_weights(*c.w, stream=side)
    made["gate_up_t"], made["down_t"] = B.llep_pack_weights_backward(*c.w, stream=side)
    experts = Int8Experts(q[0], sc[0], q[1], sc[1], q[2], sc[2], stream=side)
    made["experts.gate_up"], made["experts.down"] = experts.gate_up, experts.down
    layer.forward_int8(c.ids, c.gates, c.x, experts, stream=side)
    block.forward_int8(c.ids, c.gates, c.x, experts, stream=side)
    block.forward(c.ids, c.gates, c.x, made["gate_up"], made["down"], stream=side)
    _, _, grads = block.backward(c.x, c.d_r, c.d_h, c.gates, made["gate_up"], made["gate_up_t"],
                                 made["down_t"], stream=side)
    block.clip(grads, 1.0, stream=side)
    side.synchronize()
    made.update({k: t for k, t in {**_tensors(block), **_tensors(layer)}.items() if k not in here})
    assert len(made) > 25
    for k, t in made.items():
        assert _stream_of(t) == side.cuda_stream, k
