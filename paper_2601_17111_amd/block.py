"""One expert block of a transformer around an LLEPLayer: the norm before the
experts, the experts, and the norm, gate and residual scale after them together
with the norm before the next block; its backward; and the clipping of all of
its gradients. Allocation and call sequencing only, as in layer.py."""

from __future__ import annotations

from typing import Optional

from . import binding as B
from .layer import Int8Experts, LLEPLayer


class ExpertBlock:
    """h = norm(x) w_pre;  y = experts(h);  r = x + alpha gate norm(y) w_post;
    h_next = norm(r) w_next.

    x, r, h, h_next [T, D] in the layer's type, D at most LLEP_MAX_NORM_DIM
    (layers on their own take longer rows); w_pre, w_post, w_next [D] and
    gate ([1, D], [T, 1], [T, D] or None) in the same type. w_post or w_next may
    be None (no norm after the experts; no norm before a next block). Buffers
    and streams as in LLEPLayer.
    """

    def __init__(self, layer: LLEPLayer, w_pre, w_post=None, gate=None, w_next=None,
                 alpha: float = 1.0, eps: float = 1e-5):
        import torch
        self.layer, self.alpha, self.eps = layer, alpha, eps
        self.w_pre, self.w_post, self.gate, self.w_next = w_pre, w_post, gate, w_next
        T, D = layer.T, layer.D
        if D > B.LLEP_MAX_NORM_DIM:
            raise ValueError(f"the norms take rows of up to {B.LLEP_MAX_NORM_DIM} elements, not {D}")
        row = dict(dtype=layer.dtype, device=layer.device)
        self.h = torch.empty((T, D), **row)
        self.r = torch.empty((T, D), **row)
        self.h_next = None if w_next is None else torch.empty((T, D), **row)

    def forward(self, ids, gates, x, w_gate_up, w_down, stream=None):
        """Training forward (packed weights of llep_pack_weights). Returns (r, h_next)."""
        self.layer.check_routing(ids, gates)
        B.llep_block_norm(x, None, None, None, self.w_pre, self.alpha, self.eps, None, self.h,
                          stream=stream)
        y = self.layer.forward(ids, gates, self.h, w_gate_up, w_down, -1, stream, True)
        return self._after(x, y, stream)

    def forward_int8(self, ids, gates, x, experts: Int8Experts, stream=None):
        """Serving forward with 8-bit experts (bf16 layers): the norm before them leaves its rows
        in 8 bits. Returns (r, h_next)."""
        self.layer.check_routing(ids, gates)
        if not hasattr(self, "h_q"):
            import torch
            T, D = self.layer.T, self.layer.D
            self.h_q = B._empty((T, D), torch.int8, self.layer.device, stream)
            self.h_scale = B._empty((T,), torch.float32, self.layer.device, stream)
        B.llep_block_norm(x, None, None, None, self.w_pre, self.alpha, self.eps, None, None,
                          self.h_q, self.h_scale, stream)
        y = self.layer.forward_int8(ids, gates, self.h_q, experts, -1, stream, self.h_scale)
        return self._after(x, y, stream)

    def _after(self, x, y, stream):
        B.llep_block_norm(x, y, self.gate, self.w_post, self.w_next, self.alpha, self.eps, self.r,
                          self.h_next, stream=stream, gate_shape=self._gate_shape())
        return self.r, self.h_next

    def _gate_shape(self) -> Optional[int]:
        """LLEP_GATE_* (a gate [1, D] is one per channel also where T is 1)."""
        return B._gate_shape(self.gate, self.layer.T, self.layer.D, None)

    def backward(self, x, d_r, d_h_next, gates, w_gate_up, w_gate_up_t, w_down_t, stream=None):
        """Backward of forward() for the gradients of r and h_next (None without w_next).

        Returns (dx, d_gates, grads): grads maps "w_gate", "w_up", "w_down" (float32, as in
        LLEPLayer.backward), "w_pre", "w_post", "gate" and "w_next" to their float32 gradients
        (those that the block has)."""
        import torch
        T, D = self.layer.T, self.layer.D
        self.layer.check_backward()
        B._pairs("gates", gates, self.layer.params, torch.float32)
        if not hasattr(self, "d_y"):
            dev = self.layer.device
            self.d_x, self.d_res, self.d_y = (
                B._empty((T, D), self.layer.dtype, dev, stream) for _ in range(3))
            self.d_w = {k: B._empty(w.shape, torch.float32, dev, stream) for k, w in
                        (("w_pre", self.w_pre), ("w_post", self.w_post), ("gate", self.gate),
                         ("w_next", self.w_next)) if w is not None}
            nbytes = B.llep_block_norm_backward_workspace_bytes(T, D)
            self.norm_workspace = B._empty((max(nbytes, 16),), torch.uint8, dev, stream)
        g = self.d_w
        B.llep_block_norm_backward(self.r, self.layer.y, self.gate, self.w_post, self.w_next,
                                   self.alpha, self.eps, d_r, d_h_next, self.d_res, self.d_y,
                                   g.get("gate"), g.get("w_post"), g.get("w_next"),
                                   self.norm_workspace, stream, self._gate_shape())
        dh, d_gates, dwg, dwu, dwd = self.layer.backward(self.d_y, gates, w_gate_up, w_gate_up_t,
                                                         w_down_t, -1, stream)
        B.llep_block_norm_backward(x, None, None, None, self.w_pre, self.alpha, self.eps,
                                   self.d_res, dh, self.d_x, None, None, None, g["w_pre"],
                                   self.norm_workspace, stream)
        return self.d_x, d_gates, {"w_gate": dwg, "w_up": dwu, "w_down": dwd, **g}

    def clip(self, grads, max_norm: float, stream=None):
        """Clips backward()'s gradients in place by their global norm; returns the norm [1]."""
        import torch
        if not hasattr(self, "grad_norm"):
            dev = self.layer.device
            self.grad_norm = B._empty((1,), torch.float32, dev, stream)
            self.clip_workspace = B._empty((B.llep_clip_gradients_workspace_bytes(),),
                                           torch.uint8, dev, stream)
        B.llep_clip_gradients(list(grads.values()), max_norm, self.grad_norm, self.clip_workspace,
                              stream=stream)
        return self.grad_norm
