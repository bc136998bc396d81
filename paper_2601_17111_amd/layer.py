"""One MoE expert layer on one GPU with P virtual devices: owns the device
buffers and runs the four library calls in order. Allocation and call
sequencing only; all arithmetic happens in the library's kernels."""

from __future__ import annotations

from typing import List, Optional, Sequence

from . import binding as B


def m_local_bytes(groups: Sequence[Sequence[int]], P: int, D: int, F: int,
                  elem_bytes: int) -> List[int]:
    """Peak-memory model of each device's share (Sec. 3.2, Eq. 4) from a
    plan's group table: for every group (device, expert, row_start, n) its
    n x D token rows, the expert's three D x F SwiGLU matrices and its n x F
    intermediate, in bytes of `elem_bytes` per element."""
    out = [0] * P
    for g in groups:
        d, n = int(g[0]), int(g[3])
        out[d] += (n * (D + F) + 3 * D * F) * elem_bytes
    return out


class Int8Experts:
    """Expert weights in 8 bits for LLEPLayer.forward_int8, packed once.

    w_gate, w_up [E, F, D] and w_down [E, D, F] int8, rows = output channels,
    with a float32 scale for each: [E, F], [E, F], [E, D] (llep_quantize_rows
    on the transposed weights gives both).
    """

    def __init__(self, w_gate, gate_scale, w_up, up_scale, w_down, down_scale, stream=None):
        E, F, D = w_gate.shape
        if tuple(w_up.shape) != (E, F, D) or tuple(w_down.shape) != (E, D, F):
            raise ValueError("w_gate and w_up are [E, F, D], w_down is [E, D, F]")
        if (tuple(gate_scale.shape) != (E, F) or tuple(up_scale.shape) != (E, F)
                or tuple(down_scale.shape) != (E, D)):
            raise ValueError("scales are [E, F], [E, F] and [E, D]")
        import torch
        for what, t in (("gate_scale", gate_scale), ("up_scale", up_scale),
                        ("down_scale", down_scale)):
            B._dense(what, t, t.shape, torch.float32)
            if t.data_ptr() % 16:
                raise ValueError(f"{what} does not start on a 16-byte boundary")
        self.E, self.D, self.F = E, D, F
        self.gate_up = B.llep_pack_matrix_int8(w_gate, w_up, stream)
        self.down = B.llep_pack_matrix_int8(w_down, stream=stream)
        self.gate_scale, self.up_scale, self.down_scale = gate_scale, up_scale, down_scale

    @classmethod
    def from_weights(cls, w_gate, w_up, w_down, stream=None):
        """From the weights that llep_pack_weights takes: w_gate, w_up [E, D, F] and w_down
        [E, F, D] in bf16 or float32."""
        import torch
        parts = []
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
            for w in (w_gate, w_up, w_down):
                E, K, N = w.shape
                rows = w.transpose(1, 2).reshape(E * N, K)
                q = torch.empty((E * N, K), dtype=torch.int8, device=w.device)
                scale = torch.empty(E * N, dtype=torch.float32, device=w.device)
                B.llep_quantize_rows(rows, q, scale)
                parts += [q.view(E, N, K), scale.view(E, N)]
            return cls(*parts)


class LLEPLayer:
    """Buffers and calls for one layer shape.

    ids [T, K] int32, gates [T, K] float32, x [T, D] (bf16 or f32) are device
    tensors; w_gate_up / w_down are the packed weights (llep_pack_weights).
    The buffers made here are the current stream's: another stream that calls
    are given has to wait for it first. Those that a call makes are its stream's.
    """

    def __init__(self, T: int, K: int, E: int, P: int, D: int, F: int, capacity: int,
                 dtype, device="cuda", min_chunk: int = 1, lam: float = 0.0,
                 mode: str = "llep"):
        import torch
        self.T, self.K, self.E, self.P, self.D, self.F = T, K, E, P, D, F
        self.dtype = dtype
        self.device = device
        self.params = B.make_params(T, K, E, P, capacity, min_chunk, lam, mode)
        self.bufs = B.PlanBuffers(self.params, device)
        R = T * K
        self.x_perm = torch.empty((max(R, 1), D), dtype=dtype, device=device)
        self.out_perm = torch.empty((max(R, 1), D), dtype=dtype, device=device)
        self.gate_perm = torch.empty(max(R, 1), dtype=torch.float32, device=device)
        self.row_pair = torch.empty(max(R, 1), dtype=torch.int32, device=device)
        self.pair_row = torch.empty(max(R, 1), dtype=torch.int32, device=device)
        self.y = torch.empty((T, D), dtype=dtype, device=device)
        code = B.LLEP_BF16 if dtype == torch.bfloat16 else B.LLEP_F32
        nbytes = B.llep_grouped_ffn_workspace_bytes(self.params, F, code)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)

    def set_mode(self, mode: str):
        self.params.mode = B.LLEP_MODE_EP if mode == "ep" else B.LLEP_MODE_LLEP

    def plan(self, ids, stream=None):
        B.llep_plan(self.params, ids, self.bufs, stream)

    def permute(self, ids, gates, x, stream=None):
        self.rows_are_int8 = False
        B.llep_permute(self.params, self.bufs, ids, gates, x, self.x_perm, self.gate_perm,
                       self.row_pair, self.pair_row, stream)

    def ffn(self, w_gate_up, w_down, device: int = -1, stream=None, save_gate_up=False):
        """save_gate_up: keep g and u (self.gate_up) so that backward() does
        not recompute them."""
        if save_gate_up:
            if getattr(self, "gate_up", None) is None:
                self.gate_up = B._empty((max(self.T * self.K, 1), 2 * self.F), self.dtype,
                                        self.device, stream)
            B.llep_grouped_ffn_train(self.params, self.bufs, device, self.x_perm, w_gate_up,
                                     w_down, self.out_perm, self.gate_up, self.workspace, stream)
            self.gate_up_device = device
        else:
            B.llep_grouped_ffn(self.params, self.bufs, device, self.x_perm, w_gate_up, w_down,
                               self.out_perm, self.workspace, stream)
            self.gate_up_device = None

    def combine(self, gates, stream=None):
        B.llep_combine(self.params, self.out_perm, self.pair_row, gates, self.y, stream)

    def forward(self, ids, gates, x, w_gate_up, w_down, device: Optional[int] = -1,
                stream=None, save_gate_up=False):
        """plan -> permute -> grouped FFN (one device's groups, or all with -1)
        -> combine. Returns y (valid for every token only when device == -1).
        save_gate_up: training forward (g and u kept for backward())."""
        self.plan(ids, stream)
        self.permute(ids, gates, x, stream)
        self.ffn(w_gate_up, w_down, -1 if device is None else device, stream, save_gate_up)
        self.combine(gates, stream)
        return self.y

    def check_routing(self, ids, gates):
        """Refuses ids (int32) and gates (float32) that are not [T, K], or T K of them in order."""
        import torch
        B._pairs("ids", ids, self.params, torch.int32)
        B._pairs("gates", gates, self.params, torch.float32)

    def forward_int8(self, ids, gates, x, experts: Int8Experts, device: int = -1, stream=None,
                     x_scale=None):
        """forward() for serving with 8-bit experts (bf16 layers): the tokens to 8 bits, then
        plan -> permute (of the 8-bit rows) -> grouped FFN in 8 bits -> combine. Returns y (valid
        for every token only when device == -1).
        x [T, D] may already be 8-bit rows (int8), with their x_scale [T] (llep_block_norm and
        llep_quantize_rows write both). backward() is not available after it; a call that is
        refused changes nothing."""
        import torch
        if self.dtype != torch.bfloat16:
            raise TypeError("forward_int8 needs a bf16 layer")
        if (experts.E, experts.D, experts.F) != (self.E, self.D, self.F):
            raise ValueError("the experts do not fit this layer")
        if not -1 <= device < self.P:
            raise ValueError("device outside [-1, P)")
        self.check_routing(ids, gates)
        if x_scale is None:
            B._dense("x", x, (self.T, self.D), x.dtype)
            B._dtype_code(x)
        else:
            B._dense("x", x, (self.T, self.D), torch.int8)
            B._list("x_scale", x_scale, self.T, torch.float32)
            if x.data_ptr() % 16:
                raise ValueError("x does not start on a 16-byte boundary")
        if not hasattr(self, "int8_workspace"):
            self._make_int8_buffers(stream)
        if x_scale is None:
            B.llep_quantize_rows(x, self.x_q, self.x_scale, stream)
            x, x_scale = self.x_q, self.x_scale
        self.gate_up_device = None
        self.rows_are_int8 = True  # x_perm holds no rows of this call
        self.plan(ids, stream)
        self._permute_int8(ids, gates, x, stream)
        B.llep_grouped_ffn_int8(self.params, self.bufs, device, self.x_perm_q, x_scale,
                                self.row_pair, experts.gate_up, experts.gate_scale,
                                experts.up_scale, experts.down, experts.down_scale,
                                self.out_perm_wide, self.int8_workspace, stream)
        B.llep_combine_to_bf16(self.params, self.out_perm_wide, self.pair_row, gates, self.y,
                               stream)
        return self.y

    def _make_int8_buffers(self, stream):
        import torch
        R, D, dev = max(self.T * self.K, 1), self.D, self.device
        if D % 64 or self.F % 64 or max(D, self.F) > B.LLEP_MAX_FFN_DIM:
            raise B.LLEPError(B.LLEP_E_ARG, "forward_int8",
                              "D and F must be multiples of 64, at most LLEP_MAX_FFN_DIM")
        self.x_q = B._empty((self.T, D), torch.int8, dev, stream)
        self.x_scale = B._empty((self.T,), torch.float32, dev, stream)
        self.x_perm_q = B._empty((R, D), torch.int8, dev, stream)
        # the experts' outputs stay in float32, so that y is rounded once in any batch (in bfloat16
        # prompts take 5-6% less, but their tokens lose bits and differ from decode's)
        self.out_perm_wide = B._empty((R, D), torch.float32, dev, stream)
        nbytes = B.llep_grouped_ffn_int8_workspace_bytes(self.params, self.F)
        self.int8_workspace = B._empty((nbytes,), torch.uint8, dev, stream)

    def _permute_int8(self, ids, gates, x, stream):
        """The permutation of rows of D bytes, as D / 2 bfloat16."""
        import torch
        B.llep_permute(self.params, self.bufs, ids, gates, x.view(torch.bfloat16),
                       self.x_perm_q.view(torch.bfloat16), self.gate_perm, self.row_pair,
                       self.pair_row, stream)

    def _saved_covers(self, device: int) -> bool:
        saved = getattr(self, "gate_up_device", None)
        return saved is not None and (saved == -1 or saved == device)

    def check_backward(self):
        """Refuses a backward() whose rows forward_int8() has replaced."""
        if getattr(self, "rows_are_int8", False):
            raise RuntimeError("backward() after forward_int8()")

    def backward(self, dy, gates, w_gate_up, w_gate_up_t, w_down_t, device: int = -1,
                 stream=None):
        """Backward of forward() (bf16 or f32), reusing its plan, permutation and expert
        outputs: combine backward -> grouped FFN backward (one device's groups,
        or all with -1) -> the pairs' input gradients summed per token. Uses
        the g and u of a forward with save_gate_up (same device range), else
        recomputes them.

        Returns (dx [T, D], d_gates [T, K] float32, dw_gate, dw_up [E, D, F],
        dw_down [E, F, D] float32). dx and d_gates cover every token only when
        device == -1; the weight gradients are the device's partials, or with
        -1 the totals after the gradient return (experts without rows: zero).
        """
        import torch
        self.check_backward()
        if not hasattr(self, "d_out_perm"):
            R = max(self.T * self.K, 1)
            dev, E, D, F = self.device, self.E, self.D, self.F
            self.d_out_perm = B._empty((R, D), self.dtype, dev, stream)
            self.dx_perm = B._empty((R, D), self.dtype, dev, stream)
            self.d_gates = B._empty((self.T, self.K), torch.float32, dev, stream)
            self.dx = B._empty((self.T, D), self.dtype, dev, stream)
            self.dw_gate = B._empty((E, D, F), torch.float32, dev, stream)
            self.dw_up = B._empty((E, D, F), torch.float32, dev, stream)
            self.dw_down = B._empty((E, F, D), torch.float32, dev, stream)
            code = B.LLEP_BF16 if self.dtype == torch.bfloat16 else B.LLEP_F32
            nbytes = B.llep_grouped_ffn_backward_workspace_bytes(self.params, D, F, code)
            self.bwd_workspace = B._empty((nbytes,), torch.uint8, dev, stream)
        B.llep_zero_absent_gradients(self.params, self.bufs, device, self.dw_gate, self.dw_up,
                                     self.dw_down, stream)
        B.llep_combine_backward(self.params, self.out_perm, self.pair_row, gates, dy,
                                self.d_out_perm, self.d_gates, stream)
        B.llep_grouped_ffn_backward(self.params, self.bufs, device, self.x_perm, self.d_out_perm,
                                    w_gate_up, w_gate_up_t, w_down_t, self.dx_perm, self.dw_gate,
                                    self.dw_up, self.dw_down, self.bwd_workspace, stream,
                                    self.gate_up if self._saved_covers(device) else None)
        B.llep_combine(self.params, self.dx_perm, self.pair_row, None, self.dx, stream)
        return self.dx, self.d_gates, self.dw_gate, self.dw_up, self.dw_down
