"""The feed-forward half of a transformer layer in 8-bit integers, through the C ABI:

    stream = x + residual
    y = stream + down( round8( silu(gate) * up ) )      gate, up = products of round8( rmsnorm(stream) )

This file only allocates tensors and sequences calls; all arithmetic is in the library's kernels.
"""
from __future__ import annotations

from . import binding as nm


class FeedForwardQ8:
    """gamma: fp32 [width]; up: gated weights (2 * hidden channels of `width`); down: `width` channels of `hidden`.
    Weights packed by nm_q8_pack; from_float() makes all three from fp32 or bf16 tensors."""

    def __init__(self, gamma, up: nm.Q8Weights, down: nm.Q8Weights, eps: float = 1e-6):
        if not up.gated or down.gated:
            raise ValueError("up must be packed gated, down plain")
        if up.outs != down.width or down.channels != up.width:
            raise ValueError(f"up {up.channels} x {up.width} and down {down.channels} x {down.width} do not fit together")
        self.gamma, self.up, self.down, self.eps = gamma, up, down, eps

    @classmethod
    def from_float(cls, gamma, gate_w, up_w, down_w, eps: float = 1e-6):
        """gate_w, up_w [hidden, width], down_w [width, hidden] on the device, fp32 or bf16."""
        import torch
        return cls(gamma, nm.nm_q8_pack(torch.cat([gate_w, up_w]), gated=True), nm.nm_q8_pack(down_w), eps)

    def forward(self, x, residual=None, stream=None):
        """x, residual: [..., width] in bf16 or fp32.  Returns the new residual stream, shaped and typed like x."""
        q, s, h = nm.nm_rmsnorm_q8(x, self.gamma, residual, self.eps, stream=stream)
        hidden = nm.nm_linear_q8(q, s, self.up, dtype=x.dtype, stream=stream)
        q, s = nm.nm_quantize_q8(hidden, stream=stream)
        return nm.nm_linear_q8(q, s, self.down, residual=x if h is None else h, dtype=x.dtype, stream=stream)

    __call__ = forward
