"""The feed-forward half of a transformer layer in 8-bit integers or in MX4, and with experts, through the C ABI:

    stream = x + residual
    y = stream + down( round( silu(gate) * up ) )       gate, up = products of round( rmsnorm(stream) )

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


class FeedForwardMX4:
    """gamma: fp32 [width]; up: gated weights (2 * hidden channels of `width`); down: `width` channels of `hidden`.
    Weights packed by nm_mx4_pack; from_float() makes all three from fp32 or bf16 tensors."""

    def __init__(self, gamma, up: nm.MX4Weights, down: nm.MX4Weights, eps: float = 1e-6):
        _check_pair(up, down)
        if up.experts != 1:
            raise ValueError("up and down must be the weights of one expert")
        self.gamma, self.up, self.down, self.eps = gamma, up, down, eps

    @classmethod
    def from_float(cls, gamma, gate_w, up_w, down_w, eps: float = 1e-6):
        """gate_w, up_w [hidden, width], down_w [width, hidden] on the device, fp32 or bf16."""
        import torch
        return cls(gamma, nm.nm_mx4_pack(torch.cat([gate_w, up_w]), gated=True), nm.nm_mx4_pack(down_w), eps)

    def forward(self, x, residual=None, stream=None):
        """x, residual: [..., width] in bf16 or fp32.  Returns the new residual stream, shaped and typed like x."""
        q, s, h = nm.nm_rmsnorm_mx4(x, self.gamma, residual, self.eps, stream=stream)
        q, s = nm.nm_linear_mx4(q, s, self.up, rounded=True, stream=stream)
        return nm.nm_linear_mx4(q, s, self.down, residual=x if h is None else h, dtype=x.dtype, stream=stream)

    __call__ = forward


class ExpertsMX4:
    """A layer of experts: up: gated weights of each (2 * hidden channels of `width`), down: `width` channels of `hidden`;
    every token goes through the k experts with its largest logits, whose answers are weighted with their softmax.
    answers: the type in which an expert's answer goes to that sum.  fp32 (the default): only the sum is rounded, to x's type.  bf16
    halves the answers' bytes and rounds each of them, by 2^-8 of itself at most.
    from_float() makes the weights from fp32 or bf16 tensors."""

    def __init__(self, up: nm.MX4Weights, down: nm.MX4Weights, k: int, normalise: bool = True, answers=None):
        import torch
        _check_pair(up, down)
        if up.experts != down.experts or not 1 <= k <= up.experts:
            raise ValueError(f"up has {up.experts} experts, down {down.experts}; {k} are chosen")
        if answers not in (None, torch.float32, torch.bfloat16):
            raise ValueError(f"answers are fp32 or bf16, not {answers}")
        self.up, self.down, self.k, self.normalise, self.answers = up, down, k, normalise, answers or torch.float32

    @classmethod
    def from_float(cls, gate_w, up_w, down_w, k: int, normalise: bool = True, answers=None):
        """gate_w, up_w [experts, hidden, width], down_w [experts, width, hidden] on the device, fp32 or bf16."""
        import torch
        return cls(nm.nm_mx4_pack(torch.cat([gate_w, up_w], dim=1), gated=True), nm.nm_mx4_pack(down_w), k, normalise, answers)

    def forward(self, x, logits, residual=None, stream=None):
        """x, residual: [..., width] in bf16 or fp32 (x: the normalised rows); logits [..., experts].  Returns residual plus the
        experts' answers, shaped and typed like x."""
        if x.shape[-1] != self.up.width:   # (blocks of 32 alone would let other widths pass)
            raise ValueError(f"rows of {x.shape[-1]} values for experts of {self.up.width}")
        if x.shape[:-1] != logits.shape[:-1] or logits.shape[-1] != self.up.experts:
            raise ValueError(f"rows {tuple(x.shape)} and logits {tuple(logits.shape)} for {self.up.experts} experts do not fit together")
        to = nm.nm_route(logits, self.k, self.normalise, stream=stream)
        q, s = nm.nm_quantize_mx4(x, stream=stream)
        q, s = nm.nm_experts_mx4(q, s, self.up, to.offsets, to.rows, rounded=True, stream=stream)
        y = nm.nm_experts_mx4(q, s, self.down, to.offsets, dtype=self.answers, stream=stream)
        return nm.nm_combine(y, to.slots, to.weights, residual, dtype=x.dtype, stream=stream)

    __call__ = forward


def _check_pair(up, down):
    if not up.gated or down.gated:
        raise ValueError("up must be packed gated, down plain")
    if up.outs != down.width or down.channels != up.width:
        raise ValueError(f"up {up.channels} x {up.width} and down {down.channels} x {down.width} do not fit together")
