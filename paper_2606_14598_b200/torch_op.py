"""The fused W8A8 linear as a PyTorch custom operator and a drop-in module.

The paper lists a graph-safe custom operator as its first piece of future work (its own integration disabled
the graph tracer around every quantized linear, and the ablation with the compiler then broke the graph at each
of them). Registered through ``torch.library`` with a shape-only ("fake") implementation, the operator below is
opaque to the tracer but not a graph break: ``torch.compile(fullgraph=True)`` traces through modules that call it,
and because the library call allocates nothing and only enqueues on the current stream, the compiled function can
also be replayed from a CUDA graph.

Marshalling only: the operator's body is one call of the C ABI (``int8_linear_fused`` on bf16 activations); the
workspace it hands over is a torch allocation made inside the operator.
"""
from __future__ import annotations

import torch

from . import binding, mxfp4

__all__ = ["linear_fused", "W8A8Linear", "mxfp4_linear", "MXFP4Linear"]


def _rows(A: torch.Tensor) -> torch.Tensor:
    """[..., K] as the [M, K] that the kernels read: elements of a row side by side, rows apart by at least a row and by whole 16
    bytes, from a 16-byte boundary. Anything else (expanded rows, odd slices) is copied."""
    K = A.shape[-1]
    A2 = A.reshape(-1, K)
    if A2.stride(1) != 1 or A2.stride(0) < K or A2.stride(0) % 8 != 0 or A2.data_ptr() % 16 != 0:
        A2 = A2.clone(memory_format=torch.contiguous_format)
    return A2


class _FloatsStay(torch.nn.Module):
    """A module whose fp32 buffers (scales, bias) move with it but keep their type in .bfloat16(), .half() and .to(dtype): the
    kernels take fp32, and rounding the scales would change the weights."""

    def _apply(self, fn, recurse=True):
        kept = {name: b for name, b in self._buffers.items() if b is not None and b.dtype == torch.float32}
        super()._apply(fn, recurse)
        for name, b in kept.items():
            if self._buffers[name].dtype != torch.float32:
                self._buffers[name] = b.to(self._buffers[name].device)
        return self


@torch.library.custom_op("w8a8_b200::linear_fused", mutates_args=())
def linear_fused(A: torch.Tensor, qw: torch.Tensor, s_ch: torch.Tensor, bias: torch.Tensor | None) -> torch.Tensor:
    """bf16 [..., K] activations x int8 [N, K] per-channel weights -> bf16 [..., N] (quantize, int8 GEMM, dequantize)."""
    lead = A.shape[:-1]
    A2 = _rows(A)
    M, K = A2.shape
    N = qw.shape[0]
    out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    if M > 0:
        ws = binding.alloc_workspace(M, N, K, binding.ACT_BF16, A.device)
        binding.int8_linear_fused(A2, qw, s_ch, bias, out=out, workspace=ws)
    return out.reshape(*lead, N)


@linear_fused.register_fake
def _linear_fused_fake(A, qw, s_ch, bias):
    torch._check(A.dtype == torch.bfloat16, lambda: "activations must be bf16")
    torch._check(qw.dtype == torch.int8 and qw.dim() == 2, lambda: "weights must be int8 [N, K]")
    torch._check(A.shape[-1] == qw.shape[1], lambda: "K mismatch")
    return A.new_empty((*A.shape[:-1], qw.shape[0]), dtype=torch.bfloat16)


class W8A8Linear(_FloatsStay):
    """Drop-in replacement of an ``nn.Linear`` forward: weights are quantized once per output channel (on the
    device, by the library), activations per token on every call."""

    def __init__(self, qw: torch.Tensor, s_ch: torch.Tensor, bias: torch.Tensor | None = None):
        super().__init__()
        self.register_buffer("qw", qw)
        self.register_buffer("s_ch", s_ch)
        self.register_buffer("bias", bias)

    @classmethod
    def from_float(cls, weight: torch.Tensor, bias: torch.Tensor | None = None) -> "W8A8Linear":
        """weight: fp32 [N, K] on the CUDA device; bias: fp32 [N] or None."""
        qw, s_ch = binding.int8_quantize_weight_per_channel(weight.float().contiguous())
        return cls(qw, s_ch, None if bias is None else bias.float().contiguous())

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return linear_fused(x, self.qw, self.s_ch, self.bias)


@torch.library.custom_op("w8a8_b200::mxfp4_linear", mutates_args=())
def mxfp4_linear(A: torch.Tensor, qw: torch.Tensor, sw: torch.Tensor, bias: torch.Tensor | None) -> torch.Tensor:
    """bf16 [..., K] activations x MXFP4 weights (codes [N, K/2], scale tiles) -> bf16 [..., N]."""
    lead = A.shape[:-1]
    A2 = _rows(A)
    if A2.shape[0] == 0:
        return A.new_empty((*lead, qw.shape[0]), dtype=torch.bfloat16)
    return mxfp4.mxfp4_linear_fused(A2, qw, sw, bias).reshape(*lead, qw.shape[0])


@mxfp4_linear.register_fake
def _mxfp4_linear_fake(A, qw, sw, bias):
    torch._check(A.dtype == torch.bfloat16, lambda: "activations must be bf16")
    torch._check(qw.dtype == torch.uint8 and qw.dim() == 2, lambda: "weights must be uint8 codes [N, K/2]")
    torch._check(A.shape[-1] == 2 * qw.shape[1], lambda: "K mismatch")
    return A.new_empty((*A.shape[:-1], qw.shape[0]), dtype=torch.bfloat16)


class MXFP4Linear(_FloatsStay):
    """The 4-bit counterpart of W8A8Linear: weights are quantized to MXFP4 once, activations on every call."""

    def __init__(self, qw: torch.Tensor, sw: torch.Tensor, bias: torch.Tensor | None = None):
        super().__init__()
        self.register_buffer("qw", qw)
        self.register_buffer("sw", sw)
        self.register_buffer("bias", bias)

    @classmethod
    def from_float(cls, weight: torch.Tensor, bias: torch.Tensor | None = None) -> "MXFP4Linear":
        """weight: [N, K] on the CUDA device; bias: [N] or None."""
        qw, sw = mxfp4.mxfp4_quantize(weight.detach().float().contiguous())
        return cls(qw, sw, None if bias is None else bias.detach().float().contiguous())

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return mxfp4_linear(x, self.qw, self.sw, self.bias)
