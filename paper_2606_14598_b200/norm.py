"""Root-mean-square norm with the residual's addition, in front of a quantized linear. Python side of include/int8_norm.h (the arithmetic is stated there).

    qa, s_tok, h = int8_rmsnorm(x, weight, residual=h)       # codes for int8_linear_fused(qa, qw, s_ch, s_tok=s_tok)
    y, h = rmsnorm(x, weight, residual=h)                    # bf16, for mxfp4_linear_fused

For inference: autograd sees neither the calls nor what they write into sum_out, and results carry no gradients.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _i64, _int, _lib, _vp
from .mxfp4 import call, different_devices

INT8_NORM_K_MAX = 1 << 24
_WEIGHTS = {torch.float32: 0, torch.bfloat16: 1}

_lib.int8_rmsnorm.argtypes = [_vp, _i64, _vp, _i64, _vp, _int, ctypes.c_float, _i64, _i64, _vp, _i64, _vp, _vp, _vp, _i64, _vp]
_lib.int8_rmsnorm.restype = _int


def _matrix(t: torch.Tensor, name: str, shape, dev: int) -> int:
    """Checks bf16 [M, K] with contiguous rows on device `dev`; returns the row stride."""
    if t.dtype is not torch.bfloat16 or t.dim() != 2:
        raise TypeError(f"{name}: bf16 [M,K] expected, got {t.dtype} {tuple(t.shape)}")
    if t.shape != shape:
        raise ValueError(f"{name}: {list(shape)} expected, got {list(t.shape)}")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise TypeError(f"{name}: rows must be contiguous")
    if t.get_device() != dev:
        raise different_devices(name)
    return ld if shape[0] > 1 else shape[1]


def _inputs(x, weight, residual, sum_out):
    """Checks what both forms take: (device, M, K, the call's arguments up to s_tok's, h)."""
    dev = x.get_device()
    shape = x.shape
    ldx = _matrix(x, "x", shape, dev)
    M, K = shape
    kind = _WEIGHTS.get(weight.dtype)
    if kind is None or weight.dim() != 1 or not weight.is_contiguous():
        raise TypeError(f"weight: dense fp32 or bf16 [K] expected, got {weight.dtype} {tuple(weight.shape)}")
    if weight.shape[0] != K:
        raise ValueError(f"weight: [{K}] expected, got {list(weight.shape)}")
    if weight.get_device() != dev:
        raise different_devices("weight")
    if residual is None:
        rp, ldr, h = None, 0, x if sum_out is None else sum_out
    else:
        ldr = _matrix(residual, "residual", shape, dev)
        rp = residual.data_ptr()
        h = sum_out = torch.empty(M, K, dtype=torch.bfloat16, device=x.device) if sum_out is None else sum_out
    sp, lds = (None, 0) if sum_out is None else (sum_out.data_ptr(), _matrix(sum_out, "sum_out", shape, dev))
    return dev, M, K, (x.data_ptr(), ldx, rp, ldr, weight.data_ptr(), kind), (sp, lds), h


def int8_rmsnorm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: torch.Tensor | None = None, sum_out: torch.Tensor | None = None,
                 qa: torch.Tensor | None = None, s_tok: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """The norm of h = bf16(x + residual) as (codes int8 [M,K], scales fp32 [M], h). h is written to sum_out (which may be x or the
    residual itself); without a residual h is x. out, bf16 [M,K]: receives the norm in bf16 too."""
    dev, M, K, first, last, h = _inputs(x, weight, residual, sum_out)
    if qa is None:
        qa = torch.empty(M, K, dtype=torch.int8, device=x.device)
    elif qa.dtype is not torch.int8 or qa.shape != (M, K) or not qa.is_contiguous():
        raise ValueError(f"qa: dense int8 [{M}, {K}] expected")
    elif qa.get_device() != dev:
        raise different_devices("int8_rmsnorm")
    if s_tok is None:
        s_tok = torch.empty(M, dtype=torch.float32, device=x.device)
    elif s_tok.dtype is not torch.float32 or s_tok.shape != (M,) or not s_tok.is_contiguous():
        raise ValueError(f"s_tok: dense fp32 [{M}] expected")
    elif s_tok.get_device() != dev:
        raise different_devices("int8_rmsnorm")
    yp, ldy = (None, 0) if out is None else (out.data_ptr(), _matrix(out, "out", x.shape, dev))
    if M > 0:
        call(_lib.int8_rmsnorm, "int8_rmsnorm", dev, *first, eps, M, K, *last, qa.data_ptr(), s_tok.data_ptr(), yp, ldy)
    return qa, s_tok, h


def rmsnorm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, residual: torch.Tensor | None = None, sum_out: torch.Tensor | None = None,
            out: torch.Tensor | None = None):
    """The norm of h = bf16(x + residual) as (bf16 [M,K], h); h as for int8_rmsnorm."""
    dev, M, K, first, last, h = _inputs(x, weight, residual, sum_out)
    if out is None:
        out = torch.empty(M, K, dtype=torch.bfloat16, device=x.device)
    ldy = _matrix(out, "out", x.shape, dev)
    if M > 0:
        call(_lib.int8_rmsnorm, "rmsnorm", dev, *first, eps, M, K, *last, None, None, out.data_ptr(), ldy)
    return out, h
