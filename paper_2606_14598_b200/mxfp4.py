"""MXFP4: 4-bit weights and activations with a power-of-two scale for 32 elements. Python side of include/mxfp4_linear.h.

Marshalling only: tensors are allocated with torch and handed to the C ABI; the work runs in the library's kernels on the
tensors' device and that device's current stream. The format, the layouts and the arithmetic are stated in the header.
"""
from __future__ import annotations

import torch

from . import binding
from .binding import W8A8Error, _i64, _int, _lib, _sz, _vp

MXFP4_BF16, MXFP4_FP32, MXFP4_CODES = 0, 1, 2
MXFP4_K_MAX = 1 << 24
MXFP4_NUM_CONFIGS = 3
_DTYPES = {torch.bfloat16: MXFP4_BF16, torch.float32: MXFP4_FP32}

_lib.mxfp4_scale_bytes.argtypes = [_i64, _i64]
_lib.mxfp4_scale_bytes.restype = _sz
_lib.mxfp4_quantize.argtypes = [_vp, _int, _i64, _i64, _i64, _vp, _vp, _vp]
_lib.mxfp4_quantize.restype = _int
_lib.mxfp4_dequantize.argtypes = [_vp, _vp, _i64, _i64, _vp, _int, _i64, _vp]
_lib.mxfp4_dequantize.restype = _int
_lib.mxfp4_linear_workspace_bytes.argtypes = [_i64, _i64, _i64]
_lib.mxfp4_linear_workspace_bytes.restype = _sz
_lib.mxfp4_linear_fused.argtypes = [_vp, _int, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _sz, _vp]
_lib.mxfp4_linear_fused.restype = _int
_lib.mxfp4_linear_force_config.argtypes = [_int]
_lib.mxfp4_linear_force_config.restype = _int

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def call(fn, where: str, t: torch.Tensor, *args) -> None:
    """fn(*args, stream) on t's device and that device's current stream; raises W8A8Error unless it returns OK."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{where}: tensors must be on a CUDA device")
    if dev == torch._C._cuda_getDevice():
        status = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(dev))
    if status != 0:
        raise W8A8Error(status, where)


def same_device(where: str, t: torch.Tensor, *others) -> None:
    dev = t.get_device()
    for o in others:
        if o is not None and o.get_device() != dev:
            raise ValueError(f"{where}: tensors are on different devices")


def _scale_shape(rows: int, K: int) -> tuple[int, int, int]:
    return ((rows + 127) // 128, (K + 127) // 128, 512)


def _need_codes(codes: torch.Tensor, scales: torch.Tensor, name: str) -> None:
    if codes.dtype != torch.uint8 or codes.dim() != 2 or scales.dtype != torch.uint8:
        raise TypeError(f"{name}: uint8 codes [rows, K/2] and uint8 scale tiles expected")
    if codes.stride(1) != 1:
        raise TypeError(f"{name}: rows must be contiguous")
    if tuple(scales.shape) != _scale_shape(codes.shape[0], 2 * codes.shape[1]) or not scales.is_contiguous():
        raise ValueError(f"{name}: scale tiles must be dense {_scale_shape(codes.shape[0], 2 * codes.shape[1])}, got {tuple(scales.shape)}")


def mxfp4_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None):
    """bf16 or fp32 [M,K] -> (codes uint8 [M,K/2], scale tiles uint8 [ceil(M/128), ceil(K/128), 512])."""
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or x.dim() != 2 or x.stride(1) != 1:
        raise TypeError(f"x: bf16 or fp32 [M,K] with contiguous rows expected, got {x.dtype} {tuple(x.shape)} {x.stride()}")
    M, K = x.shape
    if codes is None:
        codes = torch.empty((M, K // 2), dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty(_scale_shape(M, K), dtype=torch.uint8, device=x.device)
    _need_codes(codes, scales, "codes")
    if codes.shape[0] != M or codes.shape[1] * 2 != K or not codes.is_contiguous():
        raise ValueError("codes must be dense [M, K/2]")
    same_device("mxfp4_quantize", x, codes, scales)
    call(_lib.mxfp4_quantize, "mxfp4_quantize", x, x.data_ptr(), dtype, M, K, x.stride(0), codes.data_ptr(), scales.data_ptr())
    return codes, scales


def mxfp4_dequantize(codes: torch.Tensor, scales: torch.Tensor, out: torch.Tensor | None = None, dtype=torch.bfloat16) -> torch.Tensor:
    """The values that codes and scale tiles stand for, exactly: bf16 or fp32 [M,K] (out's dtype, if out is given)."""
    _need_codes(codes, scales, "codes")
    if not codes.is_contiguous():
        raise ValueError("codes must be dense [M, K/2]")
    M, K = codes.shape[0], 2 * codes.shape[1]
    if out is None:
        out = torch.empty((M, K), dtype=dtype, device=codes.device)
    kind = _DTYPES.get(out.dtype)
    if kind is None or out.dim() != 2 or out.stride(1) != 1:
        raise TypeError(f"out: bf16 or fp32 with contiguous rows expected, got {out.dtype}")
    if out.shape[0] != M or out.shape[1] != K:
        raise ValueError("out must be [M, K]")
    same_device("mxfp4_dequantize", codes, scales, out)
    call(_lib.mxfp4_dequantize, "mxfp4_dequantize", codes, codes.data_ptr(), scales.data_ptr(), M, K, out.data_ptr(), kind, out.stride(0))
    return out


def mxfp4_force_config(config_id: int) -> int:
    """For sweeps and tests: the kernel configuration of the following linears (-1: chosen from the sizes). Returns the old one."""
    return int(_lib.mxfp4_linear_force_config(int(config_id)))


def mxfp4_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(_lib.mxfp4_linear_workspace_bytes(M, N, K))


def mxfp4_alloc_workspace(M: int, N: int, K: int, device="cuda") -> torch.Tensor:
    """Device scratch for mxfp4_linear_fused (torch caching-allocator blocks are 512-byte aligned)."""
    return torch.empty((mxfp4_linear_workspace_bytes(M, N, K),), dtype=torch.uint8, device=device)


def mxfp4_linear_fused(A: torch.Tensor, qw: torch.Tensor, sw: torch.Tensor, bias: torch.Tensor | None = None,
                       a_scales: torch.Tensor | None = None, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """out[M,N] bf16 = value(A) @ value(W)^T + bias. A is bf16 [M,K] (quantized inside the call), or codes uint8 [M,K/2]
    with their scale tiles a_scales; qw, sw are the weights from mxfp4_quantize."""
    _need_codes(qw, sw, "qw")
    if not qw.is_contiguous():
        raise TypeError("qw must be dense")
    if A.dim() != 2 or A.stride(1) != 1:
        raise TypeError("A: rank 2 with contiguous rows expected")
    N, K = qw.shape[0], 2 * qw.shape[1]
    M = A.shape[0]
    if a_scales is None:
        if A.dtype != torch.bfloat16:
            raise TypeError(f"A: bf16 expected, got {A.dtype}")
        a_dtype, columns = MXFP4_BF16, A.shape[1]
    else:
        _need_codes(A, a_scales, "A")
        a_dtype, columns = MXFP4_CODES, 2 * A.shape[1]
    if columns != K:
        raise ValueError(f"shape mismatch: A has K = {columns}, the weights {K}")
    if bias is not None and (bias.dtype != torch.float32 or bias.dim() != 1 or bias.shape[0] != N or bias.stride(0) != 1):
        raise TypeError("bias: fp32 [N] expected")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    elif out.dtype != torch.bfloat16 or out.dim() != 2 or out.shape[0] != M or out.shape[1] != N or out.stride(1) != 1:
        raise TypeError("out: bf16 [M,N] with contiguous rows expected")
    if workspace is None:
        workspace = mxfp4_alloc_workspace(M, N, K, A.device)
    same_device("mxfp4_linear_fused", A, a_scales, qw, sw, bias, out, workspace)
    call(_lib.mxfp4_linear_fused, "mxfp4_linear_fused", A, A.data_ptr(), a_dtype, A.stride(0), None if a_scales is None else a_scales.data_ptr(),
         qw.data_ptr(), sw.data_ptr(), None if bias is None else bias.data_ptr(), out.data_ptr(), out.stride(0), M, N, K,
         workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return out
