"""MXFP4: 4-bit weights and activations with a power-of-two scale for 32 elements. Python side of include/mxfp4_linear.h.

Marshalling only: tensors are allocated with torch and handed to the C ABI; the work runs in the library's kernels on the
tensors' device and that device's current stream. The format, the layouts and the arithmetic are stated in the header.
"""
from __future__ import annotations

import torch

from . import binding
from .binding import W8A8Error, _i64, _int, _lib, _raw_stream, _sz, _vp

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

# torch's own short way to the current device, where it has one
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def call(fn, where: str, dev: int, *args) -> None:
    """fn(*args, stream) on CUDA device `dev` and its current stream; raises W8A8Error unless it returns OK."""
    if dev < 0:
        raise ValueError(f"{where}: tensors must be on a CUDA device")
    if dev == _current_device():
        status = fn(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(dev))
    if status != 0:
        raise W8A8Error(status, where)


def different_devices(where: str) -> ValueError:
    return ValueError(f"{where}: tensors are on different devices")


def _scale_shape(rows: int, K: int) -> tuple[int, int, int]:
    return ((rows + 127) // 128, (K + 127) // 128, 512)


def _need_codes(codes: torch.Tensor, scales: torch.Tensor, name: str) -> tuple[int, int]:
    """Checks packed codes and their scale tiles; returns (rows, K)."""
    if codes.dtype is not torch.uint8 or codes.dim() != 2 or scales.dtype is not torch.uint8:
        raise TypeError(f"{name}: uint8 codes [rows, K/2] and uint8 scale tiles expected")
    rows, half = codes.shape
    if scales.shape != ((rows + 127) // 128, (half + 63) // 64, 512) or not scales.is_contiguous():
        raise ValueError(f"{name}: scale tiles must be dense {_scale_shape(rows, 2 * half)}, got {tuple(scales.shape)}")
    return rows, 2 * half


def mxfp4_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None):
    """bf16 or fp32 [M,K] -> (codes uint8 [M,K/2], scale tiles uint8 [ceil(M/128), ceil(K/128), 512])."""
    dtype = _DTYPES.get(x.dtype)
    if dtype is None or x.dim() != 2:
        raise TypeError(f"x: bf16 or fp32 [M,K] expected, got {x.dtype} {tuple(x.shape)}")
    M, K = x.shape
    ldx, one = x.stride()
    if one != 1 and K > 1:
        raise TypeError("x: rows must be contiguous")
    dev = x.get_device()
    if codes is None:
        codes = torch.empty(M, K // 2, dtype=torch.uint8, device=x.device)
    elif codes.dtype is not torch.uint8 or codes.shape != (M, K // 2) or not codes.is_contiguous():
        raise ValueError("codes must be dense uint8 [M, K/2]")
    elif codes.get_device() != dev:
        raise different_devices("mxfp4_quantize")
    if scales is None:
        scales = torch.empty((M + 127) // 128, (K + 127) // 128, 512, dtype=torch.uint8, device=x.device)
    elif scales.dtype is not torch.uint8 or scales.shape != _scale_shape(M, K) or not scales.is_contiguous():
        raise ValueError(f"scales must be dense uint8 {_scale_shape(M, K)}")
    elif scales.get_device() != dev:
        raise different_devices("mxfp4_quantize")
    call(_lib.mxfp4_quantize, "mxfp4_quantize", dev, x.data_ptr(), dtype, M, K, ldx if M > 1 else K, codes.data_ptr(), scales.data_ptr())
    return codes, scales


def mxfp4_dequantize(codes: torch.Tensor, scales: torch.Tensor, out: torch.Tensor | None = None, dtype=torch.bfloat16) -> torch.Tensor:
    """The values that codes and scale tiles stand for, exactly: bf16 or fp32 [M,K] (out's dtype, if out is given)."""
    M, K = _need_codes(codes, scales, "codes")
    if not codes.is_contiguous():
        raise ValueError("codes must be dense [M, K/2]")
    dev = codes.get_device()
    if out is None:
        kind = _DTYPES.get(dtype)
        if kind is None:
            raise TypeError(f"dtype: bf16 or fp32 expected, got {dtype}")
        out = torch.empty(M, K, dtype=dtype, device=codes.device)
        ldo = K
    else:
        kind = _DTYPES.get(out.dtype)
        if kind is None or out.dim() != 2 or out.stride(1) != 1:
            raise TypeError(f"out: bf16 or fp32 with contiguous rows expected, got {out.dtype}")
        if out.shape != (M, K):
            raise ValueError("out must be [M, K]")
        ldo = out.stride(0) if M > 1 else K
        if out.get_device() != dev:
            raise different_devices("mxfp4_dequantize")
    if scales.get_device() != dev:
        raise different_devices("mxfp4_dequantize")
    call(_lib.mxfp4_dequantize, "mxfp4_dequantize", dev, codes.data_ptr(), scales.data_ptr(), M, K, out.data_ptr(), kind, ldo)
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
    N, K = _need_codes(qw, sw, "qw")
    if not qw.is_contiguous():
        raise TypeError("qw must be dense")
    if A.dim() != 2:
        raise TypeError("A: rank 2 expected")
    M, columns = A.shape
    lda, one = A.stride()
    if one != 1 and columns > 1:
        raise TypeError("A: rows must be contiguous")
    dev = A.get_device()
    if a_scales is None:
        if A.dtype is not torch.bfloat16:
            raise TypeError(f"A: bf16 expected, got {A.dtype}")
        a_dtype, sa = MXFP4_BF16, None
        if columns != K:
            raise ValueError(f"shape mismatch: A has K = {columns}, the weights {K}")
        if M == 1:
            lda = K
    else:
        _need_codes(A, a_scales, "A")
        if 2 * columns != K:
            raise ValueError(f"shape mismatch: A has K = {2 * columns}, the weights {K}")
        if a_scales.get_device() != dev:
            raise different_devices("mxfp4_linear_fused")
        a_dtype, sa = MXFP4_CODES, a_scales.data_ptr()
        if M == 1:
            lda = columns
    if bias is None:
        b = None
    else:
        if bias.dtype is not torch.float32 or bias.shape != (N,) or not bias.is_contiguous():
            raise TypeError("bias: dense fp32 [N] expected")
        if bias.get_device() != dev:
            raise different_devices("mxfp4_linear_fused")
        b = bias.data_ptr()
    if out is None:
        out = torch.empty(M, N, dtype=torch.bfloat16, device=A.device)
        ldo = N
    else:
        if out.dtype is not torch.bfloat16 or out.shape != (M, N):
            raise TypeError("out: bf16 [M,N] expected")
        ldo, one = out.stride()
        if one != 1 and N > 1:
            raise TypeError("out: rows must be contiguous")
        if M == 1:
            ldo = N
        if out.get_device() != dev:
            raise different_devices("mxfp4_linear_fused")
    if workspace is None:
        workspace = mxfp4_alloc_workspace(M, N, K, A.device)
    elif not workspace.is_contiguous():
        raise TypeError("workspace: dense tensor expected")          # (its size is what the kernels may write)
    elif workspace.get_device() != dev:
        raise different_devices("mxfp4_linear_fused")
    if qw.get_device() != dev or sw.get_device() != dev:
        raise different_devices("mxfp4_linear_fused")
    call(_lib.mxfp4_linear_fused, "mxfp4_linear_fused", dev, A.data_ptr(), a_dtype, lda, sa, qw.data_ptr(), sw.data_ptr(), b,
         out.data_ptr(), ldo, M, N, K, workspace.data_ptr(), workspace.nbytes)
    return out
