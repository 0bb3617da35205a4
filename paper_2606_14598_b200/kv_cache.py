"""Quantized paged cache of keys and values. Python side of include/kv_cache.h (layouts and arithmetic are stated there).

    cache = QuantKVCache.empty(num_pages, page_size, heads, head_dim, "int8")       # or "mxfp4"
    kv_cache_write(cache, k, v, slots)                # new tokens [T, heads, dim] into slots = page * page_size + offset
    k, v = kv_cache_read(cache, table, cu_seqlens, total)
"""
from __future__ import annotations

import torch

from .binding import _i64, _int, _lib, _vp
from .mxfp4 import call, same_device

KV_CACHE_INT8, KV_CACHE_MXFP4 = 0, 1
KV_CACHE_MAX_DIM = 256

_lib.kv_cache_write.argtypes = [_int, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp]
_lib.kv_cache_write.restype = _int
_lib.kv_cache_read.argtypes = [_int, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64,
                               _vp, _i64, _i64, _vp, _i64, _i64, _vp]
_lib.kv_cache_read.restype = _int


class QuantKVCache:
    """The four tensors of a cache, dense: codes [num_pages, page_size, heads, dim] int8 with scales fp32 [.., heads], or
    [.., dim / 2] uint8 with scales uint8 [.., heads, ceil(dim / 32)]. The value side may be left out (None)."""

    def __init__(self, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor | None = None, v_scales: torch.Tensor | None = None):
        if k_codes.dim() != 4 or k_codes.dtype not in (torch.int8, torch.uint8):
            raise TypeError("codes: int8 or uint8 [num_pages, page_size, heads, ...] expected")
        self.fmt = KV_CACHE_INT8 if k_codes.dtype == torch.int8 else KV_CACHE_MXFP4
        self.num_pages, self.page_size, self.heads, last = k_codes.shape
        self.dim = last if self.fmt == KV_CACHE_INT8 else 2 * last
        lead = (self.num_pages, self.page_size, self.heads)
        if self.fmt == KV_CACHE_INT8:
            dtype, shape = torch.float32, lead
        else:
            dtype, shape = torch.uint8, lead + ((self.dim + 31) // 32,)
        if (v_codes is None) != (v_scales is None):
            raise ValueError("the value side needs both codes and scales")
        for name, codes, scales in (("k", k_codes, k_scales), ("v", v_codes, v_scales)):
            if codes is None:
                continue
            if codes.dtype != k_codes.dtype or codes.shape != k_codes.shape or not codes.is_contiguous():
                raise ValueError(f"{name}_codes: dense {k_codes.dtype} {tuple(k_codes.shape)} expected")
            if scales.dtype != dtype or tuple(scales.shape) != shape or not scales.is_contiguous():
                raise ValueError(f"{name}_scales: dense {dtype} {shape} expected")
        same_device("QuantKVCache", k_codes, k_scales, v_codes, v_scales)
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales

    @classmethod
    def empty(cls, num_pages: int, page_size: int, heads: int, dim: int, fmt: str = "int8", device="cuda", values: bool = True) -> "QuantKVCache":
        """A cache of zeros."""
        if fmt not in ("int8", "mxfp4"):
            raise ValueError(f"fmt: 'int8' or 'mxfp4' expected, got {fmt!r}")
        lead = (num_pages, page_size, heads)

        def side():
            if fmt == "int8":
                return torch.zeros(lead + (dim,), dtype=torch.int8, device=device), torch.zeros(lead, dtype=torch.float32, device=device)
            return (torch.zeros(lead + (dim // 2,), dtype=torch.uint8, device=device),
                    torch.zeros(lead + ((dim + 31) // 32,), dtype=torch.uint8, device=device))

        return cls(*side(), *(side() if values else (None, None)))


def _need_vectors(cache: QuantKVCache, t: torch.Tensor, name: str, rows: int) -> None:
    if t.dtype != torch.bfloat16 or t.dim() != 3 or t.stride(2) != 1:
        raise TypeError(f"{name}: bf16 [tokens, heads, dim] with contiguous heads expected, got {t.dtype} {tuple(t.shape)}")
    if t.shape[0] != rows or t.shape[1] != cache.heads or t.shape[2] != cache.dim:
        raise ValueError(f"{name}: [{rows}, {cache.heads}, {cache.dim}] expected, got {tuple(t.shape)}")


def kv_cache_write(cache: QuantKVCache, k: torch.Tensor, v: torch.Tensor | None, slots: torch.Tensor) -> None:
    """Quantizes k (and v) bf16 [T, heads, dim] into the cache at slots int64 [T]; slots outside the cache are skipped."""
    if slots.dtype != torch.int64 or slots.dim() != 1 or not slots.is_contiguous():
        raise TypeError("slots: dense int64 [tokens] expected")
    tokens = slots.shape[0]
    _need_vectors(cache, k, "k", tokens)
    if (v is None) != (cache.v_codes is None):
        raise ValueError("v goes with a cache that keeps values, and only with one")
    if v is not None:
        _need_vectors(cache, v, "v", tokens)
    same_device("kv_cache_write", cache.k_codes, k, v, slots)
    if tokens == 0:
        return
    c = cache
    call(_lib.kv_cache_write, "kv_cache_write", k, c.fmt, k.data_ptr(), k.stride(0), k.stride(1),
         None if v is None else v.data_ptr(), 0 if v is None else v.stride(0), 0 if v is None else v.stride(1), slots.data_ptr(), tokens,
         c.heads, c.dim, c.k_codes.data_ptr(), c.k_scales.data_ptr(), None if v is None else c.v_codes.data_ptr(),
         None if v is None else c.v_scales.data_ptr(), c.num_pages * c.page_size)


def kv_cache_read(cache: QuantKVCache, table: torch.Tensor, cu_seqlens: torch.Tensor, total: int, starts: torch.Tensor | None = None,
                  k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None):
    """The sequences' tokens as bf16 [total, heads, dim], one sequence after another: (k, v), or (k, None) without values.
    table int32 [B, max_pages], cu_seqlens int32 [B + 1], starts int32 [B] (first token to read of each) or None."""
    if table.dtype != torch.int32 or table.dim() != 2 or (table.numel() > 0 and table.stride(1) != 1):
        raise TypeError("table: int32 [sequences, max_pages] with contiguous rows expected")
    seqs, max_pages = table.shape
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.shape[0] != seqs + 1 or not cu_seqlens.is_contiguous():
        raise TypeError("cu_seqlens: dense int32 [sequences + 1] expected")
    if starts is not None and (starts.dtype != torch.int32 or starts.dim() != 1 or starts.shape[0] != seqs or not starts.is_contiguous()):
        raise TypeError("starts: dense int32 [sequences] expected")
    c = cache
    values = c.v_codes is not None
    if v_out is not None and not values:
        raise ValueError("v_out goes with a cache that keeps values")
    shape = (total, c.heads, c.dim)
    if k_out is None:
        k_out = torch.empty(shape, dtype=torch.bfloat16, device=c.k_codes.device)
    else:
        _need_vectors(c, k_out, "k_out", total)
    if values:
        if v_out is None:
            v_out = torch.empty(shape, dtype=torch.bfloat16, device=c.k_codes.device)
        else:
            _need_vectors(c, v_out, "v_out", total)
    same_device("kv_cache_read", c.k_codes, table, cu_seqlens, starts, k_out, v_out)
    if total == 0 or seqs == 0:
        return k_out, v_out
    call(_lib.kv_cache_read, "kv_cache_read", k_out, c.fmt, c.k_codes.data_ptr(), c.k_scales.data_ptr(),
         c.v_codes.data_ptr() if values else None, c.v_scales.data_ptr() if values else None, c.num_pages, c.page_size, c.heads, c.dim,
         table.data_ptr(), table.stride(0) if seqs > 1 else max_pages, max_pages, cu_seqlens.data_ptr(), None if starts is None else starts.data_ptr(),
         seqs, total, k_out.data_ptr(), k_out.stride(0), k_out.stride(1),
         v_out.data_ptr() if values else None, v_out.stride(0) if values else 0, v_out.stride(1) if values else 0)
    return k_out, v_out
