"""Quantized paged cache of keys and values. Python side of include/kv_cache.h (layouts and arithmetic are stated there).

    cache = QuantKVCache.empty(num_pages, page_size, heads, head_dim, "int8")       # or "mxfp4"
    kv_cache_write(cache, k, v, slots)                # new tokens [T, heads, dim] into slots = page * page_size + offset
    k, v = kv_cache_read(cache, table, cu_seqlens, total)
"""
from __future__ import annotations

import torch

from .binding import _i64, _int, _lib, _vp
from .mxfp4 import call, different_devices

KV_CACHE_INT8, KV_CACHE_MXFP4 = 0, 1
KV_CACHE_MAX_DIM = 256
KV_CACHE_ZERO_REST = 0x100

_lib.kv_cache_write.argtypes = [_int, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp]
_lib.kv_cache_write.restype = _int
_lib.kv_cache_read.argtypes = [_int, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64,
                               _vp, _i64, _i64, _vp, _i64, _i64, _vp]
_lib.kv_cache_read.restype = _int


class QuantKVCache:
    """The four tensors of a cache, dense: codes [num_pages, page_size, heads, dim] int8 with scales fp32 [.., heads], or
    [.., dim / 2] uint8 with scales uint8 [.., heads, ceil(dim / 32)]. The value side may be left out (None)."""

    def __init__(self, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor | None = None, v_scales: torch.Tensor | None = None):
        self._tensors = (k_codes, k_scales, v_codes, v_scales)           # held for as long as the cache is, and not replaced
        self._look_over()

    def _look_over(self) -> None:
        """Checks the tensors and notes what the calls need of them."""
        k_codes, k_scales, v_codes, v_scales = self._tensors
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
            for what, t in (("codes", codes), ("scales", scales)):
                if t.untyped_storage().nbytes() < (t.storage_offset() + t.numel()) * t.element_size():
                    raise ValueError(f"{name}_{what}: the tensor's memory has been given back")
        self.device, self.device_index = k_codes.device, k_codes.get_device()
        if any(t is not None and t.get_device() != self.device_index for t in (k_scales, v_codes, v_scales)):
            raise different_devices("QuantKVCache")
        self._places = self._now()

    def _now(self) -> tuple:
        k_codes, k_scales, v_codes, v_scales = self._tensors
        return k_codes.data_ptr(), k_scales.data_ptr(), None if v_codes is None else v_codes.data_ptr(), None if v_scales is None else v_scales.data_ptr()

    def places(self) -> tuple:
        """The tensors' addresses now: a caller may have moved their storage (offloaded it, given a tensor other data)."""
        if self._now() != self._places:
            self._look_over()
        return self._places

    k_codes = property(lambda self: self._tensors[0])
    k_scales = property(lambda self: self._tensors[1])
    v_codes = property(lambda self: self._tensors[2])
    v_scales = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, num_pages: int, page_size: int, heads: int, dim: int, fmt: str = "int8", device="cuda", values: bool = True) -> "QuantKVCache":
        """A cache of zeros. dim: a multiple of 8 up to 256."""
        if fmt not in ("int8", "mxfp4"):
            raise ValueError(f"fmt: 'int8' or 'mxfp4' expected, got {fmt!r}")
        if dim <= 0 or dim % 8 or dim > KV_CACHE_MAX_DIM:
            raise ValueError(f"dim: a multiple of 8 up to {KV_CACHE_MAX_DIM} expected, got {dim}")
        lead = (num_pages, page_size, heads)

        def side():
            if fmt == "int8":
                return torch.zeros(lead + (dim,), dtype=torch.int8, device=device), torch.zeros(lead, dtype=torch.float32, device=device)
            return (torch.zeros(lead + (dim // 2,), dtype=torch.uint8, device=device),
                    torch.zeros(lead + ((dim + 31) // 32,), dtype=torch.uint8, device=device))

        return cls(*side(), *(side() if values else (None, None)))


def _vectors(cache: QuantKVCache, t: torch.Tensor, name: str, rows: int) -> tuple[int, int, int]:
    """Checks bf16 [rows, heads, dim] with contiguous heads on the cache's device; returns (pointer, token stride, head stride)."""
    if t.dtype is not torch.bfloat16 or t.dim() != 3:
        raise TypeError(f"{name}: bf16 [tokens, heads, dim] expected, got {t.dtype} {tuple(t.shape)}")
    if t.shape != (rows, cache.heads, cache.dim):
        raise ValueError(f"{name}: [{rows}, {cache.heads}, {cache.dim}] expected, got {tuple(t.shape)}")
    st, sh, one = t.stride()
    if one != 1:
        raise TypeError(f"{name}: heads must be contiguous")
    if t.get_device() != cache.device_index:
        raise different_devices(name)
    return t.data_ptr(), st if rows > 1 else 0, sh if cache.heads > 1 else 0


def kv_cache_write(cache: QuantKVCache, k: torch.Tensor, v: torch.Tensor | None, slots: torch.Tensor) -> None:
    """Quantizes k (and v) bf16 [T, heads, dim] into the cache at slots int64 [T]; slots outside the cache are skipped."""
    c = cache
    kc, ks, vc, vs = c.places()
    if slots.dtype is not torch.int64 or slots.dim() != 1 or not slots.is_contiguous():
        raise TypeError("slots: dense int64 [tokens] expected")
    tokens = slots.shape[0]
    kp, kt, kh = _vectors(c, k, "k", tokens)
    if (v is None) != (vc is None):
        raise ValueError("v goes with a cache that keeps values, and only with one")
    vp, vt, vh = (None, 0, 0) if v is None else _vectors(c, v, "v", tokens)
    if slots.get_device() != c.device_index:
        raise different_devices("kv_cache_write")
    if tokens == 0:
        return
    call(_lib.kv_cache_write, "kv_cache_write", c.device_index, c.fmt, kp, kt, kh, vp, vt, vh, slots.data_ptr(), tokens, c.heads, c.dim, kc, ks, vc, vs,
         c.num_pages * c.page_size)


def kv_cache_read(cache: QuantKVCache, table: torch.Tensor, cu_seqlens: torch.Tensor, total: int, starts: torch.Tensor | None = None,
                  k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None):
    """The sequences' tokens as bf16 [total, heads, dim], one sequence after another: (k, v), or (k, None) without values.
    table int32 [B, max_pages], cu_seqlens int32 [B + 1], starts int32 [B] (first token to read of each) or None. Rows that belong to
    no sequence (total may be more than cu_seqlens[-1]) are zeros, in k_out and v_out they are left as they are."""
    if table.dtype is not torch.int32 or table.dim() != 2:
        raise TypeError("table: int32 [sequences, max_pages] expected")
    seqs, max_pages = table.shape
    row, one = table.stride()
    if one != 1 and max_pages > 1:
        raise TypeError("table: rows must be contiguous")
    if cu_seqlens.dtype is not torch.int32 or cu_seqlens.shape != (seqs + 1,) or not cu_seqlens.is_contiguous():
        raise TypeError("cu_seqlens: dense int32 [sequences + 1] expected")
    if starts is not None and (starts.dtype is not torch.int32 or starts.shape != (seqs,) or not starts.is_contiguous()):
        raise TypeError("starts: dense int32 [sequences] expected")
    c = cache
    kc, ks, vc, vs = c.places()
    dev = c.device_index
    if v_out is not None and vc is None:
        raise ValueError("v_out goes with a cache that keeps values")
    dense = c.heads * c.dim
    # where both sides are allocated here the kernel writes the rows of no sequence too
    fill = k_out is None and (vc is None or v_out is None)
    new = torch.empty if fill else torch.zeros
    if k_out is None:
        k_out = new(total, c.heads, c.dim, dtype=torch.bfloat16, device=c.device)
        kp, kt, kh = k_out.data_ptr(), dense, c.dim
    else:
        kp, kt, kh = _vectors(c, k_out, "k_out", total)
    if vc is None:
        vp, vt, vh = None, 0, 0
    elif v_out is None:
        v_out = new(total, c.heads, c.dim, dtype=torch.bfloat16, device=c.device)
        vp, vt, vh = v_out.data_ptr(), dense, c.dim
    else:
        vp, vt, vh = _vectors(c, v_out, "v_out", total)
    if table.get_device() != dev or cu_seqlens.get_device() != dev or (starts is not None and starts.get_device() != dev):
        raise different_devices("kv_cache_read")
    if total == 0 or (seqs == 0 and not fill):
        return k_out, v_out
    call(_lib.kv_cache_read, "kv_cache_read", dev, c.fmt | (KV_CACHE_ZERO_REST if fill else 0), kc, ks, vc, vs, c.num_pages, c.page_size, c.heads, c.dim, table.data_ptr(),
         row if seqs > 1 else max_pages, max_pages, cu_seqlens.data_ptr(), None if starts is None else starts.data_ptr(), seqs, total, kp, kt, kh, vp, vt, vh)
    return k_out, v_out
