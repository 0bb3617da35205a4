"""Quantized paged cache of keys and values. Python side of include/kv_cache.h (layouts and arithmetic are stated there).

    cache = QuantKVCache.empty(num_pages, page_size, heads, head_dim, "int8")       # or "mxfp4"
    kv_cache_write(cache, k, v, slots)                # new tokens [T, heads, dim] into slots = page * page_size + offset
    k, v = kv_cache_read(cache, table, cu_seqlens, total)

A decoder's step appends its tokens rotated by position, and attends to them on the codes:

    q = kv_cache_append(cache, k, v, slots, positions, cos_sin, q=q)
    out = kv_cache_attention(cache, q, table, lens, cu_q, workspace=workspace)
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _i64, _int, _lib, _sz, _vp
from .mxfp4 import call, different_devices

KV_CACHE_INT8, KV_CACHE_MXFP4 = 0, 1
KV_CACHE_MAX_DIM = 256
KV_CACHE_MAX_AXES = 8
KV_CACHE_ZERO_REST = 0x100

_lib.kv_cache_write.argtypes = [_int, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp]
_lib.kv_cache_write.restype = _int
_lib.kv_cache_read.argtypes = [_int, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64,
                               _vp, _i64, _i64, _vp, _i64, _i64, _vp]
_lib.kv_cache_read.restype = _int

_lib.kv_cache_append.argtypes = [_int, _vp, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _int, _vp, _i64, _i64, _vp,
                                 _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _i64, _vp]
_lib.kv_cache_append.restype = _int
_lib.kv_cache_rope_table.argtypes = [_vp, _i64, _i64, _i64, ctypes.c_double, _vp, _vp]
_lib.kv_cache_rope_table.restype = _int
_lib.kv_cache_attention_workspace_bytes.argtypes = [_i64] * 5
_lib.kv_cache_attention_workspace_bytes.restype = _sz
_lib.kv_cache_attention_zeroed_bytes.argtypes = [_i64] * 5
_lib.kv_cache_attention_zeroed_bytes.restype = _sz
_lib.kv_cache_attention.argtypes = [_int, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _i64, _i64, _i64,
                                    _vp, _i64, ctypes.c_float, _vp, _i64, _i64, _vp, _vp, _sz, _vp]
_lib.kv_cache_attention.restype = _int


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


def _vectors(cache: QuantKVCache, t: torch.Tensor, name: str, rows: int, heads: int | None = None) -> tuple[int, int, int]:
    """Checks bf16 [rows, heads, dim] (the cache's heads by default) with contiguous heads on the cache's device; returns (pointer, token stride,
    head stride)."""
    heads = cache.heads if heads is None else heads
    if t.dtype is not torch.bfloat16 or t.dim() != 3:
        raise TypeError(f"{name}: bf16 [tokens, heads, dim] expected, got {t.dtype} {tuple(t.shape)}")
    if t.shape != (rows, heads, cache.dim):
        raise ValueError(f"{name}: [{rows}, {heads}, {cache.dim}] expected, got {tuple(t.shape)}")
    st, sh, one = t.stride()
    if one != 1:
        raise TypeError(f"{name}: heads must be contiguous")
    if t.get_device() != cache.device_index:
        raise different_devices(name)
    return t.data_ptr(), st if rows > 1 else 0, sh if heads > 1 else 0


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


def kv_cache_rope_table(inv_freq: torch.Tensor, num_positions: int, first: int = 0, scale: float = 1.0) -> torch.Tensor:
    """The table that kv_cache_append reads, fp32 [num_positions, 2 * pairs]: cosines of (first + p) * inv_freq, then their sines, times scale.
    inv_freq: fp64 [pairs] on the CUDA device."""
    if inv_freq.dtype is not torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise TypeError("inv_freq: dense fp64 [pairs] expected")
    pairs = inv_freq.shape[0]
    table = torch.empty(num_positions, 2 * pairs, dtype=torch.float32, device=inv_freq.device)
    call(_lib.kv_cache_rope_table, "kv_cache_rope_table", inv_freq.get_device(), inv_freq.data_ptr(), pairs, first, num_positions, scale, table.data_ptr())
    return table


def kv_cache_append(cache: QuantKVCache, k: torch.Tensor, v: torch.Tensor | None, slots: torch.Tensor, positions: torch.Tensor | None = None,
                    cos_sin: torch.Tensor | None = None, axes: torch.Tensor | None = None, interleaved: bool = False, q: torch.Tensor | None = None,
                    q_out: torch.Tensor | None = None) -> torch.Tensor | None:
    """kv_cache_write of k rotated by the tokens' positions (and v as it is); returns q bf16 [T, q_heads, dim], rotated too (in q_out, which may be q).
    positions int64 [T], or [axes, T] with axes uint8 [rot / 2] telling each pair's axis; cos_sin fp32 [positions, rot] (kv_cache_rope_table); without
    a table nothing is rotated. Pairs are (2i, 2i + 1) if interleaved, else (i, i + rot / 2). For inference: autograd does not see the call."""
    c = cache
    kc, ks, vc, vs = c.places()
    dev = c.device_index
    if slots.dtype is not torch.int64 or slots.dim() != 1 or not slots.is_contiguous():
        raise TypeError("slots: dense int64 [tokens] expected")
    tokens = slots.shape[0]
    kp, kt, kh = _vectors(c, k, "k", tokens)
    if (v is None) != (vc is None):
        raise ValueError("v goes with a cache that keeps values, and only with one")
    vp, vt, vh = (None, 0, 0) if v is None else _vectors(c, v, "v", tokens)
    if slots.get_device() != dev:
        raise different_devices("kv_cache_append")
    if q is None:
        if q_out is not None:
            raise ValueError("q_out goes with q")
        qp, qt, qh, heads, op, ot, oh = None, 0, 0, 0, None, 0, 0
    else:
        if q.dim() != 3 or q.shape[1] == 0:
            raise TypeError(f"q: bf16 [tokens, heads, dim] expected, got {q.dtype} {tuple(q.shape)}")
        heads = q.shape[1]
        qp, qt, qh = _vectors(c, q, "q", tokens, heads)
        if q_out is None:
            q_out = torch.empty(tokens, heads, c.dim, dtype=torch.bfloat16, device=c.device)
        op, ot, oh = _vectors(c, q_out, "q_out", tokens, heads)
    if cos_sin is None:
        tp, rows, rot, pp, stride, count, ap = None, 0, 0, None, 0, 0, None
    else:
        if cos_sin.dtype is not torch.float32 or cos_sin.dim() != 2 or not cos_sin.is_contiguous():
            raise TypeError("cos_sin: dense fp32 [positions, rot] expected")
        rows, rot = cos_sin.shape
        if positions is None or positions.dtype is not torch.int64 or positions.dim() not in (1, 2) or not positions.is_contiguous():
            raise TypeError("positions: dense int64 [tokens] or [axes, tokens] expected")
        if positions.shape[-1] != tokens:
            raise ValueError(f"positions: {tokens} tokens expected, got {positions.shape[-1]}")
        count = 1 if positions.dim() == 1 else positions.shape[0]
        if axes is None:
            if count != 1:
                raise ValueError("axes: positions on several axes need the axis of each pair")
            ap = None
        else:
            if axes.dtype is not torch.uint8 or axes.shape != (rot // 2,) or not axes.is_contiguous():
                raise TypeError(f"axes: dense uint8 [{rot // 2}] expected")
            if axes.get_device() != dev:
                raise different_devices("kv_cache_append")
            ap = axes.data_ptr()
        if cos_sin.get_device() != dev or positions.get_device() != dev:
            raise different_devices("kv_cache_append")
        tp, pp, stride = cos_sin.data_ptr(), positions.data_ptr(), tokens
    if tokens > 0:
        call(_lib.kv_cache_append, "kv_cache_append", dev, c.fmt, qp, qt, qh, heads, op, ot, oh, kp, kt, kh, vp, vt, vh, tp, rows, rot, 1 if interleaved else 0, pp, stride,
             count, ap, slots.data_ptr(), tokens, c.heads, c.dim, kc, ks, vc, vs, c.num_pages * c.page_size)
    return q_out


def _overlap(tokens: int, heads: int, dim: int, st: int, sh: int, to: int, to_st: int, to_sh: int) -> bool:
    """Whether two sets of [tokens, heads, dim] elements share any, the second beginning `to` elements behind the first. Exact where strides are equal (slices of
    one buffer); where they are not, sets that reach into one another count as sharing."""
    ends, to_ends = (tokens - 1) * st + (heads - 1) * sh + dim, (tokens - 1) * to_st + (heads - 1) * to_sh + dim
    if to >= ends or -to >= to_ends:
        return False
    if (st, sh) != (to_st, to_sh):
        return True
    each = (heads - 1) * sh + dim
    if st and each <= to % st <= st - each:                      # tokens' heads lie side by side
        return False
    for h in range(1 - heads, heads):
        at = to + h * sh
        for more in (0, 1):
            t = min(max(-at // st + more, 1 - tokens), tokens - 1) if st else 0
            if abs(at + t * st) < dim:
                return True
    return False


def kv_cache_attention_workspace(cache: QuantKVCache, seqs: int, total_q: int, q_heads: int) -> torch.Tensor:
    """Scratch for kv_cache_attention with up to this many sequences, rows and heads of queries: made once, zero where it has to be. The calls leave it
    ready for the next one; two that may overlap on the device need one each."""
    size = int(_lib.kv_cache_attention_workspace_bytes(seqs, total_q, q_heads, cache.heads, cache.dim))
    if size == 0:
        raise ValueError(f"kv_cache_attention_workspace: {seqs} sequences, {total_q} rows and {q_heads} heads of queries do not go with {cache.heads} heads of {cache.dim}")
    workspace = torch.empty(size, dtype=torch.uint8, device=cache.device)
    workspace[:int(_lib.kv_cache_attention_zeroed_bytes(seqs, total_q, q_heads, cache.heads, cache.dim))].zero_()
    return workspace


def kv_cache_attention(cache: QuantKVCache, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, cu_q: torch.Tensor, scale: float | None = None,
                       tree: torch.Tensor | None = None, starts: torch.Tensor | None = None, out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of q bf16 [total, q_heads, dim] over the cache, bf16 [total, q_heads, dim]. Rows cu_q[b] to cu_q[b + 1] (int32 [B + 1]) are the newest tokens of
    sequence b, which are in the cache already and counted in lens (int32 [B]); table int32 [B, max_pages]. Each sees what comes before them
    and, of the new ones, those up to itself, or those whose bits are set in its row of tree int64 [total, words]; nothing ahead of starts int32 [B], new tokens included. scale:
    dim ** -0.5 by default. lse fp32 [total, q_heads] receives the logarithms of the softmax's sums. Rows of no sequence are zeros, in an out that is given
    they are left as they are. For inference: autograd does not see the call, and results carry no gradients."""
    c = cache
    if table.dtype is not torch.int32 or table.dim() != 2:
        raise TypeError("table: int32 [sequences, max_pages] expected")
    seqs, max_pages = table.shape
    row, one = table.stride()
    if one != 1 and max_pages > 1:
        raise TypeError("table: rows must be contiguous")
    if lens.dtype is not torch.int32 or lens.shape != (seqs,) or not lens.is_contiguous():
        raise TypeError("lens: dense int32 [sequences] expected")
    if cu_q.dtype is not torch.int32 or cu_q.shape != (seqs + 1,) or not cu_q.is_contiguous():
        raise TypeError("cu_q: dense int32 [sequences + 1] expected")
    if starts is not None and (starts.dtype is not torch.int32 or starts.shape != (seqs,) or not starts.is_contiguous()):
        raise TypeError("starts: dense int32 [sequences] expected")
    kc, ks, vc, vs = c.places()
    dev = c.device_index
    if vc is None:
        raise ValueError("kv_cache_attention: the cache keeps no values")
    if q.dim() != 3 or q.shape[1] == 0 or q.shape[1] % c.heads:
        raise ValueError(f"q: bf16 [tokens, a multiple of {c.heads} heads, dim] expected, got {tuple(q.shape)}")
    total, heads = q.shape[0], q.shape[1]
    qp, qt, qh = _vectors(c, q, "q", total, heads)
    words = 0
    if tree is not None:
        if tree.dtype is not torch.int64 or tree.dim() != 2 or not tree.is_contiguous():
            raise TypeError("tree: dense int64 [tokens, words] expected")
        words = tree.shape[1]
        if tree.shape[0] != total or words == 0:
            raise ValueError(f"tree: [{total}, words] expected, got {list(tree.shape)}")
    fill = out is None
    if fill:
        out = torch.empty(total, heads, c.dim, dtype=torch.bfloat16, device=c.device)
    op, ot, oh = _vectors(c, out, "out", total, heads)
    if not fill and total > 0 and abs(op - qp) < 2 * total * (qt + ot + heads * (qh + oh + c.dim)) and _overlap(total, heads, c.dim, qt, qh, (op - qp) // 2, ot, oh):
        raise ValueError("out: must not overlap q (a row of queries is read by several CTAs, at different times)")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (total, heads) or not lse.is_contiguous()):
        raise TypeError(f"lse: dense fp32 [{total}, {heads}] expected")
    if workspace is None:
        workspace = kv_cache_attention_workspace(c, seqs, total, heads)
    elif not workspace.is_contiguous():
        raise TypeError("workspace: dense tensor expected")
    if (table.get_device() != dev or lens.get_device() != dev or cu_q.get_device() != dev or workspace.get_device() != dev or (starts is not None and starts.get_device() != dev) or
            (tree is not None and tree.get_device() != dev) or (lse is not None and lse.get_device() != dev)):
        raise different_devices("kv_cache_attention")
    if total > 0 and (seqs > 0 or fill):
        call(_lib.kv_cache_attention, "kv_cache_attention", dev, c.fmt | (KV_CACHE_ZERO_REST if fill else 0), kc, ks, vc, vs, c.num_pages, c.page_size, c.heads, c.dim,
             table.data_ptr(), row if seqs > 1 else max_pages, max_pages, lens.data_ptr(), None if starts is None else starts.data_ptr(), cu_q.data_ptr(), seqs, qp, qt, qh, heads,
             total, None if tree is None else tree.data_ptr(), words, c.dim ** -0.5 if scale is None else scale, op, ot, oh, None if lse is None else lse.data_ptr(),
             workspace.data_ptr(), workspace.nbytes)
    return out
