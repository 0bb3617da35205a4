"""Attention over the quantized cache: refusals without a GPU, results against a plain 64-bit form on one."""
import ctypes
import math
import os
import random
import subprocess

import pytest
import torch

import lowbit_reference as ref
import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import kv_cache

INVALID, ALIGNMENT, WORKSPACE = 1, 2, 4
P = ctypes.c_void_p
NAN, INF = float("nan"), float("inf")


def test_refusals():
    f = kv_cache._lib.kv_cache_attention
    names = ["fmt", "kc", "ks", "vc", "vs", "num_pages", "page", "heads", "dim", "table", "stride", "max_pages", "lens", "starts", "cu", "seqs", "q", "qt", "qh", "q_heads", "total",
             "tree", "words", "scale", "out", "ot", "oh", "lse", "ws", "bytes", "stream"]
    p, size = P(4096), kv_cache._lib.kv_cache_attention_workspace_bytes(2, 6, 8, 2, 64)
    ok = dict(zip(names, [0, p, p, p, p, 4, 16, 2, 64, p, 3, 3, p, p, p, 2, p, 512, 64, 8, 6, p, 1, 0.125, p, 512, 64, p, p, size, None]))

    def status(**change):
        return f(*{**ok, **change}.values())

    for name in ("kc", "ks", "vc", "vs", "table", "lens", "cu", "q", "out"):
        assert status(**{name: None}) == INVALID, name
    assert status(fmt=2) == INVALID and status(heads=0) == INVALID and status(dim=264) == INVALID and status(page=0) == INVALID and status(num_pages=-1) == INVALID
    assert status(num_pages=1 << 28) == INVALID                                       # slots past 32 bits
    assert status(max_pages=1 << 27, stride=1 << 27) == INVALID                       # tokens of a sequence past 32 bits
    assert status(stride=2) == INVALID and status(seqs=-1) == INVALID and status(total=-1) == INVALID and status(q_heads=7) == INVALID and status(q_heads=0) == INVALID
    assert status(words=0) == INVALID and status(scale=NAN) == INVALID and status(scale=INF) == INVALID
    assert status(dim=60) == ALIGNMENT
    for name in ("qt", "qh", "ot", "oh"):
        assert status(**{name: 516}) == ALIGNMENT, name
    for name in ("kc", "vc", "q", "out"):
        assert status(**{name: P(4104)}) == ALIGNMENT, name
    for name in ("ks", "vs", "table", "lens", "starts", "cu", "lse"):
        assert status(**{name: P(4098)}) == ALIGNMENT, name
    assert status(tree=P(4100)) == ALIGNMENT
    assert status(ws=None) == WORKSPACE and status(ws=P(4096 + 128)) == WORKSPACE and status(bytes=size - 1) == WORKSPACE
    assert status(starts=None, tree=None, words=0, lse=None) not in (INVALID, ALIGNMENT, WORKSPACE)
    assert status(total=0, q=None, out=None) not in (INVALID, ALIGNMENT, WORKSPACE)
    sizes = kv_cache._lib.kv_cache_attention_workspace_bytes
    assert sizes(2, 6, 7, 2, 64) == 0 and sizes(-1, 6, 8, 2, 64) == 0 and sizes(2, 6, 8, 2, 264) == 0
    assert 0 < kv_cache._lib.kv_cache_attention_zeroed_bytes(2, 6, 8, 2, 64) < size


def test_python_refusals():
    c = w8.QuantKVCache.empty(4, 4, 2, 16, "int8", device="cpu")
    q, table, lens, cu = torch.zeros(3, 4, 16, dtype=torch.bfloat16), torch.zeros(2, 2, dtype=torch.int32), torch.ones(2, dtype=torch.int32), torch.tensor([0, 1, 3], dtype=torch.int32)
    tree = torch.zeros(3, 1, dtype=torch.int64)
    call = w8.kv_cache_attention
    for bad in ((q.float(), table, lens, cu), (q, table.long(), lens, cu), (q, table, lens.long(), cu), (q, table, lens, cu[:2]), (q, table, lens[:1], cu)):
        with pytest.raises(TypeError):
            call(c, *bad)
    for heads in (3, 0):
        with pytest.raises(ValueError):
            call(c, q[:, :heads], table, lens, cu)
    for kw in ({"tree": tree.int()}, {"tree": tree[:, 0]}, {"starts": lens.long()}, {"lse": torch.zeros(3, 2)}):
        with pytest.raises(TypeError):
            call(c, q, table, lens, cu, **kw)
    for kw in ({"tree": tree[:2]}, {"out": q[:2]}, {"out": q}, {"tree": tree[:, :0]}):
        with pytest.raises(ValueError):
            call(c, q, table, lens, cu, **kw)
    with pytest.raises(ValueError):
        call(c, q, table, lens, cu)                              # no CPU fallback
    with pytest.raises(ValueError):
        call(w8.QuantKVCache.empty(4, 4, 2, 16, "int8", device="cpu", values=False), q, table, lens, cu)
    with pytest.raises(ValueError):
        w8.kv_cache_attention_workspace(c, 2, 3, 5)


# ------------------------------------------------------------------------------------------------ on the GPU

def values(codes, scales, fmt):
    if fmt == "int8":
        return codes.double() * scales.double()[..., None]
    return ref.mx_values(ref.unpack(codes), scales.long())


class Case:
    """A cache with sequences of these lengths in scattered pages, and queries for their last tokens."""

    def __init__(self, fmt, heads, group, dim, lens, news, page=16, seed=0, tree=False, spare_pages=2, q_scale=1.0):
        gen = self.gen = torch.Generator("cuda").manual_seed(seed)
        self.fmt, self.heads, self.group, self.dim, self.page, self.news, self.lengths = fmt, heads, group, dim, page, news, lens
        counts = [(n + page - 1) // page for n in lens]
        pages = sum(counts) + spare_pages
        lead = (pages, page, heads)
        sides = []
        for _ in range(2):
            if fmt == "int8":
                sides += [torch.randint(-127, 128, lead + (dim,), generator=gen, device="cuda").to(torch.int8), torch.rand(lead, generator=gen, device="cuda") * 0.02 + 0.005]
            else:
                sides += [torch.randint(0, 256, lead + (dim // 2,), generator=gen, device="cuda").to(torch.uint8),
                          torch.randint(120, 130, lead + ((dim + 31) // 32,), generator=gen, device="cuda").to(torch.uint8)]
        self.cache = w8.QuantKVCache(*sides)
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), max(counts + [1])), -1, dtype=torch.int32, device="cuda")
        for b, n in enumerate(counts):
            self.table[b, :n] = order[sum(counts[:b]):sum(counts[:b + 1])]
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.cu = torch.tensor([sum(news[:b]) for b in range(len(news) + 1)], dtype=torch.int32, device="cuda")
        self.total = sum(news)
        self.q = (torch.randn(self.total, heads * group, dim, generator=gen, device="cuda") * q_scale).to(torch.bfloat16)
        self.starts, self.tree = None, None
        if tree:
            words = (max(news) + 63) // 64
            self.tree = torch.randint(-(1 << 63), (1 << 63) - 1, (self.total, words), generator=gen, device="cuda")

    def sees(self, b):
        """[new tokens, tokens] of sequence b."""
        n, length = self.news[b], self.lengths[b]
        t = torch.arange(length, device="cuda")
        j = t[None] - (length - n)
        if self.tree is None:
            see = j <= torch.arange(n, device="cuda")[:, None]
        else:
            bits = self.tree[int(self.cu[b]):int(self.cu[b]) + n]
            word = bits[:, (j[0].clamp(min=0) // 64).clamp(max=bits.shape[1] - 1)]
            see = (j < 0) | (((word >> j.clamp(min=0) % 64) & 1) == 1) & (j < 64 * bits.shape[1])
        if self.starts is not None:
            see = see & (t >= self.starts[b])[None]
        page_ok = (self.table[b].long() >= 0) & (self.table[b] < self.cache.num_pages)
        at = t // self.page
        return see & torch.where(at < self.table.shape[1], page_ok[at.clamp(max=self.table.shape[1] - 1)], False)[None]

    def want(self, scale):
        """(outputs, error that the roundings may add up to, log of the sums), 64 bits."""
        outs, slacks, lses = [], [], []
        flat = [t.flatten(0, 1) for t in self.cache._tensors]
        for b, n in enumerate(self.news):
            if n == 0:
                continue
            see = self.sees(b)
            t = torch.arange(self.lengths[b], device="cuda")
            page = self.table[b].long()[(t // self.page).clamp(max=self.table.shape[1] - 1)].clamp(0, max(0, self.cache.num_pages - 1))
            slot = page * self.page + t % self.page
            k, v = values(flat[0][slot], flat[1][slot], self.fmt), values(flat[2][slot], flat[3][slot], self.fmt)
            q = self.q[int(self.cu[b]):int(self.cu[b]) + n].double().view(n, self.heads, self.group, self.dim)
            s = torch.einsum("nhgd,phd->nhgp", q, k) * scale
            # a token's unit: its scale (4 bits: the largest of its blocks'), in which its codes meet the matrix instructions
            units = []
            for scales in (flat[1][slot], flat[3][slot]):
                units.append(scales.double() if self.fmt == "int8" else ref.two_to(torch.where(scales == 255, 0, scales.long()).amax(-1) - 127))
            # the score's error: dim products added in fp32 (2^-23 each, truncating adders allowed for), three factors, and the exponential's argument;
            # 4 bits: a block 2^-27 below the unit counts as zero, and its largest element is 6
            off = (torch.einsum("nhgd,phd->nhgp", q.abs(), k.abs()) * abs(scale) * (self.dim + 8) * 2.0 ** -23)
            if self.fmt == "mxfp4":
                off = off + torch.einsum("nhgd,ph->nhgp", q.abs(), units[0]) * abs(scale) * 6 * 2.0 ** -27
                # many rows: the unit is the largest of 128 tokens, at 2^12 in fp16, where a block's factor of 2^-25, 2^-37 of it, counts as zero; an element is 6 at most
                if self.lengths[b]:
                    off = off + (q.abs().sum(-1) * units[0].amax(0)[None, :, None])[..., None] * abs(scale) * 6 * 2.0 ** -37
            hidden = ~see[:, None, None]
            s = s.masked_fill(hidden, -INF)
            top = s.amax(-1, keepdim=True)
            e = torch.where(hidden, 0.0, torch.exp(s - torch.where(top == -INF, 0.0, top)))
            total = e.sum(-1, keepdim=True)
            p = e / torch.where(total == 0, 1.0, total)
            dead = (total == 0) & ~torch.isnan(total)
            off = torch.where(hidden | torch.isnan(off), 0.0, off).amax(-1, keepdim=True)
            # values of tokens that a row does not see do not reach it, NaN or not
            o = torch.stack([torch.einsum("hgp,phd->hgd", p[i][..., see[i]], v[see[i]]) for i in range(n)])
            size = torch.stack([torch.einsum("hgp,phd->hgd", p[i][..., see[i]], v[see[i]].abs()) for i in range(n)])
            o = torch.where(dead, 0.0, o)
            # weights (probability, or probability times unit) are rounded to fp16 (2^-11), and so may be unit and unit times code (many rows); sums and exponentials are fp32 (the logarithm of the unit adds 2^-16 for the spacing of
            # numbers of a few hundred); numerator and denominator carry the score's error; the output is rounded to bf16
            slack = torch.where(dead, 0.0, size) * (3 * 2.0 ** -11 + 2 * off + 2.0 ** -15 + (self.lengths[b] / 16 + 64) * 2.0 ** -23) + o.abs() * 2.0 ** -8
            # fp32 has no exponentials below 2^-126: x = 2^(s - m) for a running maximum m of at least (the tokens' largest) - 16 and, where parts meet,
            # 2^(m - M), are zero there, so a token of less than 2^-126 * 2^16 of the largest may count as nothing: its p |v|.
            small = torch.where(e < 2.0 ** -110, p, 0.0)
            lost = torch.stack([torch.einsum("hgp,phd->hgd", small[i][..., see[i]], v[see[i]].abs()) for i in range(n)])
            # weights are fp16 numbers relative to a reference that puts the row's largest at 2^7 at least, with steps of 2^-24 at the bottom: half a step
            # a token, times its value in units
            unit = units[1]
            worth = torch.where(see[:, None, None], p * unit.transpose(0, 1)[None, :, None], 0.0).nan_to_num().amax(-1)
            steps = torch.stack([torch.einsum("phd->hd", (v / torch.where(unit == 0, 1.0, unit)[..., None]).abs()[see[i]]) for i in range(n)])[:, :, None]
            slack = slack + torch.where(dead, 0.0, lost + 2.0 ** -32 * worth[..., None] * steps)
            # many rows: the weight is the probability alone; values are fp16 relative to 2^15 = a code of 128 or 8 times twice the sequence's largest unit
            whole = torch.stack([torch.einsum("phd->hd", v.abs()[see[i]]) for i in range(n)])[:, :, None]
            largest = unit.nan_to_num().amax(0)[None, :, None, None] if self.lengths[b] else 0.0
            slack = slack + torch.where(dead, 0.0, 2.0 ** -32 * whole + 2.0 ** -32 * largest)
            if self.fmt == "mxfp4":                              # values, too, lose blocks 2^-27 below their unit
                bottom = torch.stack([torch.einsum("hgp,ph->hg", p[i][..., see[i]], unit[see[i]]) for i in range(n)])[..., None]
                slack = slack + torch.where(dead, 0.0, bottom * 6 * 2.0 ** -27)
            outs.append(o.reshape(n, -1, self.dim))
            slacks.append(slack.reshape(n, -1, self.dim))
            lse = torch.where(dead, -INF, torch.log(total) + torch.where(top == -INF, 0.0, top))
            lses.append(torch.cat([lse, off + 2.0 ** -20 + (self.lengths[b] / 16 + 64) * 2.0 ** -23 * (1 + torch.where(dead, 0.0, lse.abs()))], -1).reshape(n, -1, 2))
        return torch.cat(outs), torch.cat(slacks), torch.cat(lses)

    def check(self, scale=None, **kw):
        lse = torch.full((self.total, self.heads * self.group), 9.0, device="cuda")
        got = w8.kv_cache_attention(self.cache, self.q, self.table, self.lens, self.cu, scale, tree=self.tree, starts=self.starts, lse=lse, **kw)
        want, slack, want_lse = self.want(self.dim ** -0.5 if scale is None else scale)
        assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN where it should not be, or not where it should"
        worst = ((got.double() - want).abs() - slack).nan_to_num(nan=-1.0).max().item() if got.numel() else -1
        assert worst <= 0, worst
        fine = torch.isfinite(want_lse[..., 0])
        assert torch.equal(torch.isnan(lse), torch.isnan(want_lse[..., 0])) and torch.equal(lse == -INF, want_lse[..., 0] == -INF)
        assert bool(((lse.double() - want_lse[..., 0]).abs() <= want_lse[..., 1])[fine].all())
        return got


SHAPES = [(1, 1, 64), (2, 4, 128), (3, 5, 72), (8, 8, 128), (2, 1, 256), (1, 16, 80), (2, 3, 8), (5, 2, 96), (1, 40, 64), (2, 7, 136), (3, 2, 40), (2, 2, 208), (1, 3, 224), (2, 1, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("heads,group,dim", SHAPES)
def test_one_token(fmt, heads, group, dim):
    for lens in ([1], [16], [17], [63, 64, 65, 1, 300], [1000, 5]):
        Case(fmt, heads, group, dim, lens, [1] * len(lens), seed=len(lens)).check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("heads,group,dim", SHAPES)
@pytest.mark.parametrize("tree", [False, True])
def test_several_tokens(fmt, heads, group, dim, tree):
    """Chains and trees of any bits (rows that see no new token, nor themselves), new tokens that are all a sequence has among them."""
    Case(fmt, heads, group, dim, [200, 9, 64, 33], [5, 9, 1, 17], page=20, tree=tree, seed=1).check()
    Case(fmt, heads, group, dim, [150, 333], [64, 70], page=7, tree=tree, seed=2).check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 64), (2, 4, 128), (3, 5, 72), (2, 8, 96), (1, 40, 64), (2, 3, 8), (1, 8, 104)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("news", [(20, 31, 64), (65, 3, 100), (1, 2, 130)])
def test_many_rows(fmt, heads, group, dim, tree, news):
    """From a few dozen to some hundred rows of queries a sequence and head, lengths around whole tiles of tokens."""
    Case(fmt, heads, group, dim, [n + more for n, more in zip(news, (0, 128, 700))], list(news), page=16, tree=tree, seed=3).check()
    Case(fmt, heads, group, dim, [n + more for n, more in zip(news, (127, 257, 1))], list(news), page=25, tree=tree, seed=4).check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_rows_that_see_nothing(fmt):
    c = Case(fmt, 2, 4, 128, [3, 40, 70], [3, 2, 6], tree=True)
    c.tree[0], c.tree[2] = 0, 0
    c.tree[1] = 4
    got = c.check()
    assert not got[0].any() and not got[2].any() and got[1].any()
    # windows that leave nothing before the tree, or nothing at all
    c.starts = torch.tensor([0, 39, 70], dtype=torch.int32, device="cuda")
    got = c.check()
    assert not got[5:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("page", [1, 2, 3, 4, 8, 16, 64, 100])
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_pages_windows_and_empty_sequences(fmt, page, dim):
    c = Case(fmt, 2, 5, dim, [0, 130, 0, 57, 257, 1, 0], [0, 1, 0, 3, 0, 1, 0], page=page, seed=page)
    c.check()
    c.starts = torch.tensor([0, 100, 0, 13, 0, 0, 0], dtype=torch.int32, device="cuda")
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("page", [1, 2, 3, 4, 8, 16, 32, 64, 100, 192])
@pytest.mark.parametrize("heads,group,dim", [(2, 5, 128), (1, 9, 64), (2, 12, 80)])
def test_pages_and_windows_of_many_rows(fmt, page, heads, group, dim):
    """Rows beyond a few, and beyond one tile of rows, with pages of all sizes; windows that begin anywhere, empty sequences among them."""
    c = Case(fmt, heads, group, dim, [330, 0, 64, 9, 515], [29, 0, 7, 9, 40], page=page, seed=page, tree=page % 3 == 0)
    c.check()
    c.starts = torch.tensor([31, 0, 63, 9, 190], dtype=torch.int32, device="cuda")
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group,new", [(4, 2), (2, 8), (4, 8), (3, 11), (4, 32), (4, 33), (8, 61), (1, 300)])
@pytest.mark.parametrize("dim", [64, 128])
def test_either_side_of_the_choices(fmt, group, new, dim):
    """Rows around those at which another kernel, or another form of it, is chosen."""
    Case(fmt, 2, group, dim, [new + 200, new, new + 1000], [new] * 3, page=64, seed=new, tree=True).check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("heads,group,new", [(2, 4, 1), (2, 8, 9), (1, 8, 40)])
def test_one_workspace_for_all_sizes(fmt, heads, group, new):
    """Calls of few and of many sequences and rows take turns on a workspace made for the largest; parts of sequences that CTAs share lie in it."""
    many = Case(fmt, heads, group, 128, [700 + 40 * i for i in range(60)], [new] * 60, page=16, seed=40)
    few = Case(fmt, heads, group, 128, [9000, 5000], [1, new], page=16, seed=41)
    ws = w8.kv_cache_attention_workspace(many.cache, 60, many.total, heads * group)
    for c in (many, few, many, few, few, many):
        c.check(workspace=ws)
    zeroed = kv_cache._lib.kv_cache_attention_zeroed_bytes(60, many.total, heads * group, heads, 128)
    assert not bool(ws[:zeroed].any()) and w8.int8_check_status(ws) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group,new", [(4, 1), (4, 4), (4, 20), (8, 40)])
def test_wait_runs_out_and_the_kernel_returns(fmt, group, new):
    c = Case(fmt, 2, group, 128, [900, 300], [new, new], page=64, seed=30)
    ws = w8.kv_cache_attention_workspace(c.cache, 2, 2 * new, 2 * group)
    run = lambda: w8.kv_cache_attention(c.cache, c.q, c.table, c.lens, c.cu, workspace=ws)
    want = run()
    assert w8.int8_check_status(ws) == 0
    try:
        w8.debug_set_wait_limit_ns(3_000_000)
        w8.debug_set_starve(1)
        run()
        assert w8.int8_check_status(ws) == 7 and w8.int8_sticky_status() == 7
    finally:
        w8.debug_set_starve(0)
        w8.debug_set_wait_limit_ns(0)
        w8.int8_sticky_status(clear=True)
    again = run()
    assert w8.int8_check_status(ws) == 0 and torch.equal(again, want)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_pages_outside_the_cache(fmt):
    """Such tokens are not seen (and nothing is read for them): unset pages, ids past the cache, tokens past the table."""
    c = Case(fmt, 2, 2, 64, [160, 90], [2, 2])
    c.table[0, 3], c.table[0, 5], c.table[1, 0] = -1, 1 << 30, c.cache.num_pages
    c.check()
    c.table = c.table[:, :4].contiguous()
    c.check()
    c.table = torch.full_like(c.table, -1)
    assert not c.check().any()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group", [4, 16, 40])
def test_nan_reaches_those_who_see_it(fmt, group):
    """NaN scales behind the end of a sequence, in other branches of a tree and outside a window reach nobody; those that are seen do, a block of
    a value its own elements only."""
    c = Case(fmt, 2, group, 128, [83, 64], [6, 3], tree=True, seed=5)
    bad = NAN if fmt == "int8" else 255

    def slot(b, t):
        return int(c.table[b, t // 16]), t % 16

    for t in (83, 84, 95):                                       # behind the end, in the last page
        page, at = slot(0, t)
        for scales in (c.cache.k_scales, c.cache.v_scales):
            scales[page, at] = bad
    c.check()
    assert not bool(torch.isnan(c.check()).any())
    c.tree[:] = torch.tensor([1, 3, 5, 9, 17, 33, 1, 3, 7], device="cuda")[:, None]
    page, at = slot(0, 83 - 6 + 2)                               # node 2: seen by itself alone
    c.cache.v_scales[page, at] = bad
    page, at = slot(0, 83 - 6 + 4)
    c.cache.k_scales[page, at, 1] = bad
    if fmt == "mxfp4":                                           # one block of a value, and a token that everybody sees
        page, at = slot(0, 83 - 6 + 5)
        c.cache.v_scales[page, at, 0, 2] = bad
        page, at = slot(1, 20)
        c.cache.v_scales[page, at, 1, 3] = bad
        for t in (83 - 6 + 2, 83 - 6 + 5, ):
            page, at = slot(0, t)
            c.cache.v_codes[page, at] = 0
    got = c.check()
    assert bool(torch.isnan(got[2]).all()) and bool(torch.isnan(got[4, group:]).all())
    assert not bool(torch.isnan(got[[0, 1, 3]]).any()) and not bool(torch.isnan(got[4, :group]).any())
    if fmt == "mxfp4":
        assert bool(torch.isnan(got[5, :group, 64:96]).all()) and bool(torch.isnan(got[6:, group:, 96:]).all()) and not bool(torch.isnan(got[6:, :group]).any())
    c.starts = torch.tensor([0, 21], dtype=torch.int32, device="cuda")
    got = c.check()
    assert not bool(torch.isnan(got[6:]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group", [4, 32, 130])
def test_scales_far_apart(fmt, group):
    """Keys and values of very different sizes, from token to token and (4 bits) block to block; the softmax is nearly one token in one case, nearly flat in
    the other; tokens whose values are zero keep their weight."""
    c = Case(fmt, 2, group, 128, [500, 77], [3, 1], tree=False, seed=6)
    if fmt == "int8":
        c.cache.v_scales.mul_(torch.exp2(torch.randint(-90, 90, c.cache.v_scales.shape, generator=c.gen, device="cuda").float()))
        c.cache.v_codes[::3] = 0
    else:
        c.cache.v_scales.copy_(torch.randint(0, 250, c.cache.v_scales.shape, generator=c.gen, device="cuda"))
        c.cache.v_codes[::3] = 0
        c.cache.v_scales[::3] = 0
        c.cache.k_scales.copy_(torch.randint(90, 130, c.cache.k_scales.shape, generator=c.gen, device="cuda"))
    c.check()
    c.check(scale=1e-3)
    c.q *= 2.0 ** 10
    c.check()
    c.q *= 2.0 ** -60
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group", [8, 16, 40])
def test_queries_of_any_size(fmt, group):
    c = Case(fmt, 1, group, 128, [90], [4], seed=8)
    c.q *= torch.exp2(torch.randint(-100, 3, c.q.shape[:2], generator=c.gen, device="cuda"))[..., None].to(torch.bfloat16)
    c.q[0, 0] = 0
    c.q[1, 3, 7] = NAN
    got = c.check()
    assert bool(torch.isnan(got[1, 3]).all()) and int(torch.isnan(got).any(-1).sum()) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_strides_rows_of_no_sequence_and_repeats(fmt):
    c = Case(fmt, 2, 3, 72, [120, 64, 99], [2, 4, 1], seed=3)
    want = c.check()
    wide = torch.full((c.total + 5, 9, 80), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[2:2 + c.total, 1:7, 8:] = c.q
    out = torch.full((c.total + 5, 8, 96), 5.0, dtype=torch.bfloat16, device="cuda")
    cu = c.cu + 2
    ws = w8.kv_cache_attention_workspace(c.cache, 3, c.total + 5, 6)
    zeroed = kv_cache._lib.kv_cache_attention_zeroed_bytes(3, c.total + 5, 6, 2, 72)
    for _ in range(3):
        got = w8.kv_cache_attention(c.cache, wide[:, 1:7, 8:], c.table, c.lens, cu, out=out[:, 1:7, 8:80], workspace=ws)
        assert torch.equal(got[2:2 + c.total], want) and bool((got[:2] == 5).all()) and bool((got[2 + c.total:] == 5).all())
        assert bool((out[:, 0] == 5).all()) and bool((out[:, 7] == 5).all()) and bool((out[:, :, :8] == 5).all()) and bool((out[:, :, 80:] == 5).all())
        assert not ws[:zeroed].any()
    # an output that the call allocates: zeros there
    lse = torch.zeros(c.total + 5, 6, device="cuda")
    got = w8.kv_cache_attention(c.cache, wide[:, 1:7, 8:], c.table, c.lens, cu, lse=lse)
    assert torch.equal(got[2:2 + c.total], want) and not got[:2].any() and not got[2 + c.total:].any() and bool((lse[:2] == -INF).all()) and bool((lse[2 + c.total:] == -INF).all())
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert not w8.kv_cache_attention(c.cache, c.q, c.table[:0], none, torch.zeros(1, dtype=torch.int32, device="cuda")).any()
    assert w8.kv_cache_attention(c.cache, c.q[:0], c.table, c.lens, torch.zeros(4, dtype=torch.int32, device="cuda")).shape == (0, 6, 72)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_many_sequences(fmt):
    """More sequences than a CTA has threads, and more work than the grid takes in one go; lengths and new tokens of all sizes."""
    lens = [(i * 37) % 150 for i in range(301)]
    Case(fmt, 3, 2, 64, lens, [min(n, i % 4) for i, n in enumerate(lens)], seed=11).check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_long_sequences(fmt):
    Case(fmt, 2, 4, 128, [40000, 3], [1, 1], page=64, seed=12).check()
    Case(fmt, 1, 8, 128, [30001], [30], page=16, tree=True, seed=13).check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_a_prompt_as_a_chain(fmt):
    Case(fmt, 2, 2, 64, [700, 321], [700, 300], page=32, seed=14).check()


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A cache of more than 4 GB a side, read at its far end."""
    page, heads, dim = 64, 8, 256
    pages = (5 << 30) // (page * heads * dim)
    small = Case("int8", heads, 2, dim, [200, 77], [1, 3], page=page, seed=15)
    sides = [torch.empty(pages, *t.shape[1:], dtype=t.dtype, device="cuda") for t in small.cache._tensors]
    for big, t in zip(sides, small.cache._tensors):
        big[-t.shape[0]:] = t
    want = small.check()
    table = torch.where(small.table >= 0, small.table + (pages - small.cache.num_pages), small.table)
    assert torch.equal(w8.kv_cache_attention(w8.QuantKVCache(*sides), small.q, table, small.lens, small.cu), want)


@pytest.mark.gpu
def test_graphs_and_streams():
    """Two captured graphs that share a workspace, replayed in turn; a call on another stream with a workspace of its own."""
    cases = [Case("int8", 2, 4, 128, [900, 300], [1, 1], seed=16), Case("mxfp4", 2, 4, 128, [500, 200], [7, 3], tree=True, seed=17)]
    ws = w8.kv_cache_attention_workspace(cases[0].cache, 2, 10, 8)
    want = [c.check() for c in cases]
    outs, graphs = [torch.zeros_like(w) for w in want], []
    torch.cuda.synchronize()
    for c, out in zip(cases, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            w8.kv_cache_attention(c.cache, c.q, c.table, c.lens, c.cu, tree=c.tree, out=out, workspace=ws)
        graphs.append(graph)
    for _ in range(3):
        for out in outs:
            out.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    side = torch.cuda.Stream()
    mine, its = (w8.kv_cache_attention_workspace(c.cache, 2, 10, 8) for c in cases)
    torch.cuda.synchronize()
    for _ in range(20):
        a = w8.kv_cache_attention(cases[0].cache, cases[0].q, cases[0].table, cases[0].lens, cases[0].cu, workspace=mine)
        with torch.cuda.stream(side):
            b = w8.kv_cache_attention(cases[1].cache, cases[1].q, cases[1].table, cases[1].lens, cases[1].cu, tree=cases[1].tree, workspace=its)
    torch.cuda.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_norm_append_attend(fmt):
    """The operators in a row, as a decoder's step: norm, int8 projection, append, attention; against 64 bits from the codes that each step left."""
    gen = torch.Generator("cuda").manual_seed(20)
    width, heads, group, dim, page = 256, 2, 2, 64, 16
    x = torch.randn(5, width, generator=gen, device="cuda").to(torch.bfloat16)
    qw, s_ch = w8.int8_quantize_weight_per_channel(torch.randn((group + 2) * heads * dim, width, generator=gen, device="cuda") * width ** -0.5)
    c = Case(fmt, heads, group, dim, [53, 30], [3, 2], page=page, seed=21, tree=True)
    table = w8.kv_cache_rope_table(torch.tensor([10000.0 ** (-i / 32) for i in range(32)], dtype=torch.float64, device="cuda"), 64)
    qa, s_tok, h = w8.int8_rmsnorm(x, torch.ones(width, device="cuda"), residual=x)
    qkv = w8.int8_linear_fused(qa, qw, s_ch, None, s_tok=s_tok).view(5, -1, dim)
    where = torch.tensor([50, 51, 52, 28, 29], device="cuda")
    slots = c.table[torch.tensor([0, 0, 0, 1, 1], device="cuda"), where // page].long() * page + where % page
    c.q = w8.kv_cache_append(c.cache, qkv[:, 4:6], qkv[:, 6:], slots, where, table, q=qkv[:, :4])
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group,new", [(4, 1), (16, 2), (40, 3), (8, 30)])
@pytest.mark.parametrize("power", [12, 16, 20, 22, 24, 25, 26, 27, 28, 29, 30, 32, 40, 100])
def test_scores_of_any_size(fmt, group, new, power):
    """Large queries: a row is its largest token's value, however far the spacing of numbers of its scores' size is above the logarithm of a scale."""
    c = Case(fmt, 2, group, 128, [300, 5000, new + 40], [new] * 3, seed=52)
    if fmt == "int8":
        c.cache.v_scales.mul_(2.0 ** -9)
    c.q *= 2.0 ** power
    got = c.check().double().view(c.total, 2, group, 128)
    flat, rows = [t.flatten(0, 1) for t in c.cache._tensors], 0
    for b in range(3):
        see, t = c.sees(b), torch.arange(c.lengths[b], device="cuda")
        slot = c.table[b].long()[t // c.page] * c.page + t % c.page
        k, v = values(flat[0][slot], flat[1][slot], fmt), values(flat[2][slot], flat[3][slot], fmt)
        q = c.q[new * b:new * (b + 1)].double().view(new, 2, group, 128)
        s = (torch.einsum("nhgd,phd->nhgp", q, k) * 128 ** -0.5).masked_fill(~see[:, None, None], -INF)
        # error of a score: as in Case.want; all others together then weigh less than 5000 * 2^-60 of the largest
        off = (torch.einsum("nhgd,phd->nhgp", q.abs(), k.abs()) * 128 ** -0.5 * (128 + 8) * 2.0 ** -23).amax(-1) + q.abs().amax(-1) * k.abs().amax() * 128 * 2.0 ** -27
        first, second = s.topk(2, -1).values.unbind(-1)
        alone = first - second > 2 * off + 42
        want = v[s.argmax(-1), torch.arange(2, device="cuda")[None, :, None]]
        # weight, unit and unit times code rounded to fp16, the output to bf16
        wrong = (got[new * b:new * (b + 1)] - want).abs() > want.abs() * (2.0 ** -8 + 3 * 2.0 ** -11) + 2.0 ** -32 * v.abs().amax()
        assert not bool((wrong.any(-1) & alone).any())
        rows += int(alone.sum())
    assert rows > c.total * group


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group,new", [(4, 1), (16, 2), (40, 3), (8, 30)])
def test_keys_of_any_size(fmt, group, new):
    """Large keys, with ordinary queries (whose scores fp32 holds) and with small ones."""
    for power in (60, 90, 105):
        c = Case(fmt, 2, group, 128, [300, new + 40], [new] * 2, seed=53)
        if fmt == "int8":
            c.cache.k_scales.mul_(2.0 ** power)
        else:
            c.cache.k_scales.add_(power)
        assert bool(torch.isfinite(c.check()).all())
        c.q *= 2.0 ** -power
        c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group,new", [(4, 4), (40, 3), (8, 30)])
@pytest.mark.parametrize("power", [12, 40, 100])
@pytest.mark.parametrize("dim", [64, 72, 128])
def test_a_large_query_leaves_the_others_alone(fmt, group, new, power, dim):
    """A node, and a head of another, that are far larger than the rest; rows of few and of many to a tile."""
    c = Case(fmt, 2, group, dim, [300, new + 40], [new, new], seed=50)
    c.q[1] *= 2.0 ** power
    c.q[new + 2, 3] *= 2.0 ** power
    c.check()
    c.check(scale=-0.05)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("group,new", [(4, 4), (40, 3), (8, 30)])
@pytest.mark.parametrize("power", [7, 8, 9, 30])
@pytest.mark.parametrize("dim", [64, 128])
def test_small_queries_beside_ordinary_ones(fmt, group, new, power, dim):
    """Large keys: the small queries have scores of ordinary size, the others see one token each."""
    c = Case(fmt, 2, group, dim, [300, new + 40], [new, new], seed=51)
    if fmt == "int8":
        c.cache.k_scales.mul_(2.0 ** power)
    else:
        c.cache.k_scales.add_(power)
    c.q[::2] *= 2.0 ** -power
    c.q[:, 1::3] *= 2.0 ** -power
    c.check()


def test_scales_are_fetched_within_their_buffer(tmp_path):
    """MXFP4 scales come as 4-byte words: up to a head's last byte, and from no byte before the buffer, whatever the caches' sizes."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_14598_b200", "csrc")
    source = tmp_path / "words.cpp"
    source.write_text('''
        #include "scale_words.h"
        int main() {
            for (int blocks = 1; blocks <= 8; ++blocks)
                for (int64_t entries = 1; entries <= 70; ++entries)
                    for (int64_t entry = 0; entry < entries; ++entry) {
                        const w8a8::ScaleWords w = w8a8::scale_words(entry, blocks);
                        int64_t end = w.from;
                        for (int i = 0; i < (blocks <= 4 ? 2 : 3); ++i) {
                            if (w.bytes(i) < 0 || w.bytes(i) > 4 || (w.bytes(i) > 0 && w.from + 4 * i != end)) return 1;     // without gaps
                            end += w.bytes(i);
                        }
                        if (w.from < 0 || w.from % 4 || w.from + w.shift != entry * blocks || end != (entry + 1) * blocks || end > entries * blocks) return 2;
                    }
            return 0;
        }''')
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", csrc, str(source), "-o", str(tmp_path / "words")], check=True)
    assert subprocess.run([str(tmp_path / "words")]).returncode == 0


def test_outputs_over_queries_are_refused():
    """Views of one buffer that share elements, wherever they begin; those that share none are fine."""
    c = w8.QuantKVCache.empty(4, 4, 2, 16, "int8", device="cpu")
    table, lens, cu = torch.zeros(2, 2, dtype=torch.int32), torch.ones(2, dtype=torch.int32), torch.tensor([0, 1, 3], dtype=torch.int32)
    wide = torch.zeros(8, 12, 48, dtype=torch.bfloat16)

    def refused(q, out):
        with pytest.raises(ValueError) as e:
            w8.kv_cache_attention(c, q, table, lens, cu, out=out)
        return "overlap" in str(e.value)                         # (else: not on a CUDA device)

    q = wide[2:5, 4:8, 16:32]
    for over in (q, wide[3:6, 4:8, 16:32], wide[0:3, 4:8, 16:32], wide[2:5, 7:11, 16:32], wide[2:5, 4:8, 24:40], wide[2:5, 1:5, 8:24], wide[4:7, 2:6, 16:32]):
        assert refused(q, over)
    for beside in (wide[5:8, 4:8, 16:32], wide[2:5, 8:12, 16:32], wide[2:5, 0:4, 16:32], wide[2:5, 4:8, 32:48], wide[2:5, 4:8, 0:16], wide[3:6, 0:4, 24:40], torch.zeros(3, 4, 16, dtype=torch.bfloat16)):
        assert not refused(q, beside)
    dense = torch.zeros(3 * 4 * 16 + 64, dtype=torch.bfloat16)
    assert refused(dense[:192].view(3, 4, 16), dense[8:200].view(3, 4, 16)) and not refused(dense[64:].view(3, 4, 16).expand(3, 4, 16), dense.new_zeros(3, 4, 16))
    assert refused(dense[:192].view(3, 4, 16), dense[:64].view(1, 4, 16).expand(3, 4, 16))


@pytest.mark.parametrize("seed", range(4))
def test_what_overlaps(seed):
    """Against all elements' places."""
    rng = random.Random(seed)
    for _ in range(400):
        tokens, heads, dim = rng.randint(1, 5), rng.randint(1, 4), 8 * rng.randint(1, 3)
        st, sh = 8 * rng.randint(0, 20), 8 * rng.randint(0, 6)
        if tokens == 1:
            st = 0
        if heads == 1:
            sh = 0
        to = 8 * rng.randint(-60, 60)
        mine = {t * st + h * sh + e for t in range(tokens) for h in range(heads) for e in range(dim)}
        assert kv_cache._overlap(tokens, heads, dim, st, sh, to, st, sh) == any(x + to in mine for x in mine)


@pytest.mark.gpu
def test_outputs_over_queries_are_refused_by_the_library():
    c = Case("int8", 2, 2, 64, [40, 30], [2, 2], seed=54)
    wide = torch.zeros(8, 12, 64, dtype=torch.bfloat16, device="cuda")
    ws = w8.kv_cache_attention_workspace(c.cache, 2, 4, 4)
    kc, ks, vc, vs = c.cache.places()

    def status(q, out):
        return kv_cache._lib.kv_cache_attention(0, kc, ks, vc, vs, c.cache.num_pages, c.page, 2, 64, c.table.data_ptr(), c.table.stride(0), c.table.shape[1], c.lens.data_ptr(), None,
                                                c.cu.data_ptr(), 2, q.data_ptr(), q.stride(0), q.stride(1), 4, 4, None, 0, 0.125, out.data_ptr(), out.stride(0), out.stride(1), None,
                                                ws.data_ptr(), ws.nbytes, torch.cuda.current_stream().cuda_stream)

    q = wide[2:6, 4:8]
    for over in (q, wide[3:7, 4:8], wide[0:4, 6:10], wide[2:6, 1:5], wide[2:6, 4:8].transpose(0, 1)):
        assert status(q, over) == INVALID
    for beside in (wide[2:6, 0:4], wide[2:6, 8:12], wide[3:7, 0:4], torch.empty(4, 4, 64, dtype=torch.bfloat16, device="cuda")):
        assert status(q, beside) == 0
    torch.cuda.synchronize()


def test_workspaces_with_too_few_counters_are_refused():
    """A workspace made for many rows of few sequences, or for other heads, and a call with many sequences: its counters would lie where parts were."""
    lib = kv_cache._lib
    p, need = P(4096), lib.kv_cache_attention_workspace_bytes

    def status(size, seqs, total, q_heads, heads, dim):
        return lib.kv_cache_attention(0, p, p, p, p, 4, 16, heads, dim, p, 3, 3, p, None, p, seqs, p, q_heads * dim, dim, q_heads, total, None, 0, 0.125, p, q_heads * dim, dim,
                                      None, p, size, None)

    for made in ((2, 6000, 8, 2, 64), (1, 400, 64, 8, 128), (1, 300, 4, 2, 256), (1, 1, 4, 2, 128)):
        size = need(*made)
        for seqs, total, q_heads, heads, dim in ((9000, 1, 8, 2, 64), (9000, 10, 8, 2, 128), (7000, 7000, 4, 4, 256), (90000, 90000, 64, 8, 128)):
            counters = lib.kv_cache_attention_zeroed_bytes(seqs, total, q_heads, heads, dim)
            assert counters > lib.kv_cache_attention_zeroed_bytes(*made) and status(size, seqs, total, q_heads, heads, dim) == WORKSPACE


def test_python_workspace_is_zero_where_it_has_to_be():
    for fmt in ("int8", "mxfp4"):
        c = w8.QuantKVCache.empty(4, 4, 2, 64, fmt, device="cpu")
        ws = w8.kv_cache_attention_workspace(c, 500, 3000, 16)
        zeroed = kv_cache._lib.kv_cache_attention_zeroed_bytes(500, 3000, 16, 2, 64)
        assert ws.nbytes == kv_cache._lib.kv_cache_attention_workspace_bytes(500, 3000, 16, 2, 64) and 0 < zeroed < ws.nbytes and not bool(ws[:zeroed].any())
