"""Appending rotated keys and values to the quantized cache: refusals without a GPU, queries and codes to the bit against plain 64-bit forms on one."""
import ctypes
import math

import pytest
import torch

import lowbit_reference as ref
import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import kv_cache

INVALID, ALIGNMENT = 1, 2
P = ctypes.c_void_p
NAN = float("nan")


def test_refusals():
    f = kv_cache._lib.kv_cache_append
    names = ["fmt", "q", "qt", "qh", "q_heads", "qo", "ot", "oh", "k", "kt", "kh", "v", "vt", "vh", "cs", "positions_of", "rot", "inter", "pos", "stride", "axes", "axis_of", "slots",
             "tokens", "heads", "dim", "kc", "ks", "vc", "vs", "num_slots", "stream"]
    p = P(4096)
    ok = dict(zip(names, [0, p, 256, 64, 4, p, 256, 64, p, 128, 64, p, 128, 64, p, 100, 64, 0, p, 3, 3, p, p, 3, 2, 64, p, p, p, p, 32, None]))

    def status(**change):
        return f(*{**ok, **change}.values())

    for name in ("q", "qo", "k", "pos", "axis_of", "slots", "kc", "ks", "vc", "vs"):
        assert status(**{name: None}) == INVALID, name
    assert status(fmt=2) == INVALID and status(heads=0) == INVALID and status(dim=0) == INVALID and status(dim=264) == INVALID and status(heads=1025) == INVALID
    assert status(q_heads=-1) == INVALID and status(q_heads=1025) == INVALID and status(tokens=-1) == INVALID and status(num_slots=-1) == INVALID
    assert status(rot=0) == INVALID and status(rot=72) == INVALID and status(axes=0) == INVALID and status(axes=9) == INVALID and status(stride=2) == INVALID
    assert status(positions_of=-1) == INVALID
    for name in ("qt", "qh", "ot", "oh", "kt", "kh", "vt", "vh"):
        assert status(**{name: 132}) == ALIGNMENT, name
    for name in ("q", "qo", "k", "v", "cs", "kc", "vc"):
        assert status(**{name: P(4104)}) == ALIGNMENT, name
    assert status(dim=60, rot=56) == ALIGNMENT and status(rot=60) == ALIGNMENT and status(slots=P(4100)) == ALIGNMENT and status(pos=P(4100)) == ALIGNMENT
    assert status(ks=P(4098)) == ALIGNMENT
    # no queries, no rotation, no values, one axis, no tokens: what they would need is not asked for
    assert status(q=None, qo=None, q_heads=0) not in (INVALID, ALIGNMENT)
    assert status(cs=None, pos=None, axis_of=None, rot=0, axes=0) not in (INVALID, ALIGNMENT)
    assert status(v=None, vc=None, vs=None) not in (INVALID, ALIGNMENT)
    assert status(axes=1, axis_of=None, stride=0) not in (INVALID, ALIGNMENT)
    assert status(tokens=0, k=None, slots=None, q=None, qo=None, pos=None, v=None) not in (INVALID, ALIGNMENT)
    table = kv_cache._lib.kv_cache_rope_table
    assert table(None, 8, 0, 4, 1.0, p, None) == INVALID and table(p, 0, 0, 4, 1.0, p, None) == INVALID and table(p, 8, 0, -1, 1.0, p, None) == INVALID
    assert table(p, 8, 0, 4, NAN, p, None) == INVALID and table(p, 8, 0, 4, 1.0, None, None) == INVALID and table(P(4100), 8, 0, 4, 1.0, p, None) == ALIGNMENT
    assert table(p, 8, 1 << 53, 4, 1.0, p, None) == INVALID


def test_python_refusals():
    c = w8.QuantKVCache.empty(2, 4, 3, 16, "int8", device="cpu")
    k, q = torch.zeros(5, 3, 16, dtype=torch.bfloat16), torch.zeros(5, 6, 16, dtype=torch.bfloat16)
    slots, pos, cs = torch.arange(5), torch.arange(5), torch.zeros(9, 16)
    call = w8.kv_cache_append
    with pytest.raises(ValueError):
        call(c, k, None, slots)
    with pytest.raises(TypeError):
        call(c, k, k, slots, cos_sin=cs)
    with pytest.raises(TypeError):
        call(c, k, k, slots, pos.int(), cs)
    with pytest.raises(ValueError):
        call(c, k, k, slots, pos[:4], cs)
    with pytest.raises(TypeError):
        call(c, k, k, slots, pos, cs.double())
    with pytest.raises(ValueError):
        call(c, k, k, slots, pos.expand(2, 5).contiguous(), cs)
    with pytest.raises(TypeError):
        call(c, k, k, slots, pos.expand(2, 5).contiguous(), cs, axes=torch.zeros(7, dtype=torch.uint8))
    with pytest.raises(TypeError):
        call(c, k, k, slots, pos, cs, q=q.float())
    with pytest.raises(ValueError):
        call(c, k, k, slots, pos, cs, q=q[:4])
    with pytest.raises(ValueError):
        call(c, k, k, slots, pos, cs, q_out=q)
    with pytest.raises(ValueError):
        call(c, k, k, slots, pos, cs, q=q)                       # no CPU fallback
    with pytest.raises(TypeError):
        w8.kv_cache_rope_table(torch.ones(8), 4)
    with pytest.raises(ValueError):
        w8.kv_cache_rope_table(torch.ones(8, dtype=torch.float64), 4)


# ------------------------------------------------------------------------------------------------ on the GPU

def single(x):
    return x.float().double()


def rotate(x, cos_sin, positions, axes, interleaved):
    """[T, heads, dim] in 64 bits, pair by pair, rounded to fp32 where the definition rounds; positions outside the table give NaN."""
    rot = cos_sin.shape[1]
    pairs, out = rot // 2, x.double().clone()
    positions = positions if positions.dim() == 2 else positions[None]
    for i in range(pairs):
        axis = 0 if axes is None else int(axes[i])
        if axis < positions.shape[0]:
            p = positions[axis]
            inside = (p >= 0) & (p < cos_sin.shape[0])
            p = p.clamp(0, cos_sin.shape[0] - 1)
            c, s = (torch.where(inside, cos_sin[p, i + n * pairs].double(), NAN)[:, None] for n in (0, 1))
        else:
            c = s = torch.full((x.shape[0], 1), NAN, dtype=torch.float64, device=x.device)
        one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        a, b = x[..., one].double(), x[..., two].double()
        out[..., one], out[..., two] = single(single(a * c) - single(b * s)), single(single(b * c) + single(a * s))
    return out


def contents(fmt, x):
    """Codes and scales that a cache keeps of [T, heads, dim]."""
    if fmt == "int8":
        codes, s = ref.int8_quantize(x)
        return codes.to(torch.int8), s.float()
    codes, s = ref.mx_quantize(x)
    return ref.pack(codes), s.to(torch.uint8)


def same(a, b):
    return bool(((a == b) | (torch.isnan(a.float()) & torch.isnan(b.float()))).all())


def check(fmt, tokens, q_heads, heads, dim, rot, axes=1, interleaved=False, page=16, positions=None, values=True, seed=0, in_place=False, slots=None, x=None):
    gen = torch.Generator("cuda").manual_seed(seed)
    pages = (tokens + page - 1) // page + 2
    cache = w8.QuantKVCache.empty(pages, page, heads, dim, fmt, values=values)
    for t in cache._tensors:                                     # what is in the cache before stays where nothing is appended
        if t is not None:
            t.copy_(torch.randint(1, 100, t.shape, generator=gen, device="cuda").to(t.dtype))
    before = [None if t is None else t.clone() for t in cache._tensors]
    x = torch.randn(tokens, q_heads + 2 * heads, dim, generator=gen, device="cuda").to(torch.bfloat16) if x is None else x
    q, k, v = x[:, :q_heads], x[:, q_heads:q_heads + heads], x[:, q_heads + heads:]
    if slots is None:
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:tokens]
    cos_sin = torch.randn(50, rot, generator=gen, device="cuda") if rot else None
    if positions is None:
        positions = torch.randint(0, 50, (axes, tokens), generator=gen, device="cuda")
    axis_of = torch.randint(0, axes, (rot // 2,), generator=gen, device="cuda").to(torch.uint8) if rot and axes > 1 else None
    want_q, want_k = (rotate(t, cos_sin, positions, axis_of, interleaved) if rot else t.double() for t in (q, k))
    want = [*contents(fmt, want_k), *(contents(fmt, v.double()) if values else (None, None))]
    got = w8.kv_cache_append(cache, k, v if values else None, slots, positions[0] if axes == 1 else positions, cos_sin, axes=axis_of, interleaved=interleaved,
                             q=q if q_heads else None, q_out=q if in_place and q_heads else None)
    if q_heads:
        assert ref.same_values(got, want_q)
    else:
        assert got is None
    kept = (slots >= 0) & (slots < pages * page)
    for t, old, new in zip(cache._tensors, before, want):
        if t is None:
            continue
        flat = old.flatten(0, 1)
        flat[slots[kept]] = new[kept]
        assert same(t.flatten(0, 1), flat)
    return cache, got


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("q_heads,heads,dim,rot", [(4, 2, 64, 64), (1, 1, 8, 8), (16, 16, 72, 72), (10, 5, 80, 40), (8, 1, 96, 24), (32, 8, 128, 128), (3, 3, 256, 256), (6, 2, 136, 104), (0, 7, 128, 64)])
def test_one_axis(fmt, q_heads, heads, dim, rot, interleaved):
    for tokens in (1, 3, 77):
        check(fmt, tokens, q_heads, heads, dim, rot, interleaved=interleaved, seed=tokens)
    check(fmt, 19, q_heads, heads, dim, rot, interleaved=interleaved, in_place=True, values=False)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("axes", [2, 3, 8])
def test_several_axes(fmt, axes, interleaved):
    check(fmt, 41, 5, 5, 72, 72, axes=axes, interleaved=interleaved)
    check(fmt, 300, 8, 2, 128, 96, axes=axes, interleaved=interleaved, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_sections_of_pairs(fmt):
    """Runs of pairs on one axis, the way that images are given: time, then height, then width."""
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(60, 6, 64, generator=gen, device="cuda").to(torch.bfloat16)
    cache = w8.QuantKVCache.empty(4, 16, 2, 64, fmt)
    where = torch.arange(60, device="cuda")
    positions = torch.stack([where // 30, where // 6 % 5, where % 6])
    axes = torch.tensor([0] * 8 + [1] * 12 + [2] * 12, dtype=torch.uint8, device="cuda")
    table = w8.kv_cache_rope_table(torch.tensor([100.0 ** (-i / 32) for i in range(32)], dtype=torch.float64, device="cuda"), 30)
    q = w8.kv_cache_append(cache, x[:, 2:4], x[:, 4:], where, positions, table, axes=axes, q=x[:, :2])
    assert ref.same_values(q, rotate(x[:, :2], table, positions, axes, False))
    codes, scales = contents(fmt, rotate(x[:, 2:4], table, positions, axes, False))
    assert torch.equal(cache.k_codes.flatten(0, 1)[:60], codes) and torch.equal(cache.k_scales.flatten(0, 1)[:60], scales)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_without_rotation_it_is_a_write(fmt):
    gen = torch.Generator("cuda").manual_seed(1)
    a, b = (w8.QuantKVCache.empty(20, 16, 3, 72, fmt) for _ in range(2))
    x = (torch.randn(300, 9, 72, generator=gen, device="cuda") * torch.exp2(torch.randint(-60, 60, (300, 9, 1), generator=gen, device="cuda"))).to(torch.bfloat16)
    x[5, 3] = 0
    x[6, 4, 3], x[7, 7, 70] = NAN, float("inf")
    slots = torch.randperm(320, generator=gen, device="cuda")[:300]
    w8.kv_cache_write(a, x[:, 3:6], x[:, 6:], slots)
    q = w8.kv_cache_append(b, x[:, 3:6], x[:, 6:], slots, q=x[:, :3])
    assert same(q, x[:, :3])
    for s, t in zip(a._tensors, b._tensors):
        assert same(s, t)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_positions_and_slots_outside(fmt, interleaved):
    """A position outside the table makes the token NaN (visibly), a slot outside the cache leaves the cache alone; other tokens do not notice."""
    positions = torch.randint(0, 50, (1, 40), device="cuda")
    positions[0, 3], positions[0, 4], positions[0, 5] = -1, 50, 1 << 40
    slots = torch.randperm(64, device="cuda")[:40]
    slots[7], slots[8], slots[9] = -1, 80, 1 << 50
    cache, q = check(fmt, 40, 4, 2, 128, 64, positions=positions, slots=slots, interleaved=interleaved)
    assert bool(torch.isnan(q[3:6, :, :64]).all()) and not bool(torch.isnan(q[3:6, :, 64:]).any()) and not bool(torch.isnan(q[7:]).any())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_extremes(fmt):
    gen = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(64, 12, 128, generator=gen, device="cuda") * torch.exp2(torch.randint(-120, 110, (64, 12, 1), generator=gen, device="cuda"))
    x[0] = 0
    x = x.to(torch.bfloat16)
    x[1, 4, 5], x[2, 5, 100], x[3, 9, 0] = NAN, float("inf"), -float("inf")
    check(fmt, 64, 4, 4, 128, 64, x=x)
    check(fmt, 64, 4, 4, 128, 128, x=x, interleaved=True)


@pytest.mark.gpu
def test_rope_table():
    """Angles of far positions: 64 bits, against the same in Python's floats."""
    freq = [10000.0 ** (-i / 16) for i in range(16)]
    for first, scale in ((0, 1.0), (1 << 20, 0.5), (-7, 1.0)):
        got = w8.kv_cache_rope_table(torch.tensor(freq, dtype=torch.float64, device="cuda"), 33, first, scale).cpu()
        want = torch.tensor([[scale * f((first + p) * w) for f in (math.cos, math.sin) for w in freq] for p in range(33)], dtype=torch.float64)
        assert got.shape == (33, 32)
        assert bool(((got.double() - want).abs() <= want.abs() * 2.0 ** -24 + 1e-15).all())     # one rounding to fp32, and 64-bit errors
    assert w8.kv_cache_rope_table(torch.ones(4, dtype=torch.float64, device="cuda"), 0).shape == (0, 8)


@pytest.mark.gpu
def test_no_tokens_graph_and_stream():
    gen = torch.Generator("cuda").manual_seed(4)
    x = torch.randn(9, 8, 64, generator=gen, device="cuda").to(torch.bfloat16)
    slots, positions, cos_sin = torch.arange(9, device="cuda"), torch.arange(9, device="cuda"), torch.randn(9, 64, generator=gen, device="cuda")
    a, b = (w8.QuantKVCache.empty(1, 16, 2, 64, "int8") for _ in range(2))
    want = w8.kv_cache_append(a, x[:, 4:6], x[:, 6:], slots, positions, cos_sin, q=x[:, :4])
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        w8.kv_cache_append(b, x[:, 4:6], x[:, 6:], slots, positions, cos_sin, q=x[:, :4], q_out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all(torch.equal(s, t) for s, t in zip(a._tensors, b._tensors))
    assert w8.kv_cache_append(a, x[:0, 4:6], x[:0, 6:], slots[:0], positions[:0], cos_sin, q=x[:0, :4]).shape == (0, 4, 64)


@pytest.mark.gpu
def test_many_tokens():
    """More tokens than the grid has CTAs: the loop over them."""
    check("int8", 6001, 3, 1, 64, 64, page=64)
    check("mxfp4", 6001, 3, 1, 72, 72, page=64, interleaved=True)
