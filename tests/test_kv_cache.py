"""The quantized paged cache: refusals without a GPU, contents and values read back against plain 64-bit forms on one."""
import ctypes

import pytest
import torch

import lowbit_reference as ref
import paper_2606_14598_b200 as w8
from paper_2606_14598_b200 import kv_cache

INVALID, ALIGNMENT = 1, 2
P = ctypes.c_void_p


def test_write_refusals():
    f = kv_cache._lib.kv_cache_write
    names = ["fmt", "k", "kt", "kh", "v", "vt", "vh", "slots", "tokens", "heads", "dim", "kc", "ks", "vc", "vs", "num_slots", "stream"]
    ok = dict(zip(names, [0, P(4096), 128, 64, P(4096), 128, 64, P(4096), 3, 2, 64, P(4096), P(4096), P(4096), P(4096), 32, None]))

    def status(**change):
        return f(*{**ok, **change}.values())

    for name in ("k", "slots", "kc", "ks", "vc", "vs"):
        assert status(**{name: None}) == INVALID, name
    assert status(fmt=2) == INVALID and status(heads=0) == INVALID and status(dim=0) == INVALID and status(dim=264) == INVALID
    assert status(heads=1025) == INVALID and status(heads=1 << 40) == INVALID
    assert status(tokens=-1) == INVALID and status(num_slots=-1) == INVALID
    assert status(dim=12) == ALIGNMENT and status(kt=129) == ALIGNMENT and status(kh=60) == ALIGNMENT and status(vt=4) == ALIGNMENT
    for name in ("k", "v", "kc", "vc"):
        assert status(**{name: P(4104)}) == ALIGNMENT, name
    assert status(slots=P(4100)) == ALIGNMENT and status(ks=P(4098)) == ALIGNMENT


def test_read_refusals():
    f = kv_cache._lib.kv_cache_read
    names = ["fmt", "kc", "ks", "vc", "vs", "num_pages", "page", "heads", "dim", "table", "stride", "max_pages", "cu", "starts", "seqs", "total",
             "ko", "kt", "kh", "vo", "vt", "vh", "stream"]
    ok = dict(zip(names, [1, P(4096), P(4096), P(4096), P(4096), 4, 16, 2, 64, P(4096), 3, 3, P(4096), None, 2, 10,
                          P(4096), 128, 64, P(4096), 128, 64, None]))

    def status(**change):
        return f(*{**ok, **change}.values())

    for name in ("kc", "ks", "vc", "vs", "table", "cu", "ko"):
        assert status(**{name: None}) == INVALID, name
    assert status(page=0) == INVALID and status(num_pages=-1) == INVALID and status(stride=2) == INVALID and status(total=-1) == INVALID
    assert status(total=1 << 31) == INVALID and status(seqs=-1) == INVALID and status(fmt=-1) == INVALID
    assert status(dim=20) == ALIGNMENT and status(kt=100) == ALIGNMENT and status(vh=2) == ALIGNMENT
    for name in ("kc", "vc", "ko", "vo"):
        assert status(**{name: P(4104)}) == ALIGNMENT, name
    assert status(table=P(4097)) == ALIGNMENT and status(cu=P(4098)) == ALIGNMENT and status(starts=P(4098)) == ALIGNMENT


def test_python_refusals():
    c = w8.QuantKVCache.empty(2, 4, 3, 16, "int8", device="cpu")
    k = torch.zeros(5, 3, 16, dtype=torch.bfloat16)
    slots = torch.arange(5)
    with pytest.raises(TypeError):
        w8.kv_cache_write(c, k.float(), k, slots)
    with pytest.raises(TypeError):
        w8.kv_cache_write(c, k, k, slots.int())
    with pytest.raises(ValueError):
        w8.kv_cache_write(c, k[:4], k, slots)
    with pytest.raises(ValueError):
        w8.kv_cache_write(c, k, None, slots)
    with pytest.raises(ValueError):
        w8.kv_cache_write(c, k, k, slots)                        # no CPU fallback
    with pytest.raises(ValueError):
        w8.QuantKVCache.empty(2, 4, 3, 16, "int4", device="cpu")
    with pytest.raises(ValueError):
        w8.QuantKVCache(c.k_codes, c.k_scales, c.v_codes)
    with pytest.raises(ValueError):
        w8.QuantKVCache(c.k_codes, c.k_scales[:, :2])
    table, cu = torch.zeros(2, 1, dtype=torch.int32), torch.tensor([0, 1, 3], dtype=torch.int32)
    with pytest.raises(TypeError):
        w8.kv_cache_read(c, table.long(), cu, 3)
    with pytest.raises(TypeError):
        w8.kv_cache_read(c, table, cu[:2], 3)
    with pytest.raises(TypeError):
        w8.kv_cache_read(c, table, cu, 3, starts=cu)
    with pytest.raises(ValueError):
        w8.kv_cache_read(c, table, cu, 3, k_out=torch.zeros(2, 3, 16, dtype=torch.bfloat16))


@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_head_sizes_that_the_kernels_do_not_take(fmt):
    """Refused when the cache is made (an odd size in 4 bits would have made a cache of one element less a head)."""
    for dim in (0, -8, 4, 35, 63, 264):
        with pytest.raises(ValueError):
            w8.QuantKVCache.empty(2, 4, 3, dim, fmt, device="cpu")
    for dim in (8, 72, 256):
        assert w8.QuantKVCache.empty(2, 4, 3, dim, fmt, device="cpu").dim == dim


def test_calls_on_nothing_are_not_refused():
    """No tokens, no slots, no rows, no pages: whatever has no elements may be NULL (a tensor without elements has no address). None of
    these calls launches anything; without a GPU they end at the check of the device."""
    write, read = kv_cache._lib.kv_cache_write, kv_cache._lib.kv_cache_read
    p = P(4096)
    assert write(0, None, 0, 0, None, 0, 0, None, 0, 2, 64, p, p, None, None, 32, None) not in (INVALID, ALIGNMENT)
    assert write(1, p, 128, 64, p, 128, 64, p, 3, 2, 64, None, None, None, None, 0, None) not in (INVALID, ALIGNMENT)
    assert write(1, None, 0, 0, None, 0, 0, None, 0, 2, 64, None, None, None, None, 0, None) not in (INVALID, ALIGNMENT)
    assert read(0, p, p, p, p, 4, 16, 2, 64, p, 3, 3, p, None, 2, 0, None, 0, 0, None, 0, 0, None) not in (INVALID, ALIGNMENT)
    assert read(1, None, None, None, None, 0, 16, 2, 64, p, 3, 3, p, None, 2, 0, None, 0, 0, None, 0, 0, None) not in (INVALID, ALIGNMENT)
    # what has elements is still needed
    assert write(0, None, 0, 0, None, 0, 0, p, 1, 2, 64, p, p, None, None, 32, None) == INVALID
    assert write(0, None, 0, 0, None, 0, 0, None, 0, 2, 64, None, p, None, None, 32, None) == INVALID
    assert read(0, None, p, None, None, 4, 16, 2, 64, p, 3, 3, p, None, 2, 0, None, 0, 0, None, 0, 0, None) == INVALID


@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_storage_moved_after_the_cache_was_made(monkeypatch, fmt):
    """The calls get the addresses that the tensors have at the time of the call, and sizes that go with them; memory that has been given
    back is refused. (The calls themselves are recorded: no GPU.)"""
    seen = []
    monkeypatch.setattr(kv_cache, "call", lambda fn, where, dev, *args: seen.append((where, args)))
    c = w8.QuantKVCache.empty(2, 4, 3, 16, fmt, device="cpu")
    k, slots = torch.zeros(5, 3, 16, dtype=torch.bfloat16), torch.arange(5)
    table, cu = torch.zeros(1, 2, dtype=torch.int32), torch.tensor([0, 5], dtype=torch.int32)

    def places():
        seen.clear()
        w8.kv_cache_write(c, k, k, slots)
        w8.kv_cache_read(c, table, cu, 5)
        (_, write), (_, read) = seen
        assert write[11:15] == read[1:5] and write[15] == read[5] * read[6] == c.num_pages * c.page_size
        return write[11:15]

    def now():
        return tuple(t.data_ptr() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales))

    assert places() == now()
    old = c.k_codes.data
    c.k_codes.data = old.clone()
    assert c.k_codes.data_ptr() != old.data_ptr() and places() == now()
    keep = c.v_scales.clone()
    size = c.v_scales.untyped_storage().nbytes()
    c.v_scales.untyped_storage().resize_(0)
    with pytest.raises(ValueError):
        places()
    c.v_scales.untyped_storage().resize_(size)
    c.v_scales.copy_(keep)
    assert places() == now()
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):                # grown by a page
        t.data = torch.cat([t, t[:1]])
    assert places() == now() and c.num_pages == 3
    c.k_scales.data = c.k_scales[:2].clone()
    with pytest.raises(ValueError):
        places()


def test_copy_of_a_cache_has_memory_of_its_own():
    import copy
    import pickle
    c = w8.QuantKVCache.empty(2, 4, 3, 16, "int8", device="cpu")
    for other in (copy.deepcopy(c), pickle.loads(pickle.dumps(c))):
        assert other.places() == tuple(t.data_ptr() for t in (other.k_codes, other.k_scales, other.v_codes, other.v_scales))
        assert not set(other.places()) & set(c.places())


# ------------------------------------------------------------------------------------------ on the GPU

def random_cache(fmt, pages, page, heads, dim, values=True):
    c = w8.QuantKVCache.empty(pages, page, heads, dim, fmt, values=values)
    for codes, scales in ((c.k_codes, c.k_scales), (c.v_codes, c.v_scales)):
        if codes is None:
            continue
        if fmt == "int8":
            codes.copy_(torch.randint(-127, 128, codes.shape, device="cuda"))
            scales.copy_(torch.rand(scales.shape, device="cuda") + 0.01)
        else:
            codes.copy_(torch.randint(0, 256, codes.shape, device="cuda"))
            scales.copy_(torch.randint(100, 150, scales.shape, device="cuda"))
    return c


def expected_write(fmt, codes, scales, x, slots):
    codes, scales = codes.clone().flatten(0, 1), scales.clone().flatten(0, 1)
    keep = (slots >= 0) & (slots < codes.shape[0])
    if fmt == "int8":
        q, s = ref.int8_quantize(x)
        q, s = q.to(torch.int8), s.float()
    else:
        q, s = ref.mx_quantize(x)
        q, s = ref.pack(q), s.to(torch.uint8)
    codes[slots[keep]], scales[slots[keep]] = q[keep], s[keep]
    return codes, scales


def same(a, b):
    return torch.equal(a, b) if a.dtype != torch.float32 else ref.same_values(a, b)


def expected_read(fmt, codes, scales, table, lens, starts, page):
    codes, scales, out = codes.flatten(0, 1), scales.flatten(0, 1), []
    dim = codes.shape[2] * (1 if fmt == "int8" else 2)
    for b, n in enumerate(lens):
        for p in range(starts[b], starts[b] + n):
            at = p // page
            id = int(table[b, at]) if 0 <= p and at < table.shape[1] else -1
            if 0 <= id < codes.shape[0] // page:
                row = id * page + p % page
                if fmt == "int8":
                    out.append((codes[row].float() * scales[row][:, None]).double())     # fp32 product, as defined
                else:
                    out.append(ref.mx_values(ref.unpack(codes[row]), scales[row].long()))
            else:
                out.append(torch.zeros(codes.shape[1], dim, dtype=torch.float64, device=codes.device))
    return torch.stack(out) if out else torch.zeros(0, codes.shape[1], dim, dtype=torch.float64, device=codes.device)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 8, 1), (1, 8, 128, 16), (5, 3, 16, 4), (33, 2, 24, 7), (64, 5, 64, 16), (70, 4, 72, 100),
                                                   (129, 3, 80, 32), (17, 2, 96, 16), (257, 36, 128, 16), (40, 3, 200, 8), (31, 7, 256, 64)])
def test_write(fmt, tokens, heads, dim, page):
    pages = tokens // page + 3
    c = random_cache(fmt, pages, page, heads, dim)
    slots = torch.randperm(pages * page, device="cuda")[:tokens]
    slots[0] = -1 if tokens > 1 else slots[0]
    if tokens > 4:
        slots[2], slots[4] = pages * page, 1 << 40                  # outside: skipped
    qkv = torch.randn(tokens, 3, heads, dim, device="cuda").bfloat16()
    qkv[tokens // 2, 1:] = 0
    if tokens > 8:
        qkv[7, 1, 0, dim - 1], qkv[7, 2, heads - 1, 0] = float("nan"), float("-inf")
        qkv[8, 1:] *= 2.0 ** -125
        qkv[6, 1:] *= 2.0 ** 120
    k, v = qkv[:, 1], qkv[:, 2]                                      # strided: slices of a fused projection
    want = [expected_write(fmt, *side, x, slots) for side, x in (((c.k_codes, c.k_scales), k), ((c.v_codes, c.v_scales), v))]
    w8.kv_cache_write(c, k, v, slots)
    got = [(c.k_codes, c.k_scales), (c.v_codes, c.v_scales)]
    for (gc, gs), (wc, ws) in zip(got, want):
        assert same(gc.flatten(0, 1), wc) and same(gs.flatten(0, 1), ws)
    # the same vectors 16 bytes off a 32-byte boundary, and heads 8 elements apart from a multiple of 16: the same contents
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        t.zero_()
    off = torch.empty(8 + tokens * 3 * heads * (dim + 8), device="cuda", dtype=torch.bfloat16)[8:].view(tokens, 3, heads, dim + 8)[..., :dim]
    off.copy_(qkv)
    w8.kv_cache_write(c, off[:, 1], off[:, 2], slots)
    keep = slots[(slots >= 0) & (slots < pages * page)]
    for (gc, gs), (wc, ws) in zip(got, want):
        assert same(gc.flatten(0, 1)[keep], wc[keep]) and same(gs.flatten(0, 1)[keep], ws[keep])


@pytest.mark.gpu
def test_int8_codes_over_many_scales():
    """16 million elements under 65536 scales from 2^-130 to 2^120, ties of the quotient among them: the codes and scales are those
    of the fp32 division and quotient, whatever way the kernel takes to them."""
    g = torch.Generator("cuda").manual_seed(11)
    x = torch.randn(8192, 8, 256, generator=g, device="cuda") * torch.exp2(torch.randint(-130, 118, (8192, 8, 1), generator=g, device="cuda").float())
    steps = torch.randint(-254, 255, (512, 8, 256), generator=g, device="cuda") / 2.0       # halves of a step of 1: amax 127, every tie
    steps[:, :, 0] = 127.0
    x[:512] = steps * torch.exp2(torch.randint(-100, 100, (512, 8, 1), generator=g, device="cuda").float())
    x = x.bfloat16()
    c = w8.QuantKVCache.empty(128, 64, 8, 256, "int8", values=False)
    w8.kv_cache_write(c, x, None, torch.arange(8192, device="cuda"))
    q, s = ref.int8_quantize(x)
    assert torch.equal(c.k_codes.flatten(0, 1), q.to(torch.int8)) and torch.equal(c.k_scales.flatten(0, 1), s.float())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("lens,heads,dim,page", [([1], 1, 8, 1), ([0, 1, 0, 17, 33, 0], 2, 64, 16), ([100], 5, 72, 16), ([5, 250, 3], 3, 128, 32),
                                                 ([64, 64], 8, 128, 64), ([7, 0, 130], 4, 80, 100), ([40, 1, 1, 1, 60], 2, 256, 7), ([35], 36, 96, 16),
                                                 ([90, 20], 3, 24, 5)])
@pytest.mark.parametrize("window", [False, True])
def test_read(fmt, lens, heads, dim, page, window):
    starts = [(3 * i + 2) % 11 if window else 0 for i in range(len(lens))]
    most = max((n + s + page - 1) // page for n, s in zip(lens, starts)) + 1
    pages = len(lens) * most
    c = random_cache(fmt, pages, page, heads, dim)
    table = torch.randperm(pages, device="cuda").int().view(len(lens), most)
    if page > 1 and len(lens) > 1:
        table[1, 0], table[0, most - 1] = -1, pages                  # missing pages read as zeros
    wide = torch.full((len(lens), most + 2), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :most] = table
    cu = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    first = torch.tensor(starts, dtype=torch.int32, device="cuda") if window else None
    total = sum(lens)
    k, v = w8.kv_cache_read(c, wide[:, :most], cu, total, starts=first)
    assert k.shape == v.shape == (total, heads, dim)
    assert ref.same_values(k, expected_read(fmt, c.k_codes, c.k_scales, table, lens, starts, page))
    assert ref.same_values(v, expected_read(fmt, c.v_codes, c.v_scales, table, lens, starts, page))
    # into strided outputs with rows past the last sequence: only the tokens' heads are written
    buf = torch.full((total + 3, 3, heads, dim), 5.0, device="cuda", dtype=torch.bfloat16)
    w8.kv_cache_read(c, wide[:, :most], cu, total + 3, starts=first, k_out=buf[:, 0], v_out=buf[:, 2])
    assert torch.equal(buf[:total, 0], k) and torch.equal(buf[:total, 2], v)
    assert (buf[total:] == 5).all() and (buf[:, 1] == 5).all()
    # 16 bytes off a 32-byte boundary
    off = torch.empty(8 + total * heads * dim, device="cuda", dtype=torch.bfloat16)[8:].view(total, heads, dim)
    w8.kv_cache_read(c, wide[:, :most], cu, total, starts=first, k_out=off, v_out=buf[:total, 1])
    assert torch.equal(off, k) and torch.equal(buf[:total, 1], v)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_read_past_the_table_and_negative_starts(fmt):
    c = random_cache(fmt, 4, 16, 2, 64)
    table = torch.tensor([[2, 0]], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    k, _ = w8.kv_cache_read(c, table, cu, 50, starts=torch.tensor([-5], dtype=torch.int32, device="cuda"))
    assert (k[:5] == 0).all() and (k[37:] == 0).all()
    assert ref.same_values(k[5:37], expected_read(fmt, c.k_codes, c.k_scales, table, [32], [0], 16))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_one_sided_cache_empty_calls_and_graph(fmt):
    c = w8.QuantKVCache.empty(3, 16, 2, 128, fmt, values=False)
    assert (w8.kv_cache_read(c, torch.zeros(1, 3, dtype=torch.int32, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda"), 4)[0] == 0).all()
    x = torch.randn(20, 2, 128, device="cuda").bfloat16()
    slots = torch.arange(5, 25, device="cuda")
    w8.kv_cache_write(c, x[:0], None, slots[:0])
    table, cu = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    first = torch.tensor([5], dtype=torch.int32, device="cuda")
    empty, none = w8.kv_cache_read(c, table, cu, 0)
    assert empty.shape == (0, 2, 128) and none is None
    out = torch.zeros_like(x)
    w8.kv_cache_write(c, x, None, slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w8.kv_cache_write(c, x, None, slots)
        w8.kv_cache_read(c, table, cu, 20, starts=first, k_out=out)
    x.copy_(torch.randn(20, 2, 128, device="cuda"))
    graph.replay()
    codes, scales = ref.int8_quantize(x) if fmt == "int8" else ref.mx_quantize(x)
    want = (codes.float() * scales.float()[..., None]).double() if fmt == "int8" else ref.mx_values(codes, scales)
    assert ref.same_values(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("values", [True, False])
def test_rows_of_no_sequence(fmt, values):
    """A total beyond the sequences, sequences that begin behind row 0, no sequences at all: the other rows are zeros in outputs that the
    call allocates, and stay as they are in the caller's."""
    heads, dim, total = 3, 72, 300
    c = random_cache(fmt, 20, 16, heads, dim, values=values)
    table = torch.randperm(20, device="cuda").int().view(2, 10)

    def soil():                                                      # blocks that the allocations below get hold NaN
        for _ in range(4):
            torch.full((total, heads, dim), float("nan"), device="cuda", dtype=torch.bfloat16)

    for begin, lens in ((0, [30, 150]), (17, [100, 1]), (5, [0, 0])):
        cu = torch.tensor([begin, begin + lens[0], begin + sum(lens)], dtype=torch.int32, device="cuda")
        end = begin + sum(lens)
        soil()
        got = w8.kv_cache_read(c, table, cu, total)
        for out, codes, scales in ((got[0], c.k_codes, c.k_scales), (got[1], c.v_codes, c.v_scales)):
            if codes is None:
                assert out is None
                continue
            assert (out[:begin] == 0).all() and (out[end:] == 0).all()
            assert ref.same_values(out[begin:end], expected_read(fmt, codes, scales, table, lens, [0, 0], 16))
        soil()
        mine = torch.full((total, heads, dim), 5.0, device="cuda", dtype=torch.bfloat16)
        again = w8.kv_cache_read(c, table, cu, total, k_out=mine)
        assert again[0] is mine and torch.equal(mine[begin:end], got[0][begin:end]) and (mine[:begin] == 5).all() and (mine[end:] == 5).all()
        assert not values or torch.equal(again[1], got[1])
    soil()
    none = w8.kv_cache_read(c, table[:0], cu[:1], total)
    assert (none[0] == 0).all() and (none[1] is None if not values else (none[1] == 0).all())
    w8.kv_cache_read(c, table[:0], cu[:1], total, k_out=mine.fill_(5.0))
    assert (mine == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_cache_without_pages(fmt):
    c = w8.QuantKVCache.empty(0, 16, 2, 64, fmt)
    x = torch.randn(5, 2, 64, device="cuda").bfloat16()
    w8.kv_cache_write(c, x, x, torch.arange(5, device="cuda"))                 # no slot is inside
    cu = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    for table in (torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 0, dtype=torch.int32, device="cuda")):
        k, v = w8.kv_cache_read(c, table, cu, 5)
        assert (k == 0).all() and (v == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("heads,dim,tokens", [(1, 8, 200003), (40, 64, 40007)])
def test_write_of_more_tokens_than_the_grid_holds(fmt, heads, dim, tokens):
    """A launch covers 75776 tokens of up to 256 lanes at a time (half of that where a token takes two CTAs): more go round its loop. The same
    contents as writes of pieces that do not."""
    page, piece = 64, 4096
    pages = tokens // page + 2
    slots = torch.randperm(pages * page, device="cuda")[:tokens]
    slots[::1001] = -1
    x = torch.randn(tokens, 2, heads, dim, device="cuda").bfloat16()
    whole, parts = (w8.QuantKVCache.empty(pages, page, heads, dim, fmt) for _ in range(2))
    w8.kv_cache_write(whole, x[:, 0], x[:, 1], slots)
    for t in range(0, tokens, piece):
        w8.kv_cache_write(parts, x[t:t + piece, 0], x[t:t + piece, 1], slots[t:t + piece])
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(whole, name), getattr(parts, name)), name
    last = slots[tokens - 1]                                          # (its slot was written at all)
    assert whole.k_scales.flatten(0, 1)[last].any()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
@pytest.mark.parametrize("heads,dim,seqs,most", [(1, 8, 1500, 300), (1, 24, 3, 90000), (40, 64, 300, 400)])
def test_read_of_more_tokens_than_the_grid_holds(fmt, heads, dim, seqs, most):
    """The loop over the grid again, with hundreds of sequences to search (more than a CTA has threads) and with a few long ones."""
    g = torch.Generator("cuda").manual_seed(seqs)
    page = 16
    lens = torch.randint(0, most + 1, (seqs,), generator=g, device="cuda")
    lens[0], lens[seqs // 2], lens[-1] = 0, most, most
    starts = torch.randint(0, 40, (seqs,), generator=g, device="cuda")
    width = int((lens + starts).max()) // page + 1
    pages = 997
    c = random_cache(fmt, pages, page, heads, dim)
    table = torch.randint(0, pages, (seqs, width), generator=g, device="cuda")
    table[torch.rand(seqs, width, generator=g, device="cuda") < 0.01] = -1
    cu = torch.cat([lens.new_zeros(1), lens.cumsum(0)])
    total = int(cu[-1])
    assert total > 2 * 75776 or (heads * dim > 2048 and total > 37888)
    k, v = w8.kv_cache_read(c, table.int(), cu.int(), total, starts=starts.int())
    seq = torch.repeat_interleave(torch.arange(seqs, device="cuda"), lens)
    at = torch.arange(total, device="cuda") - cu[seq] + starts[seq]
    id = table[seq, at // page]
    row = (id * page + at % page).clamp(min=0)
    for out, codes, scales in ((k, c.k_codes.flatten(0, 1), c.k_scales.flatten(0, 1)), (v, c.v_codes.flatten(0, 1), c.v_scales.flatten(0, 1))):
        for t in range(0, total, 20000):
            r, there = row[t:t + 20000], (id[t:t + 20000] >= 0)[:, None, None]
            want = (codes[r].float() * scales[r][..., None]).double() if fmt == "int8" else ref.mx_values(ref.unpack(codes[r]), scales[r].long())
            assert ref.same_values(out[t:t + 20000], torch.where(there, want, torch.zeros_like(want))), t


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "mxfp4"])
def test_offsets_past_32_bits(fmt):
    heads, dim, page = 64, 256, 64
    pages = ((1 << 32) // (heads * dim * page // (1 if fmt == "int8" else 2))) + 3        # the codes pass 2^32 bytes
    c = w8.QuantKVCache.empty(pages, page, heads, dim, fmt, values=False)
    x = torch.randn(page, heads, dim, device="cuda").bfloat16()
    slots = torch.arange((pages - 1) * page, pages * page, device="cuda")
    w8.kv_cache_write(c, x, None, slots)
    table, cu = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda"), torch.tensor([0, page], dtype=torch.int32, device="cuda")
    k, _ = w8.kv_cache_read(c, table, cu, page)
    codes, scales = ref.int8_quantize(x) if fmt == "int8" else ref.mx_quantize(x)
    want = (codes.float() * scales.float()[..., None]).double() if fmt == "int8" else ref.mx_values(codes, scales)
    assert ref.same_values(k, want)
    assert not c.k_codes[: pages - 1].any()
