"""Workloads of the operators around a quantized cache and the int8 linear: in plain form and through the package.

Three kinds of pass, over the sizes that a token-by-token decoder, a decoder that checks drafted tokens and a diffusion
transformer give them:

* ``norm``    h = bf16(x + residual), the root-mean-square norm of h times a weight, as int8 codes with a scale a row (what the
              int8 linear takes) or as bf16 (what the 4-bit linear takes).
* ``append``  new tokens' queries and keys rotated by their positions (one axis, or time, height and width), keys and values
              quantized into a paged cache (int8 with a scale a head, or MXFP4); the new tokens are then read back.
* ``attend``  attention of new tokens over the cache: one token a sequence, or a tree of drafted ones, each of which sees the
              sequence before the tree and its own ancestors.

``own`` is false for the plain torch forms and true for the package's kernels.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 32
EPS = 1e-6
# magnitudes of the eight E2M1 codes; bit 3 of a code is the sign
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one token ahead of a projection: what a decoder does twice a layer; latency counts
        {"name": "norm_one_token", "op": "norm", "m": 1, "k": 4608, "out": "int8", "residual": True, "pad": 0},
        # all tokens of a 1024-pixel image with its prompt, ahead of the int8 projections of a block
        {"name": "norm_image_int8", "op": "norm", "m": 4110, "k": 4608, "out": "int8", "residual": True, "pad": 0},
        # two images' tokens ahead of a 4-bit linear, a slice of a wider buffer, odd row count
        {"name": "norm_wide_bf16", "op": "norm", "m": 8221, "k": 12288, "out": "bf16", "residual": True, "pad": 64},
        # one new token in each of 48 sequences of a decoder with grouped heads
        {"name": "append_step_int8", "op": "append", "fmt": "int8", "seqs": 48, "new": 1, "context": 4000, "q_heads": 32, "heads": 8, "dim": 128, "rot": 128, "axes": 1,
         "interleaved": False, "page": 16},
        # a long prompt's tokens at once
        {"name": "append_prompt_int8", "op": "append", "fmt": "int8", "seqs": 2, "new": 8000, "context": 8000, "q_heads": 32, "heads": 8, "dim": 128, "rot": 128, "axes": 1,
         "interleaved": False, "page": 64},
        # two images' tokens, positions in time, height and width, odd head size
        {"name": "append_image_mxfp4", "op": "append", "fmt": "mxfp4", "seqs": 2, "new": 4110, "context": 4110, "q_heads": 16, "heads": 16, "dim": 72, "rot": 72, "axes": 3,
         "interleaved": True, "page": 64},
        # one token of one short conversation: latency counts
        {"name": "attend_one_int8", "op": "attend", "fmt": "int8", "seqs": 1, "new": 1, "context": 777, "q_heads": 32, "heads": 8, "dim": 128, "page": 16},
        # one new token in each of 48 sequences of very different lengths
        {"name": "attend_step_int8", "op": "attend", "fmt": "int8", "seqs": 48, "new": 1, "context": 4000, "q_heads": 32, "heads": 8, "dim": 128, "page": 16},
        # one new token in each of a few long sequences
        {"name": "attend_long_mxfp4", "op": "attend", "fmt": "mxfp4", "seqs": 12, "new": 1, "context": 30000, "q_heads": 64, "heads": 8, "dim": 128, "page": 64},
        # small trees of drafted tokens, one head of keys a query head, odd head size
        {"name": "attend_draft_mxfp4", "op": "attend", "fmt": "mxfp4", "seqs": 5, "new": 7, "context": 1500, "q_heads": 16, "heads": 16, "dim": 72, "page": 16},
        # trees of drafted tokens in a batch
        {"name": "attend_tree_int8", "op": "attend", "fmt": "int8", "seqs": 12, "new": 32, "context": 6000, "q_heads": 32, "heads": 8, "dim": 128, "page": 64},
        # large trees over long documents
        {"name": "attend_tree_mxfp4", "op": "attend", "fmt": "mxfp4", "seqs": 3, "new": 61, "context": 20000, "q_heads": 64, "heads": 8, "dim": 128, "page": 64},
    ]


def draw(rng):
    def spread(lo, hi, step=1):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))

    op = rng.choice(("norm", "append", "append", "attend", "attend", "attend"))
    if op == "norm":
        k = spread(256, 12288, 16)
        return {"op": op, "m": spread(1, min(16384, 8221 * 12288 // k)), "k": k, "out": rng.choice(("int8", "int8", "bf16")), "residual": rng.random() < 0.8, "pad": rng.choice((0, 64))}
    fmt = rng.choice(("int8", "mxfp4"))
    heads, group = rng.choice((1, 2, 5, 8, 16)), rng.choice((1, 2, 4, 5, 8))
    dim, page = rng.choice((64, 72, 80, 96, 128, 256)), rng.choice((16, 32, 64, 100))
    if op == "append":
        axes = rng.choice((1, 1, 3))
        rot = dim if axes == 3 else rng.choice((dim, dim, dim // 2 // 8 * 8))
        case = {"op": op, "fmt": fmt, "q_heads": heads * group, "heads": heads, "dim": dim, "rot": rot, "axes": axes, "interleaved": rng.random() < 0.5, "page": page}
        if rng.random() < 0.5:
            most = 16000 * 48 * 128 // ((group + 2) * heads * dim)
            new = spread(16, min(8000, most))
            return {**case, "seqs": rng.randint(1, 2) if 2 * new <= most else 1, "new": new, "context": new}
        return {**case, "seqs": spread(1, 64), "new": rng.choice((1, 1, 1, 4)), "context": spread(64, 4000)}
    new = rng.choice((1, 1, 1, 2, spread(3, 64)))
    seqs = spread(1, 64)
    # no more bytes than the longest listed case, and no more products than the largest tree
    most = min(12 * 30000 * 8 * 128 // (seqs * heads * dim), 3 * 61 * 20000 * 64 * 128 // (seqs * new * heads * group * dim))
    return {"op": op, "fmt": fmt, "seqs": seqs, "new": new, "context": spread(64, max(65, min(30000, most))), "q_heads": heads * group, "heads": heads, "dim": dim, "page": page}


# ------------------------------------------------------------------------------------------------ inputs

def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def activations(gen, m, k):
    """N(0, 1) with one channel in a hundred twenty times as large, the outlier channels of a transformer's activations."""
    loud = torch.randperm(k, generator=gen, device=DEV)[: max(1, k // 100)]
    x = normal(gen, m, k)
    x[:, loud] *= 20.0
    return x


def lengths(case):
    """Tokens of each sequence of a cache: from a quarter of the context to all of it, in no order (odd ones among them)."""
    seqs, most = case["seqs"], case["context"]
    least = max(min(case["new"], most), most // 4)
    return [most - (most - least) * (i * 29 % seqs) // seqs for i in range(seqs)]


def news(case):
    """New tokens of each sequence: the same number when they are appended or are one each; trees differ in size."""
    if case["op"] == "append" or case["new"] == 1:
        return [case["new"]] * case["seqs"]
    return [max(1, min(n, case["new"] - i % 3)) for i, n in enumerate(lengths(case))]


def trees(counts, seed):
    """For each node the bits of its ancestors and itself: node j's parent is one of the nodes before it, or the sequence."""
    rng, rows = random.Random(seed), []
    for n in counts:
        bits = []
        for j in range(n):
            parent = rng.randint(max(-1, j - 12), j - 1) if j else -1
            bits.append((1 << j) | (bits[parent] if parent >= 0 else 0))
        rows += [b - (1 << 64) if b >> 63 else b for b in bits]
    return torch.tensor(rows, dtype=torch.int64, device=DEV)[:, None]


def angles(case):
    """cos and sin of (position x frequency) [positions, rot]: cosines of all pairs, then their sines; pairs of an axis have its frequencies."""
    pairs = case["rot"] // 2
    axis = axis_of_pair(case)
    at = [sum(a == b for b in axis[:i]) for i, a in enumerate(axis)]
    count = [axis.count(a) for a in axis]
    freq = torch.tensor([10000.0 ** (-i / c) for i, c in zip(at, count)], dtype=torch.float64, device=DEV)
    t = torch.arange(case["context"] + 1, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.cat([t.cos(), t.sin()], 1).float() if pairs else None


def axis_of_pair(case):
    """A quarter of the pairs turn with time, the others with height and width."""
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return [0] * pairs
    first, second = pairs // 4, pairs // 4 + (pairs - pairs // 4) // 2
    return [0 if i < first else 1 if i < second else 2 for i in range(pairs)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    state = {"op": case["op"], "case": case}
    if case["op"] == "norm":
        m, k, pad = case["m"], case["k"], case["pad"]
        state["x"] = activations(gen, m, k + pad).to(torch.bfloat16)[:, :k]
        state["residual"] = (normal(gen, m, k + pad) * 3.0).to(torch.bfloat16)[:, :k] if case["residual"] else None
        state["weight"] = 1.0 + 0.2 * normal(gen, k)
        return state
    seqs, heads, dim, page, q_heads = case["seqs"], case["heads"], case["dim"], case["page"], case["q_heads"]
    counts = news(case)
    lens, new = torch.tensor(lengths(case), device=DEV), torch.tensor(counts, device=DEV)
    pages_of = (lens + page - 1) // page
    most, count = int(pages_of.max()), int(pages_of.sum()) + 3
    order = torch.randperm(count, generator=gen, device=DEV)
    first = torch.cumsum(pages_of, 0) - pages_of
    slot = torch.arange(most, device=DEV)
    table = torch.where(slot < pages_of[:, None], order[(first[:, None] + slot).clamp(max=count - 1)], -1)
    state["table"] = table.to(torch.int32)
    state["lens"] = lens.to(torch.int32)
    state["starts"] = (lens - new).to(torch.int32)
    state["total"] = sum(counts)
    state["cu"] = torch.cat([new.new_zeros(1), torch.cumsum(new, 0)]).to(torch.int32)
    seq = torch.repeat_interleave(torch.arange(seqs, device=DEV), new)
    node = torch.arange(state["total"], device=DEV) - state["cu"][seq]
    where = lens[seq] - new[seq] + node
    # queries, keys and values come out of a fused projection: [tokens, query heads + 2 x heads, dim]
    qkv = activations(gen, state["total"], (q_heads + 2 * heads) * dim if case["op"] == "append" else q_heads * dim).to(torch.bfloat16).view(state["total"], -1, dim)
    state["q"] = qkv[:, :q_heads]
    for which in "kv":
        if case["fmt"] == "int8":
            codes = torch.randint(-127, 128, (count, page, heads, dim), generator=gen, device=DEV, dtype=torch.int8)
            scales = torch.rand(count, page, heads, generator=gen, device=DEV) * 0.01 + 0.01
        else:
            codes = torch.randint(0, 256, (count, page, heads, dim // 2), generator=gen, device=DEV, dtype=torch.uint8)
            scales = torch.randint(124, 128, (count, page, heads, (dim + 31) // 32), generator=gen, device=DEV, dtype=torch.uint8)
        state[which + "_codes"], state[which + "_scales"] = codes, scales
    if case["op"] == "append":
        state["k"], state["v"] = qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
        state["slots"] = table[seq, where // page] * page + where % page
        side = max(1, math.isqrt(case["context"]))
        state["positions"] = torch.stack([where // (side * side), where // side % side, where % side]) if case["axes"] == 3 else where
        state["cos_sin"] = angles(case)
        state["axes"] = torch.tensor(axis_of_pair(case), dtype=torch.uint8, device=DEV) if case["axes"] > 1 else None
        return state
    state["tree"] = None if case["new"] == 1 else trees(counts, seed)
    # the rows of the queries in a padded batch [sequences, most new tokens]
    state["padded"] = seq * max(counts) + node
    return state


# ------------------------------------------------------------------------------------------------ plain forms

def from_mxfp4(codes, scale_bytes):
    """The fp32 values that packed codes [..., K / 2] and scale bytes [..., ceil(K / 32)] stand for."""
    table = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], dim=-1)
    code = code.view(*codes.shape[:-1], 2 * codes.shape[-1])
    e = scale_bytes.to(torch.int32)
    scale = torch.where(e == 0, torch.full_like(e, 1 << 22), e << 23).view(torch.float32)
    return table[code.int()] * scale.repeat_interleave(BLOCK, dim=-1)[..., :code.shape[-1]]


def to_mxfp4(x):
    """Packed codes and scale bytes of fp32 [..., K]: 2 ** (floor(log2(largest of 32)) - 2), nearest E2M1 value, ties to the even code."""
    k = x.shape[-1]
    blocks = (k + BLOCK - 1) // BLOCK
    if k % BLOCK:
        x = torch.cat([x, x.new_zeros(*x.shape[:-1], blocks * BLOCK - k)], dim=-1)
    x = x.view(*x.shape[:-1], blocks, BLOCK)
    scale = ((x.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp(min=0)
    mag = x.abs() * ((254 - scale) << 23).view(torch.float32)[..., None]
    code = (mag > 0.25).to(torch.uint8)
    code += mag >= 0.75
    code += mag > 1.25
    code += mag >= 1.75
    code += mag > 2.5
    code += mag >= 3.5
    code += mag > 5.0
    code += (x < 0).to(torch.uint8) * 8
    code = code.view(*code.shape[:-2], blocks * BLOCK)[..., :k]
    return code[..., 0::2] | (code[..., 1::2] << 4), scale.to(torch.uint8)


def to_int8(x):
    """(whole numbers, scales) of fp32 rows: the largest magnitude / 127 is the scale of a row."""
    largest = x.abs().amax(-1)
    s = torch.where(largest > 0, largest / torch.full_like(largest, 127.0), torch.ones_like(largest))
    return torch.round(x / s[..., None]).clamp(-127, 127), s


def plain_norm(state):
    h = state["x"] if state["residual"] is None else (state["x"].float() + state["residual"].float()).to(torch.bfloat16)
    # codes go by h * weight alone: the norm is a factor of the whole row, and of its scale
    u = h.float() * state["weight"]
    r = (h.double().square().mean(-1) + EPS).rsqrt().float()
    if state["case"]["out"] == "bf16":
        return h, (u * r[:, None]).to(torch.bfloat16)
    q, s = to_int8(u)
    return h, (q * (s * r)[:, None]).to(torch.bfloat16)


def plain_rotate(state, x):
    """fp32 [tokens, heads, dim] rotated: pair i of a token by the angle of its position on the pair's axis."""
    case = state["case"]
    rot, pairs = case["rot"], case["rot"] // 2
    at = state["positions"][state["axes"].long()].t() if case["axes"] > 1 else state["positions"][:, None].expand(-1, pairs)
    pair = torch.arange(pairs, device=DEV)
    c, s = state["cos_sin"][at, pair][:, None], state["cos_sin"][at, pairs + pair][:, None]
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :pairs], x[..., pairs:rot])
    turned = (a * c - b * s, b * c + a * s)
    turned = torch.stack(turned, -1).flatten(-2) if case["interleaved"] else torch.cat(turned, -1)
    return torch.cat([turned, x[..., rot:]], -1)


def plain_store(state, which, x):
    codes, scales, slots = state[which + "_codes"].flatten(0, 1), state[which + "_scales"].flatten(0, 1), state["slots"]
    if state["case"]["fmt"] == "int8":
        q, s = to_int8(x)
        codes[slots], scales[slots] = q.to(torch.int8), s
        return (codes[slots].float() * scales[slots][..., None]).to(torch.bfloat16)
    codes[slots], scales[slots] = to_mxfp4(x)
    return from_mxfp4(codes[slots], scales[slots]).to(torch.bfloat16)


def plain_append(state):
    return plain_rotate(state, state["q"]).to(torch.bfloat16), plain_store(state, "k", plain_rotate(state, state["k"])), plain_store(state, "v", state["v"].float())


def plain_values(state, which, row):
    codes, scales = state[which + "_codes"].flatten(0, 1)[row], state[which + "_scales"].flatten(0, 1)[row]
    return codes.float() * scales[..., None] if state["case"]["fmt"] == "int8" else from_mxfp4(codes, scales)


def plain_attend(state):
    case = state["case"]
    seqs, heads, dim, page, most = case["seqs"], case["heads"], case["dim"], case["page"], max(news(case))
    p = torch.arange(case["context"], device=DEV)
    row = state["table"].long()[:, p // page].clamp(min=0) * page + p % page
    k, v = plain_values(state, "k", row), plain_values(state, "v", row)
    q = torch.zeros(seqs * most, case["q_heads"], dim, device=DEV)
    q[state["padded"]] = state["q"].float()
    q = q.view(seqs, most, heads, -1, dim)
    j = p - state["starts"][:, None]                                     # which node of the tree a token is, below 0: before it
    seen = (p < state["lens"][:, None])[:, None].expand(-1, most, -1)
    if state["tree"] is not None:
        bits = torch.zeros(seqs * most, 1, dtype=torch.int64, device=DEV)
        bits[state["padded"]] = state["tree"]
        seen = seen & ((j < 0)[:, None] | ((bits.view(seqs, most, 1) >> j.clamp(0, 63)[:, None] & 1) == 1))
    s = torch.einsum("bnhgd,bphd->bhgnp", q, k) * dim ** -0.5
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    e = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.einsum("bhgnp,bphd->bnhgd", e / e.sum(-1, keepdim=True), v)
    return o.reshape(seqs * most, -1, dim)[state["padded"]].to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if not own:
        return {"norm": plain_norm, "append": plain_append, "attend": plain_attend}[state["op"]](state)
    import paper_2606_14598_b200 as w8
    if state["op"] == "norm":
        x = state["x"]
        if "sum" not in state:
            state["sum"] = torch.empty_like(x, memory_format=torch.contiguous_format) if state["residual"] is not None else None
            state["y"] = torch.empty(x.shape, dtype=torch.bfloat16, device=DEV)
            state["qa"] = torch.empty(x.shape, dtype=torch.int8, device=DEV)
            state["s_tok"] = torch.empty(x.shape[0], device=DEV)
        if state["case"]["out"] == "bf16":
            y, h = w8.rmsnorm(x, state["weight"], EPS, residual=state["residual"], sum_out=state["sum"], out=state["y"])
            return h, y
        qa, s_tok, h = w8.int8_rmsnorm(x, state["weight"], EPS, residual=state["residual"], sum_out=state["sum"], qa=state["qa"], s_tok=state["s_tok"])
        return h, torch.mul(qa, s_tok[:, None], out=state["y"])          # (the values that the codes stand for)
    if "cache" not in state:
        state["cache"] = w8.QuantKVCache(state["k_codes"], state["k_scales"], state["v_codes"], state["v_scales"])
        state["out"] = torch.empty(state["q"].shape, dtype=torch.bfloat16, device=DEV)
        if state["op"] == "append":
            state["k_out"], state["v_out"] = (torch.empty(state["k"].shape, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        else:
            state["ws"] = w8.kv_cache_attention_workspace(state["cache"], state["case"]["seqs"], state["total"], state["case"]["q_heads"])
    if state["op"] == "append":
        q = w8.kv_cache_append(state["cache"], state["k"], state["v"], state["slots"], state["positions"], state["cos_sin"], axes=state["axes"],
                               interleaved=state["case"]["interleaved"], q=state["q"], q_out=state["out"])
        return (q, *w8.kv_cache_read(state["cache"], state["table"], state["cu"], state["total"], starts=state["starts"], k_out=state["k_out"], v_out=state["v_out"]))
    return w8.kv_cache_attention(state["cache"], state["q"], state["table"], state["lens"], state["cu"], tree=state["tree"], out=state["out"], workspace=state["ws"])


def work(case):
    if case["op"] == "norm":
        return {"bytes": case["m"] * case["k"] * (2 + 4 * case["residual"] + (1 if case["out"] == "int8" else 2)) + 4 * case["k"], "flops": 0}
    dim, heads, q_heads = case["dim"], case["heads"], case["q_heads"]
    kept = dim + 4 if case["fmt"] == "int8" else dim // 2 + (dim + 31) // 32
    if case["op"] == "append":
        tokens = case["seqs"] * case["new"]
        return {"bytes": tokens * (q_heads * 4 * dim + 2 * heads * (2 * dim + kept + 2 * dim) + 4 * case["rot"]), "flops": 0}
    lens, counts = lengths(case), news(case)
    return {"bytes": 2 * heads * kept * sum(lens) + 4 * q_heads * dim * sum(counts), "flops": 4 * q_heads * dim * sum(a * b for a, b in zip(lens, counts))}


# ------------------------------------------------------------------------------------------------ 64 bits

def single(x):
    """Rounded once to fp32, for the steps that are fp32 by definition."""
    return x.float().double()


def exact_int8(x):
    """The values of a row's int8 form; the scale and the quotient are fp32 by definition."""
    top = x.abs().amax(-1, keepdim=True)
    s = torch.where(top > 0, single(top / 127.0), 1.0)
    return torch.round(single(x / s)).clamp(-127, 127), s


def two_to(exponent):
    """2 ** exponent in 64 bits, from the bits of the number."""
    return ((exponent + 1023) << 52).view(torch.float64)


def exact_mxfp4(x):
    """The values that a matrix's MXFP4 form stands for, in 64 bits."""
    k = x.shape[-1]
    block = torch.arange(k, device=x.device) // BLOCK
    top = torch.zeros(*x.shape[:-1], (k + BLOCK - 1) // BLOCK, dtype=torch.float64, device=x.device)
    top = top.scatter_reduce(-1, block.expand(x.shape), x.abs(), "amax")
    exponent = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(min=-127)
    scale = two_to(exponent.long())[..., block]
    y = x.abs() / scale
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    return torch.sign(x) * (torch.round(y / step) * step).clamp(max=6.0) * scale


def exact_codes(state, which, b, n):
    """The values of the first n cached tokens of sequence b, [n, heads, dim]."""
    page = state["case"]["page"]
    pages = state["table"][b, : (n + page - 1) // page].long()
    codes, scales = state[which + "_codes"][pages].flatten(0, 1)[:n], state[which + "_scales"][pages].flatten(0, 1)[:n]
    if state["case"]["fmt"] == "int8":
        return codes.double() * scales.double()[..., None]
    code = torch.stack((codes.long() % 16, codes.long() // 16), -1).flatten(-2)
    up, half = code % 8 // 2, code % 2
    mag = torch.where(up == 0, half * 0.5, (1 + half * 0.5) * two_to(up - 1))
    return mag * (1.0 - 2.0 * (code >= 8)) * two_to(scales.long() - 127)[..., torch.arange(code.shape[-1], device=DEV) // BLOCK]


def exact_turn(case, state, x):
    """Rotation of [tokens, heads, dim] pair by pair; products and sums are fp32 by definition, as keys are quantized from them."""
    pairs, out = case["rot"] // 2, x.double().clone()
    axis = axis_of_pair(case)
    for i in range(pairs):
        one, two = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + pairs)
        where = state["positions"][axis[i]] if case["axes"] > 1 else state["positions"]
        c, s = (state["cos_sin"][where, i + n * pairs].double()[:, None] for n in (0, 1))
        a, b = x[..., one].double(), x[..., two].double()
        out[..., one] = single(single(a * c) - single(b * s))
        out[..., two] = single(single(b * c) + single(a * s))
    return out


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm":
        h = state["x"].double()
        if case["residual"]:
            h = single(h + state["residual"].double()).float().to(torch.bfloat16).double()   # bf16 by definition
        u = single(h * state["weight"].double())
        r = 1.0 / torch.sqrt((h * h).sum(-1, keepdim=True) / case["k"] + EPS)
        if case["out"] == "bf16":
            return h, u * r
        q, s = exact_int8(u)
        return h, q * s * r
    if case["op"] == "append":
        q, k, v = exact_turn(case, state, state["q"]), exact_turn(case, state, state["k"]), state["v"].double()
        if case["fmt"] == "mxfp4":
            return q, exact_mxfp4(k), exact_mxfp4(v)
        return q, *(a * b for a, b in (exact_int8(k), exact_int8(v)))
    out, first, heads = [], 0, case["heads"]
    for b, (n, new) in enumerate(zip(lengths(case), news(case))):
        k, v = exact_codes(state, "k", b, n), exact_codes(state, "v", b, n)
        q = state["q"][first:first + new].double().view(new, heads, -1, case["dim"])
        s = torch.einsum("nhgd,phd->nhgp", q, k) / math.sqrt(case["dim"])
        if state["tree"] is not None:
            word = state["tree"][first:first + new, 0]
            seen = torch.stack([(word & (1 << j if j < 63 else -(1 << 63))) != 0 for j in range(new)], -1)
            s[..., n - new:][~seen[:, None, None].expand(-1, *s.shape[1:3], -1)] = -math.inf
        out.append(torch.einsum("nhgp,phd->nhgd", s.softmax(-1), v).reshape(new, -1, case["dim"]))
        first += new
    return torch.cat(out)
