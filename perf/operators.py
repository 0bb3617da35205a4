"""Workloads of the 4-bit and cached operators: what a user's program calls, in plain form and through the package.

Three kinds of pass, each over the sizes that a diffusion transformer or a token-by-token decoder gives it:

* ``linear``    out = bf16(values(quantize(A)) @ values(W)^T + bias): activations quantized to MXFP4 on the fly,
                weights kept in MXFP4 (blocks of 32 along K, one power-of-two scale a block).
* ``quantize``  a matrix to MXFP4 and back to the values it stands for.
* ``cache``     new tokens' keys and values quantized into a paged cache (int8 with a scale a head, or MXFP4), then the
                sequences read back through their page tables.

``own`` is false for the plain torch forms and true for the package's kernels. The scales of an MXFP4 matrix are kept
in tiles of 128 rows x 4 blocks (512 bytes: row r, block c at 16 * (r % 32) + 4 * (r // 32) + c), tiles row by row.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32
# magnitudes of the eight E2M1 codes; bit 3 of a code is the sign
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one token through a square projection: what a decoder does per step; latency counts
        {"name": "linear_one_token", "op": "linear", "m": 1, "n": 4608, "k": 4608, "bias": True},
        # the adaLN modulation of a block: two conditioning vectors, six outputs a channel
        {"name": "linear_adaln", "op": "linear", "m": 2, "n": 27648, "k": 4608, "bias": True},
        # a short prompt through an odd-sized projection
        {"name": "linear_prompt", "op": "linear", "m": 77, "n": 2048, "k": 1056, "bias": True},
        # fused query / key / value projection at 1024 pixels: 4096 image tokens and a 14-token prompt
        {"name": "linear_qkv", "op": "linear", "m": 4110, "n": 13824, "k": 4608, "bias": False},
        # feed-forward down-projection of the same block
        {"name": "linear_ffn_down", "op": "linear", "m": 4110, "n": 4608, "k": 12288, "bias": True},
        # activations of a short prompt
        {"name": "quantize_prompt", "op": "quantize", "m": 77, "k": 4608, "dtype": "bf16", "pad": 0},
        # the hidden activations of a feed-forward layer, a slice of a wider buffer
        {"name": "quantize_hidden", "op": "quantize", "m": 4110, "k": 12288, "dtype": "bf16", "pad": 64},
        # a weight matrix at load time
        {"name": "quantize_weight", "op": "quantize", "m": 13824, "k": 4608, "dtype": "fp32", "pad": 0},
        # a prompt's keys and values, written once and read back at every sampling step
        {"name": "cache_prompt_int8", "op": "cache", "fmt": "int8", "seqs": 1, "new": 512, "context": 512, "heads": 36, "dim": 128, "page": 16},
        # a whole image's keys and values kept between sampling steps, odd head size
        {"name": "cache_image_mxfp4", "op": "cache", "fmt": "mxfp4", "seqs": 2, "new": 4110, "context": 4110, "heads": 16, "dim": 72, "page": 64},
        # one new token in each of 48 sequences of very different lengths
        {"name": "cache_step_int8", "op": "cache", "fmt": "int8", "seqs": 48, "new": 1, "context": 4000, "heads": 8, "dim": 128, "page": 16},
        # one new token in each of a few long sequences
        {"name": "cache_step_mxfp4", "op": "cache", "fmt": "mxfp4", "seqs": 12, "new": 1, "context": 30000, "heads": 8, "dim": 128, "page": 64},
    ]


def draw(rng):
    def spread(lo, hi, step=1):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))

    op = rng.choice(("linear", "linear", "quantize", "cache", "cache"))
    if op == "linear":
        n, k = spread(256, 27648, 8), spread(256, 12288, 32)
        most = 4110 * 13824 * 4608 // (n * k)
        return {"op": op, "m": spread(1, max(2, min(8192, most))), "n": n, "k": k, "bias": rng.random() < 0.7}
    if op == "quantize":
        k = spread(256, 12288, 32)
        dtype = rng.choice(("bf16", "bf16", "fp32"))
        return {"op": op, "m": spread(1, 13824 * 4608 // k), "k": k, "dtype": dtype, "pad": rng.choice((0, 64, 4608))}
    fmt = rng.choice(("int8", "mxfp4"))
    heads, dim = rng.choice((2, 5, 8, 16, 24, 36)), rng.choice((64, 72, 80, 96, 128, 256))
    page = rng.choice((16, 32, 64, 100))
    if rng.random() < 0.5:
        new = spread(16, 4200)
        return {"op": op, "fmt": fmt, "seqs": rng.randint(1, 2), "new": new, "context": new, "heads": heads, "dim": dim, "page": page}
    seqs = spread(1, 64)
    most = 12 * 30000 * 8 * 128 // (seqs * heads * dim)
    return {"op": op, "fmt": fmt, "seqs": seqs, "new": rng.choice((1, 1, 1, 4)), "context": spread(64, min(30000, most)), "heads": heads, "dim": dim, "page": page}


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
    least = max(case["new"], most // 4)
    return [most - (most - least) * (i * 29 % seqs) // seqs for i in range(seqs)]


def tile_scales(rows):
    """Row-major block scales [M, K / 32] in tiles of 128 rows x 4 blocks: [ceil(M / 128), ceil(K / 128), 512], zero filled."""
    m, kb = rows.shape
    mt, kt = (m + 127) // 128, (kb + 3) // 4
    full = torch.zeros(mt * 128, kt * 4, dtype=torch.uint8, device=rows.device)
    full[:m, :kb] = rows
    return full.view(mt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).reshape(mt, kt, 512).contiguous()


def untile_scales(tiles, m, kb):
    mt, kt, _ = tiles.shape
    return tiles.view(mt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(mt * 128, kt * 4)[:m, :kb]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    state = {"op": case["op"], "case": case}
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        state["A"] = activations(gen, m, k).to(torch.bfloat16)
        codes, rows = to_mxfp4(normal(gen, n, k) * 0.02)
        state["qw"], state["sw"] = codes, tile_scales(rows)
        state["bias"] = normal(gen, n) * 0.01 if case["bias"] else None
    elif case["op"] == "quantize":
        m, k = case["m"], case["k"]
        x = activations(gen, m, k + case["pad"]) if case["dtype"] == "bf16" else normal(gen, m, k + case["pad"]) * 0.02
        state["x"] = (x.to(torch.bfloat16) if case["dtype"] == "bf16" else x)[:, :k]
    else:
        seqs, new, heads, dim, page = case["seqs"], case["new"], case["heads"], case["dim"], case["page"]
        lens = torch.tensor(lengths(case), device=DEV)
        pages_of = (lens + page - 1) // page
        most, count = int(pages_of.max()), int(pages_of.sum()) + 3
        order = torch.randperm(count, generator=gen, device=DEV)
        first = torch.cumsum(pages_of, 0) - pages_of
        slot = torch.arange(most, device=DEV)
        table = torch.where(slot < pages_of[:, None], order[(first[:, None] + slot).clamp(max=count - 1)], -1)
        where = lens[:, None] - new + torch.arange(new, device=DEV)
        state["table"] = table.to(torch.int32)
        state["cu"] = torch.cat([lens.new_zeros(1), torch.cumsum(lens, 0)]).to(torch.int32)
        state["total"] = int(lens.sum())
        state["slots"] = (torch.gather(table, 1, where // page) * page + where % page).reshape(-1)
        # keys and values come out of a fused projection: [tokens, 3, heads, dim]
        qkv = activations(gen, seqs * new, 3 * heads * dim).to(torch.bfloat16).view(seqs * new, 3, heads, dim)
        state["qkv"], state["k"], state["v"] = qkv, qkv[:, 1], qkv[:, 2]
        for which in "kv":
            if case["fmt"] == "int8":
                codes = torch.randint(-127, 128, (count, page, heads, dim), generator=gen, device=DEV, dtype=torch.int8)
                scales = torch.rand(count, page, heads, generator=gen, device=DEV) * 0.03 + 0.01
            else:
                codes = torch.randint(0, 256, (count, page, heads, dim // 2), generator=gen, device=DEV, dtype=torch.uint8)
                scales = torch.randint(124, 129, (count, page, heads, (dim + 31) // 32), generator=gen, device=DEV, dtype=torch.uint8)
            state[which + "_codes"], state[which + "_scales"] = codes, scales
    return state


# ------------------------------------------------------------------------------------------------ plain forms

def to_mxfp4(x):
    """(packed codes [..., K / 2], scale bytes [..., ceil(K / 32)]): the largest magnitude of a block of 32 sets the scale
    2 ** (floor(log2(largest)) - 2), the elements are rounded to the nearest of the E2M1 values, ties to the even code."""
    k = x.shape[-1]
    blocks = (k + BLOCK - 1) // BLOCK
    x = x.float()
    if k % BLOCK:
        x = torch.cat([x, x.new_zeros(*x.shape[:-1], blocks * BLOCK - k)], dim=-1)
    x = x.view(*x.shape[:-1], blocks, BLOCK)
    biased = x.abs().amax(-1).view(torch.int32) >> 23
    scale = (biased - 2).clamp(min=0)
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


def power_of_two(scale_bytes):
    """2 ** (byte - 127) in fp32 (byte 0 is a subnormal number)."""
    e = scale_bytes.to(torch.int32)
    return torch.where(e == 0, torch.full_like(e, 1 << 22), e << 23).view(torch.float32)


def from_mxfp4(codes, scale_bytes):
    """The fp32 values that packed codes and row-major scale bytes stand for."""
    table = torch.tensor(MAGNITUDES + tuple(-v for v in MAGNITUDES), device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], dim=-1)
    code = code.view(*codes.shape[:-1], 2 * codes.shape[-1])
    k = code.shape[-1]
    return table[code.int()] * power_of_two(scale_bytes).repeat_interleave(BLOCK, dim=-1)[..., :k]


def plain_linear(state):
    a = from_mxfp4(*to_mxfp4(state["A"]))
    n, k = state["qw"].shape[0], a.shape[1]
    w = from_mxfp4(state["qw"], untile_scales(state["sw"], n, k // BLOCK))
    out = a @ w.t()
    return (out if state["bias"] is None else out + state["bias"]).to(torch.bfloat16)


def plain_quantize(state):
    x = state["x"]
    return from_mxfp4(*to_mxfp4(x)).to(x.dtype)


def plain_cache(state):
    case, slots = state["case"], state["slots"]
    page, t = case["page"], torch.arange(state["total"], device=DEV)
    seq = (t[:, None] >= state["cu"][None, 1:]).sum(1)
    at = t - state["cu"][seq]
    row = state["table"][seq, at // page].long() * page + at % page
    return plain_store(state, "k", slots, row), plain_store(state, "v", slots, row)


def plain_store(state, which, slots, row):
    codes, scales, x = state[which + "_codes"], state[which + "_scales"], state[which].float()
    if state["case"]["fmt"] == "int8":
        largest = x.abs().amax(-1)
        s = torch.where(largest > 0, largest / torch.full_like(largest, 127.0), torch.ones_like(largest))
        codes.flatten(0, 1)[slots] = torch.round(x / s[..., None]).clamp(-127, 127).to(torch.int8)
        scales.flatten(0, 1)[slots] = s
        return (codes.flatten(0, 1)[row].float() * scales.flatten(0, 1)[row][..., None]).to(torch.bfloat16)
    new_codes, new_scales = to_mxfp4(x)
    codes.flatten(0, 1)[slots] = new_codes
    scales.flatten(0, 1)[slots] = new_scales
    return from_mxfp4(codes.flatten(0, 1)[row], scales.flatten(0, 1)[row]).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if not own:
        return {"linear": plain_linear, "quantize": plain_quantize, "cache": plain_cache}[state["op"]](state)
    import paper_2606_14598_b200 as w8
    if state["op"] == "linear":
        if "ws" not in state:
            (m, k), n = state["A"].shape, state["qw"].shape[0]
            state["ws"] = w8.mxfp4_alloc_workspace(m, n, k, DEV)
            state["out"] = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
        return w8.mxfp4_linear_fused(state["A"], state["qw"], state["sw"], state["bias"], out=state["out"], workspace=state["ws"])
    if state["op"] == "quantize":
        codes, scales = w8.mxfp4_quantize(state["x"])
        return w8.mxfp4_dequantize(codes, scales, dtype=state["x"].dtype)
    if "cache" not in state:
        state["cache"] = w8.QuantKVCache(state["k_codes"], state["k_scales"], state["v_codes"], state["v_scales"])
    w8.kv_cache_write(state["cache"], state["k"], state["v"], state["slots"])
    return w8.kv_cache_read(state["cache"], state["table"], state["cu"], state["total"])


def work(case):
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * m * k + n * k / 2 + n * k / BLOCK + 4 * n * case["bias"] + 2 * m * n, "flops": 2 * m * n * k}
    if case["op"] == "quantize":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["m"] * case["k"] * (2 * size + 0.5 + 1 / BLOCK), "flops": 0}
    dim, heads = case["dim"], case["heads"]
    kept = dim + 4 if case["fmt"] == "int8" else dim // 2 + (dim + 31) // 32
    tokens = sum(lengths(case))
    return {"bytes": 2 * heads * (case["seqs"] * case["new"] * 2 * dim + tokens * (kept + 2 * dim)), "flops": 0}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "linear":
        n, k = case["n"], case["k"]
        tiles = state["sw"]
        r, c = torch.arange(n, device=DEV)[:, None], torch.arange(k // BLOCK, device=DEV)[None, :]
        e = tiles[r // 128, c // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + c % 4]
        out = exact_mxfp4(state["A"]) @ exact_values(state["qw"], e).t()
        return out if state["bias"] is None else out + state["bias"].double()
    if case["op"] == "quantize":
        return exact_mxfp4(state["x"])
    page, table, cu = case["page"], state["table"].long(), state["cu"].long()
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device=DEV), cu[1:] - cu[:-1])
    at = torch.arange(state["total"], device=DEV) - cu[seq]
    row = table[seq, torch.div(at, page, rounding_mode="floor")] * page + torch.remainder(at, page)
    fresh = torch.full((table.max().item() * page + page,), -1, device=DEV)
    fresh[state["slots"]] = torch.arange(state["slots"].numel(), device=DEV)
    out = []
    for which in "kv":
        if case["fmt"] == "int8":
            # the scale and the quotient are fp32 by definition: both are rounded once from 64 bits
            x = state[which].double()
            top = x.abs().amax(-1, keepdim=True)
            s = torch.where(top > 0, (top / 127.0).float().double(), 1.0)
            new = torch.round((x / s).float().double()).clamp(-127, 127) * s
            old = state[which + "_codes"].flatten(0, 1)[row].double() * state[which + "_scales"].flatten(0, 1)[row].double()[..., None]
        else:
            new = exact_mxfp4(state[which])
            old = exact_values(state[which + "_codes"].flatten(0, 1)[row], state[which + "_scales"].flatten(0, 1)[row])
        hit = fresh[row]
        old[hit >= 0] = new[hit[hit >= 0]]
        out.append(old)
    return tuple(out)


def two_to(exponent):
    """2 ** exponent in 64 bits, from the bits of the number."""
    return ((exponent + 1023) << 52).view(torch.float64)


def exact_values(codes, e):
    lo, hi = codes.long() % 16, codes.long() // 16
    code = torch.stack((lo, hi), -1).flatten(-2)
    exponent, fraction = code % 8 // 2, code % 2
    mag = torch.where(exponent == 0, fraction * 0.5, (1 + fraction * 0.5) * two_to(exponent - 1))
    sign = 1.0 - 2.0 * (code >= 8)
    block = torch.arange(code.shape[-1], device=code.device) // BLOCK
    return sign * mag * two_to(e.long() - 127)[..., block]


def exact_mxfp4(x):
    """The values that a matrix's MXFP4 form stands for, in 64 bits."""
    k = x.shape[-1]
    x = x.double()
    block = torch.arange(k, device=x.device) // BLOCK
    top = torch.zeros(*x.shape[:-1], (k + BLOCK - 1) // BLOCK, dtype=torch.float64, device=x.device)
    top = top.scatter_reduce(-1, block.expand(x.shape), x.abs(), "amax")
    exponent = (torch.frexp(top)[1] - 1 - 2).clamp(min=-127)
    exponent = torch.where(top > 0, exponent, torch.full_like(exponent, -127))
    scale = two_to(exponent.long())[..., block]
    y = x.abs() / scale
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    return torch.sign(x) * (torch.round(y / step) * step).clamp(max=6.0) * scale
