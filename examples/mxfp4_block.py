"""A text-to-image attention block in four bits, over a few sampling steps.

The image tokens go through MXFP4 linears (query / key / value projection, output projection, feed-forward). The prompt is the
same at every step: its keys and values are computed once, kept in a quantized paged cache, and read back at each step next to
the image's own. Two prompts of different lengths share the cache.

    python examples/mxfp4_block.py [--format int8|mxfp4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_14598_b200 as w8  # noqa: E402
from paper_2606_14598_b200.torch_op import MXFP4Linear  # noqa: E402


def attention(q, k, v):
    """[tokens, heads, dim] each; plain softmax attention in fp32."""
    s = torch.einsum("thd,shd->hts", q.float(), k.float()) * q.shape[-1] ** -0.5
    return torch.einsum("hts,shd->thd", s.softmax(-1), v.float()).to(torch.bfloat16)


def run(fmt: str = "int8", steps: int = 3, image: int = 300, prompts=(37, 61), heads: int = 6, dim: int = 64, seed: int = 0):
    """Returns (four-bit result, full-precision result) of the last step, fp32 [prompts, image, width]."""
    gen = torch.Generator("cuda").manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    width, page = heads * dim, 16
    weights = {name: rand(n, k) * k ** -0.5 for name, n, k in [("qkv", 3 * width, width), ("out", width, width),
                                                               ("up", 4 * width, width), ("down", width, 4 * width)]}
    layers = {name: MXFP4Linear.from_float(w) for name, w in weights.items()}
    plain = {name: (lambda w: lambda x: (x.float() @ w.t()))(w) for name, w in weights.items()}
    texts = [rand(n, width).to(torch.bfloat16) for n in prompts]
    noise = [rand(image, width).to(torch.bfloat16) for _ in prompts]

    # the prompts' keys and values, once: pages handed out in turn
    counts = [(n + page - 1) // page for n in prompts]
    cache = w8.QuantKVCache.empty(sum(counts), page, heads, dim, fmt)
    table = torch.full((len(prompts), max(counts)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(prompts):
        first = sum(counts[:b])
        table[b, : counts[b]] = torch.arange(first, first + counts[b], dtype=torch.int32)
        kv = layers["qkv"](texts[b]).view(n, 3, heads, dim)
        slots = table[b, : counts[b]].long().repeat_interleave(page)[:n] * page + torch.arange(n, device="cuda") % page
        w8.kv_cache_write(cache, kv[:, 1], kv[:, 2], slots)
    cu = torch.tensor([sum(prompts[:b]) for b in range(len(prompts) + 1)], dtype=torch.int32, device="cuda")

    def block(x, k_text, v_text, linear):
        q, k, v = linear["qkv"](x).to(torch.bfloat16).view(-1, 3, heads, dim).unbind(1)
        x = x + linear["out"](attention(q, torch.cat([k_text, k]), torch.cat([v_text, v])).reshape(-1, width)).to(torch.bfloat16)
        return x + linear["down"](torch.nn.functional.gelu(linear["up"](x).to(torch.bfloat16))).to(torch.bfloat16)

    four, full = list(noise), list(noise)
    for _ in range(steps):
        k_all, v_all = w8.kv_cache_read(cache, table, cu, sum(prompts))
        for b, n in enumerate(prompts):
            at = sum(prompts[:b])
            four[b] = block(four[b], k_all[at:at + n], v_all[at:at + n], layers)
            k, v = plain["qkv"](texts[b]).to(torch.bfloat16).view(n, 3, heads, dim)[:, 1:].unbind(1)
            full[b] = block(full[b], k, v, plain)
    return torch.stack(four).float(), torch.stack(full).float()


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--format", choices=("int8", "mxfp4"), default="int8")
    a, b = run(p.parse_args().format)
    cosine = torch.nn.functional.cosine_similarity(a.flatten(), b.flatten(), dim=0).item()
    print(f"four-bit block against fp32: cosine {cosine:.4f}, relative error {((a - b).norm() / b.norm()).item():.3f}")
