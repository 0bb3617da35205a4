"""Plain 64-bit forms of the MXFP4 format and of the int8 head quantizer, for the tests. Independent of the package."""
import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def mx_quantize(x):
    """x [..., K] (any K) -> (codes int64 [..., K], scale bytes int64 [..., ceil(K / 32)])."""
    x = x.double()
    k, blocks = x.shape[-1], (x.shape[-1] + 31) // 32
    pad = torch.zeros(*x.shape[:-1], blocks * 32 - k, dtype=torch.float64, device=x.device)
    b = torch.cat([x, pad], -1).view(*x.shape[:-1], blocks, 32)
    bad = ~torch.isfinite(b).all(-1)
    b = torch.where(bad[..., None], torch.zeros_like(b), b)
    amax = b.abs().amax(-1)
    e = torch.where(amax > 0, (torch.frexp(amax)[1].long() - 3).clamp(min=-127), torch.full_like(amax, -127).long())
    y = b.abs() / two_to(e)[..., None]
    dist = (y[..., None] - GRID.to(x.device)).abs()
    near = dist == dist.amin(-1, keepdim=True)
    even = torch.arange(8, device=x.device) % 2 == 0
    code = torch.where((near & even).any(-1), (near & even).int().argmax(-1), near.int().argmax(-1))
    code = code + 8 * (torch.signbit(b) & ~bad[..., None])
    return code.view(*x.shape[:-1], blocks * 32)[..., :k], torch.where(bad, torch.full_like(e, 255), e + 127)


def mx_values(codes, scale_bytes):
    """Integer codes [..., K] and scale bytes [..., ceil(K / 32)] -> float64 values."""
    mag = GRID.to(codes.device)[codes % 8] * (1 - 2 * (codes >= 8).double())
    s = torch.where(scale_bytes == 255, torch.full(scale_bytes.shape, float("nan"), dtype=torch.float64, device=codes.device),
                    two_to(scale_bytes - 127))
    return mag * s.repeat_interleave(32, -1)[..., : codes.shape[-1]]


def pack(codes):
    return (codes[..., 0::2] + 16 * codes[..., 1::2]).to(torch.uint8)


def unpack(packed):
    p = packed.long()
    return torch.stack([p % 16, p // 16], -1).flatten(-2)


def tile(rows):
    """Row-major scale bytes [M, K / 32] -> tiles [ceil(M / 128), ceil(K / 128), 512], entry by entry."""
    m, kb = rows.shape
    out = torch.zeros((m + 127) // 128, (kb + 3) // 4, 512, dtype=torch.uint8, device=rows.device)
    r, c = torch.meshgrid(torch.arange(m, device=rows.device), torch.arange(kb, device=rows.device), indexing="ij")
    out[r // 128, c // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + c % 4] = rows.to(torch.uint8)
    return out


def int8_quantize(x):
    """x [..., D] -> (codes int64, scales float64 holding fp32 numbers): scale and quotient are fp32 by definition."""
    x = x.double()
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    amax = x.abs().amax(-1)
    s = torch.where(amax > 0, (amax / 127).float().double(), torch.ones_like(amax))
    q = torch.round((x / s[..., None]).float().double()).clamp(-127, 127).long()
    return q, torch.where(bad, torch.full_like(s, float("nan")), s)


def same_values(got, want):
    """Equal numbers (NaN equal to NaN) after rounding `want` once to got's type."""
    want = want.to(got.dtype)
    return bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())
