"""Plain 64-bit forms of the 4-bit block-scaled operators, on the CPU."""
import torch

from tests.q8_util import up

E2M1 = torch.float4_e2m1fn_x2
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
HALF4 = 2.0 ** -2            # half a step of rounding, relative to a value of at least 0.5 steps' binade: 1 of 4 .. 6, 0.25 of 1
TINY4 = 2.0 ** -2            # and half the smallest step


def exponent4(amax):
    """Smallest e >= -126 with amax <= 6 2^e (0 for zeros), by search."""
    amax = amax.double()
    e = torch.full(amax.shape, -126, dtype=torch.int32)
    for _ in range(260):
        e = torch.where(amax > torch.ldexp(torch.full_like(amax, 6.0), e), e + 1, e)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def nearest4(v):
    """Codes (0 .. 7) of magnitudes: the nearest grid value, of two the even
    code; 6 for what lies above."""
    d = (v.abs()[..., None] - GRID).abs()
    best = d.amin(dim=-1, keepdim=True)
    code = torch.arange(8).expand(d.shape)
    even = torch.where((d == best) & (code % 2 == 0), code, 9).amin(dim=-1)
    any_ = torch.where(d == best, code, 9).amin(dim=-1)
    tie = (d == best).sum(dim=-1) > 1
    return torch.where(tie, even, any_)


def quantize4_ref(x):
    """x [batch, rows, cols] on the CPU -> (bytes as uint8, scales as uint8)."""
    b, rows, cols = x.shape
    nc = -(-cols // 32)
    p = torch.zeros(b, rows, nc * 32, dtype=torch.float64)
    p[:, :, :cols] = x.double()
    p = p.reshape(b, rows, nc, 32)
    bad = ~torch.isfinite(p).all(dim=3)
    e = exponent4(torch.where(bad[..., None], torch.zeros_like(p), p).abs().amax(dim=3))
    v = torch.where(bad[..., None], torch.zeros_like(p), torch.ldexp(p, -e[..., None]))
    code = nearest4(v) + 8 * torch.signbit(v).long()
    code = code.reshape(b, rows, nc * 16, 2)
    s = torch.full((b, rows, up(nc, 4)), 127, dtype=torch.uint8)
    s[:, :, :nc] = torch.where(bad, 255, e + 127).to(torch.uint8)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), s


def values4(v):
    """Bytes [..., n] as float64 [..., 2 n] on the CPU."""
    b = v.cpu().view(torch.uint8).long()
    grid = torch.cat([GRID, -GRID])
    return grid[torch.stack([b & 15, b >> 4], dim=-1)].reshape(*b.shape[:-1], -1)


def scales4(s, blocks):
    """Scale bytes [..., n] of `blocks` blocks as float64 factors of single
    values (255: NaN)."""
    b = s.cpu().view(torch.uint8)[..., :blocks]
    f = torch.ldexp(torch.ones(b.shape, dtype=torch.float64), b.int() - 127)
    return torch.where(b == 255, float("nan"), f).repeat_interleave(32, dim=-1)


def dequantize4(v, s):
    """(values, scales) of one matrix or a batch -> float64 on the CPU."""
    f = values4(v)
    return f * scales4(s, f.shape[-1] // 32)
