"""Plain 64-bit forms of the 8-bit block-scaled operators, on the CPU."""
import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
# half a step of rounding, relative to a normal value, and half the smallest step
HALF = {torch.float8_e4m3fn: 2.0 ** -4, torch.float8_e5m2: 2.0 ** -3}
TINY = {torch.float8_e4m3fn: 2.0 ** -10, torch.float8_e5m2: 2.0 ** -17}


def up(n, m):
    return -(-n // m) * m


def scale_exponent(amax, fmt):
    """Smallest e >= -126 with amax <= top 2^e (0 for zeros), by search."""
    amax = amax.double()
    e = torch.full(amax.shape, -126, dtype=torch.int32)
    for _ in range(260):
        e = torch.where(amax > torch.ldexp(torch.full_like(amax, TOP[fmt]), e), e + 1, e)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def quantize_ref(x, fmt, block_rows):
    """x [batch, rows, cols] on the CPU -> (bytes as uint8, scales as uint8)."""
    b, rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // 128)
    p = torch.zeros(b, nr * block_rows, nc * 128, dtype=torch.float64)
    p[:, :rows, :cols] = x.double()
    p = p.reshape(b, nr, block_rows, nc, 128)
    mag = torch.where(torch.isfinite(p), p.abs(), 0.0)
    e = scale_exponent(mag.amax(dim=(2, 4)), fmt)
    scaled = torch.ldexp(p, -e[:, :, None, :, None])
    # from float32: exact for float32 input down to far below the smallest
    # step, and torch rounds float32 to the formats to nearest even
    v = scaled.float().to(fmt).view(torch.uint8).reshape(b, nr * block_rows, nc * 128)
    s = torch.full((b, nr, up(nc, 4)), 127, dtype=torch.uint8)
    s[:, :, :nc] = (e + 127).to(torch.uint8)
    return v[:, :rows, :up(cols, 16)], s


def dequantize(v, s, block_rows):
    """(values, scales) of one matrix or a batch -> float64 on the CPU."""
    f = torch.ldexp(torch.ones(s.shape, dtype=torch.float64), s.cpu().view(torch.uint8).int() - 127)
    f = f.repeat_interleave(128, dim=-1)[..., :v.shape[-1]]
    if block_rows > 1:
        f = f.repeat_interleave(block_rows, dim=-2)[..., :v.shape[-2], :]
    return v.cpu().double() * f
