"""The operators of a residual stage in 64 bits, from their definitions, for the tests (no code of the library)."""
import math
import struct

import torch

from tests.operators_plain import E32, place, up

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LOW = 0xFFFFFFFF


def single(v):
    return struct.unpack("f", struct.pack("f", v))[0]


def mixed(h):
    """The 32-bit finaliser of MurmurHash3, on words held in 64 bits."""
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & LOW
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & LOW
    return h ^ (h >> 16)


def draws(rows, cols, seed, offset, device="cuda"):
    """The 24-bit numbers r (U = r 2^-24) of a rows x cols matrix; counters wrap at 2^64."""
    offset = offset % (1 << 64)
    offset = offset - (1 << 64) if offset >> 63 else offset
    ctr = (torch.arange(rows * cols, device=device) + offset).view(rows, cols)
    quad = (ctr >> 2) & ((1 << 62) - 1)
    key = mixed((quad >> 32) ^ (seed & LOW) ^ 0x9E3779B9) ^ (seed >> 32 & LOW)
    h = mixed((quad & LOW) ^ key)
    lane = torch.tensor([1, 0x9E3779B1, 0x85EBCA77, 0xC2B2AE3D], device=device)[ctr & 3]
    return (h * lane & LOW) >> 8


def kept(rows, cols, p, seed, offset, device="cuda"):
    return draws(rows, cols, seed, offset, device) >= math.ceil(single(p) * 2 ** 24)


def dropped32(x, p, seed, offset):
    """x / (1 - p) where kept, else 0, in the fp32 operations that the definition names (one product)."""
    if p == 0:
        return x.float()
    scale = single(1 / (1 - single(p))) if single(p) < 1 else 0.0
    return torch.where(kept(*x.shape, p, seed, offset, x.device), x.float() * scale, 0.0)


def rms(s, gamma, eps):
    """-> y, rstd in 64 bits."""
    s = s.double()
    rstd = 1 / torch.sqrt(s.square().mean(1) + eps)
    return s * rstd[:, None] * (1.0 if gamma is None else gamma.double()), rstd


def rms_grad(dy, s, gamma, rstd, dsum):
    """-> dx, dgamma in 64 bits, and the magnitudes that bound their rounding."""
    dy, xhat = dy.double(), s.double() * rstd.double()[:, None]
    h = dy * (1.0 if gamma is None else gamma.double())
    rstd = rstd.double()[:, None]
    dx = rstd * (h - xhat * (h * xhat).mean(1, keepdim=True))
    size = rstd * (h.abs() + xhat.abs() * (h * xhat).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, size = dx + dsum.double(), size + dsum.double().abs()
    return dx, (dy * xhat).sum(0), size, (dy * xhat).abs().sum(0)


def code4(x, square, r=None):
    """-> codes (rows x cols, 0 to 15), scale bytes (rows x blocks) along the rows of x; r: 24-bit numbers for stochastic rounding."""
    x = x.double()
    rows, cols = x.shape
    blocks = -(-cols // 32)
    wide = torch.zeros(up(rows, 32), blocks * 32, dtype=torch.float64, device=x.device)
    wide[:rows, :cols] = x
    most = wide.abs().view(wide.shape[0], blocks, 32)
    bad = ~torch.isfinite(most).all(2)
    most = torch.where(torch.isfinite(most), most, 0.0).amax(2)
    if square:
        most = most.view(-1, 32, blocks).amax(1).repeat_interleave(32, 0)
        bad = bad.view(-1, 32, blocks).any(1).repeat_interleave(32, 0)
    most, bad = most[:rows], bad[:rows]
    mantissa, exponent = torch.frexp(most)                      # most = mantissa 2^exponent, 6 = 0.75 * 2^3
    e = torch.where(most > 0, (exponent - 3 + (mantissa > 0.75).int()).clamp(min=-127), 0)
    two = torch.ldexp(torch.ones_like(most), e).repeat_interleave(32, 1)[:, :cols]
    t = torch.where(bad.repeat_interleave(32, 1)[:, :cols], 0.0, x.abs() / two)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    below = (torch.searchsorted(grid, t.contiguous(), right=True) - 1).clamp(max=6)
    share = (t - grid[below]) / (grid[below + 1] - grid[below])
    if r is None:
        above = (share > 0.5) | ((share == 0.5) & (below % 2 == 1))
    else:
        above = r.double() * 2.0 ** -24 < share
    codes = below + above.long()
    codes = codes + 8 * torch.signbit(x).long()
    codes = torch.where(bad.repeat_interleave(32, 1)[:, :cols], 0, codes)
    return codes, torch.where(bad, 255, e.long() + 127)


def packed4(codes):
    """Two to a byte, rows of a multiple of 32 codes."""
    rows, cols = codes.shape
    wide = torch.zeros(rows, up(cols, 32), dtype=torch.int64, device=codes.device)
    wide[:, :cols] = codes
    return (wide[:, 0::2] | wide[:, 1::2] << 4).to(torch.uint8)


def scales4(byte, rows, cols):
    """The scales as the library keeps them: 127 wherever there is no block."""
    out = torch.full((512 * (up(rows, 128) // 128) * (up(cols, 128) // 128),), 127, dtype=torch.uint8, device=byte.device)
    r, b = torch.arange(byte.shape[0], device=byte.device)[:, None], torch.arange(byte.shape[1], device=byte.device)[None]
    out[place(r, b, rows)] = byte.to(torch.uint8)
    return out


def values4(codes, byte, cols):
    """The 64-bit values of codes (rows x cols, 0 to 15) and scale bytes."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device=codes.device)
    two = torch.where(byte == 255, float("nan"), torch.ldexp(torch.ones_like(byte, dtype=torch.float64), byte.int() - 127))
    return grid[codes] * two.repeat_interleave(32, 1)[:, :cols]


def decode4(q, scales, cols):
    """The 64-bit values of a coded matrix as the library keeps it."""
    rows = q.shape[0]
    codes = torch.stack([q & 15, q >> 4], 2).view(rows, -1)[:, :cols].long()
    r, b = torch.arange(rows, device=q.device)[:, None], torch.arange(-(-cols // 32), device=q.device)[None]
    return values4(codes, scales[place(r, b, rows)].long(), cols)


__all__ = ["E32", "code4", "decode4", "draws", "dropped32", "kept", "packed4", "place", "rms", "rms_grad", "scales4", "single", "up", "values4"]
