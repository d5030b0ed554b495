"""The operators beside the codec in 64 bits, from their definitions, for the tests (no code of the library)."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # of one rounding (bf16: with room for a double one)
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
E32 = 2.0 ** -24


def norm(x, gamma, beta, eps):
    """-> y, mean, rstd in 64 bits."""
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    g = 1.0 if gamma is None else gamma.double()
    b = 0.0 if beta is None else beta.double()
    return (x - mean[:, None]) * rstd[:, None] * g + b, mean, rstd


def norm_grad(dy, x, gamma, mean, rstd):
    """-> dx, dgamma, dbeta in 64 bits, and the sums of magnitudes that bound their rounding."""
    x, dy = x.double(), dy.double()
    mean, rstd = mean.double()[:, None], rstd.double()[:, None]
    xhat = (x - mean) * rstd
    h = dy * (1.0 if gamma is None else gamma.double())
    m1, m2 = h.mean(1, keepdim=True), (h * xhat).mean(1, keepdim=True)
    dx = rstd * (h - m1 - xhat * m2)
    # xhat itself is off by a few roundings of (|x| + |mean|) rstd
    wide = (x.abs() + mean.abs()) * rstd
    size = rstd * (h.abs() + h.abs().mean(1, keepdim=True) + wide * (h.abs() * wide).mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0), size, (dy.abs() * wide).sum(0), dy.abs().sum(0)


LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def up(v, to):
    return -(-v // to) * to


def quantize(x, fmt, square):
    """-> codes (rows x cols rounded up to 16, uint8), exponents (rows x ceil(cols / 128)) of a CPU tensor, row by row."""
    bits, low = (3, -6) if fmt == "e4m3" else (2, -14)
    top = LARGEST[fmt]
    rows, cols = x.shape
    x = x.double()
    finite = torch.where(torch.isfinite(x), x.abs(), 0.0)
    blocks = -(-cols // 128)
    e = torch.zeros(rows, blocks, dtype=torch.int64)
    values = torch.zeros(rows, up(cols, 16), dtype=torch.float64)
    for b in range(blocks):
        part = finite[:, 128 * b:128 * b + 128]
        for r in range(rows):
            piece = part[r // 128 * 128:r // 128 * 128 + 128] if square else part[r]
            a = float(piece.max())
            if a > 0:
                k = math.frexp(a)[1] - math.frexp(top)[1] - 2
                while math.ldexp(a, -k) > top:
                    k += 1
                e[r, b] = max(-127, min(127, k))
        two = torch.ldexp(torch.ones(rows, dtype=torch.float64), -e[:, b])[:, None]
        t = x[:, 128 * b:128 * b + 128] * two
        exponent = torch.frexp(torch.where(torch.isfinite(t), t, 0.0))[1] - 1
        step = torch.ldexp(torch.ones_like(t), exponent.clamp(min=low) - bits)
        t = torch.where(torch.isfinite(t), torch.round(t / step) * step, float("nan"))
        values[:, 128 * b:128 * b + t.shape[1]] = t
    codes = values.float().to(FLOAT8[fmt]).view(torch.uint8)  # exact: the values are the format's
    return codes, e


def place(r, b, rows):
    """Byte of row r, block b in the scales of a matrix of `rows` rows."""
    return ((b // 4) * (up(rows, 128) // 128) + r // 128) * 512 + (r % 32) * 16 + (r // 32 % 4) * 4 + b % 4


def scale_bytes(e, rows, cols):
    """The scales as the library keeps them: 127 wherever there is no block."""
    out = torch.full((512 * (up(rows, 128) // 128) * (up(cols, 512) // 512),), 127, dtype=torch.uint8)
    r, b = torch.arange(e.shape[0])[:, None], torch.arange(e.shape[1])[None]
    out[place(r, b, rows)] = (e + 127).to(torch.uint8)
    return out


def decode(codes, scales, fmt, k):
    """The 64-bit values of a coded matrix (rows x k)."""
    rows = codes.shape[0]
    r, b = torch.arange(rows, device=codes.device)[:, None], torch.arange(-(-k // 128), device=codes.device)[None]
    e = scales[place(r, b, rows)].double() - 127
    v = codes[:, :k].contiguous().view(FLOAT8[fmt]).float().double()
    return v * torch.ldexp(torch.ones_like(e), e.int()).repeat_interleave(128, 1)[:, :k]
