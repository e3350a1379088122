"""Plain forms, in 64 bits, of rotary positions and of the paged cache in 32, 16 or 8 bits: what the library is tested against."""
import math

import torch

# the magnitudes of e4m3 in the order of their codes
GRID = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]


def quantise_row(row):
    """(scale byte, codes) of a list of numbers, by the format's definition."""
    if not all(math.isfinite(x) for x in row):
        return 255, [0] * len(row)
    most = max(abs(x) for x in row)
    e = -100
    while most > 448.0 * 2.0 ** e:
        e += 1
    codes = []
    for x in row:
        far = [abs(abs(x) / 2.0 ** e - g) for g in GRID]
        best = min(range(len(GRID)), key=lambda c: (far[c], c % 2))
        codes.append(best + (128 if math.copysign(1, x) < 0 else 0))
    return e + 127, codes


def quantise(x):
    """Codes [.., d] and scales [..] (uint8) of rows [.., d]: the same on tensors."""
    x = x.double()
    grid = torch.tensor(GRID, dtype=torch.float64)
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], 0.0, x)
    powers = torch.tensor([2.0 ** e for e in range(-100, 121)], dtype=torch.float64)
    at = torch.searchsorted(powers * 448.0, x.abs().amax(-1, keepdim=True))
    far = x.abs() / powers[at]
    up = torch.searchsorted(grid, far).clamp(1, len(GRID) - 1)
    low, high = far - grid[up - 1], grid[up] - far
    codes = torch.where((high < low) | ((high == low) & (up % 2 == 0)), up, up - 1) + 128 * torch.signbit(x)
    return torch.where(bad[..., None], 0, codes).to(torch.uint8), torch.where(bad, 255, at[..., 0] + 27).to(torch.uint8)


def values(codes, scales):
    """What rows of codes [.., d] and scales [..] stand for."""
    grid = torch.tensor(GRID + [math.nan], dtype=torch.float64)
    x = grid[(codes & 127).long()] * torch.where(codes >= 128, -1.0, 1.0).double()
    return x * torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))[..., None]


def held(x, kind):
    """What rows [.., d] are held as in a cache of type `kind`."""
    if kind == torch.float8_e4m3fn:
        return values(*quantise(x))
    return x.to(kind).double()


def rotate(x, positions, inv_freq, layout, mscale):
    """Heads [tokens, heads, d] rotated, and the sum of the magnitudes of the two products of each number (0 where it is not rotated)."""
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    for i, f in enumerate(inv_freq.double().tolist()):
        a, b = (i, i + inv_freq.numel()) if layout == "half" else (2 * i, 2 * i + 1)
        angle = [p * f for p in positions.tolist()]
        c = torch.tensor([math.cos(t) * mscale for t in angle], dtype=torch.float64)[:, None]
        s = torch.tensor([math.sin(t) * mscale for t in angle], dtype=torch.float64)[:, None]
        xa, xb = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
        size[..., a], size[..., b] = (xa * c).abs() + (xb * s).abs(), (xb * c).abs() + (xa * s).abs()
    return y, size


def rotation_error(y, size, dtype):
    """How far a rotated number may be off: sine and cosine, and each product, are rounded to fp32, and their sum (2^-24 each; and 2^-46 where these meet);
    bf16 rounds once more (2^-8).  Numbers that are not rotated are exact."""
    off = size * (2 * 2.0 ** -24 + 2.0 ** -46) + (y.abs() + size * 2.0 ** -22) * 2.0 ** -24
    if dtype == torch.bfloat16:
        off = off + (y.abs() + off) * 2.0 ** -8
    return torch.where(size > 0, off + 1e-44, 0.0)
