"""The paged 4-bit cache in plain form, 64 bits and loops, for the tests: the format, the allocator, the attention."""
from __future__ import annotations

import math

import torch

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def quantise_block(x):
    """(scale byte, 32 codes) of 32 Python floats, by the definition."""
    if not all(math.isfinite(v) for v in x):
        return 255, [0] * 32
    most = max(abs(v) for v in x)
    e = -100
    while e < 125 and most >= 7.0 * 2.0 ** e:      # the least power of two that the largest magnitude is below 7 times of
        e += 1
    codes = []
    for v in x:
        off = [abs(abs(v) / 2.0 ** e - g) for g in GRID]
        best = min(range(8), key=lambda c: (off[c], c % 2))
        codes.append(best + (8 if math.copysign(1.0, v) < 0 else 0))
    return e + 127, codes


def quantise(x):
    """Codes [.., d / 2] and scales [.., d / 32] of rows [.., d] (any floating type), in 64 bits, all blocks at once."""
    b = x.double().unflatten(-1, (-1, 32))
    finite = torch.isfinite(b).all(-1)
    most = torch.where(finite, b.abs().amax(-1), 0.0)
    powers = 2.0 ** torch.arange(-100, 126, dtype=torch.float64)
    e = torch.searchsorted(7.0 * powers, most.contiguous(), right=True).clamp(max=225)
    a = torch.where(finite[..., None], b.abs() / powers[e][..., None], 0.0)
    grid = torch.tensor(GRID, dtype=torch.float64)
    off = (a[..., None] - grid).abs()
    near = off.amin(-1, keepdim=True)
    even = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    code = even[(off == near)[..., even].int().argmax(-1)]                 # ties: an even code first
    code = torch.where(finite[..., None], code + 8 * torch.signbit(b), 0).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), torch.where(finite, e + 27, 255).to(torch.uint8)


def values(codes, scales):
    grid = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    power = torch.where(scales == 255, math.nan, 2.0 ** (scales.double() - 127))
    return grid[c.long()] * power.repeat_interleave(32, -1)


class Allocator:
    """laq_block_map with Python lists."""

    def __init__(self, n, n_blocks, width, block_rows, free):
        self.rows, self.table, self.free = [0] * n, [[-1] * width for _ in range(n)], list(free)
        self.width, self.br, self.n_blocks, self.refused = width, block_rows, n_blocks, 0

    def step(self, add, n_slots):
        br, n = self.br, len(add)
        ceil = lambda r: -(-r // br)  # noqa: E731
        new = [max(r + a, 0) for r, a in zip(self.rows, add)]
        for i in reversed(range(n)):
            for b in reversed(range(ceil(new[i]), ceil(self.rows[i]))):
                self.free.append(self.table[i][b])
        there, asked, self.refused = len(self.free), 0, 0
        start, slots = [0], []
        for i in range(n):
            need = max(ceil(new[i]) - ceil(self.rows[i]), 0)
            wide = ceil(new[i]) > self.width
            asked += 0 if wide else need
            if wide or (need and asked > there):
                self.refused += 1
                slots += [-1] * max(add[i], 0)
            else:
                for b in range(ceil(self.rows[i]), ceil(self.rows[i]) + need):
                    self.table[i][b] = self.free.pop()
                slots += [self.table[i][r // br] * br + r % br for r in range(self.rows[i], new[i])]
                self.rows[i] = new[i]
            start.append(start[-1] + max(add[i], 0))
        return start, (slots + [-1] * n_slots)[:n_slots]


def attention(q, k, v, seen, scale):
    """One token: q [Hq, d], k, v [H, rows, d] in 64 bits, the first `seen` rows; rows that are nobody's are None-masked by the caller.
    Returns out, lse, and sum of p |v| and the largest sum of |q k| * scale, for the bounds."""
    Hq, d = q.shape
    H = k.shape[0]
    if seen <= 0:
        return torch.zeros(Hq, d, dtype=torch.float64), torch.full((Hq,), -math.inf, dtype=torch.float64), torch.zeros(Hq, d, dtype=torch.float64), torch.zeros(Hq)
    kk, vv = k[:, :seen].repeat_interleave(Hq // H, 0), v[:, :seen].repeat_interleave(Hq // H, 0)
    s = torch.einsum("hd,hrd->hr", q, kk) * scale
    p = torch.softmax(s, -1)
    return (torch.einsum("hr,hrd->hd", p, vv), torch.logsumexp(s, -1), torch.einsum("hr,hrd->hd", p, vv.abs()),
            (torch.einsum("hd,hrd->hr", q.abs(), kk.abs()) * scale).amax(-1))
