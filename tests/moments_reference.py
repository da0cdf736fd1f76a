"""AdamW and moments in 8 bits from their definitions, in 64 bits and on the CPU; nothing of the library is used."""
import math

import torch

BLOCK = 32


def mix(h):
    """32 bits of an int64 tensor"""
    h = h ^ (h >> 16)
    h = (h * 0xF704BB15) & 0xFFFFFFFF
    h = h ^ (h >> 15)
    h = (h * 0x371E2E67) & 0xFFFFFFFF
    return h ^ (h >> 16)


def random_bits(seed, step, number, place):
    """(for the first moment, for the second): 16 bits a value, for places int64"""
    one = lambda x: torch.tensor(x, dtype=torch.int64)   # noqa: E731
    key = mix(one(seed & 0xFFFFFFFF))
    for word in (seed >> 32, step & 0xFFFFFFFF, number):
        key = mix(one(word) ^ key)
    r = mix((place & 0xFFFFFFFF) ^ mix((place >> 32) ^ key))
    return r & 0xFFFF, r >> 16


def magnitudes(second):
    """the finite magnitudes of the codes in rising order: place = code"""
    first = -22 if second else -6
    t = [m / 8 * 2.0 ** first for m in range(8)]
    for e in range(first, 9):
        t += [(1 + m / 8) * 2.0 ** e for m in range(8)]
    return torch.tensor(t[:-1], dtype=torch.float64)   # the last one is NaN's


def values(codes, scales, second):
    """64-bit values of codes [n] and scale bytes [ceil(n / 32)]"""
    c = codes.reshape(-1).cpu().long()
    grid = torch.cat([magnitudes(second), torch.tensor([math.nan], dtype=torch.float64)])
    v = grid[c] if second else torch.where(c >= 128, -grid[c & 127], grid[c & 127])
    return v * torch.exp2(scales.cpu().double() - 127).repeat_interleave(BLOCK)[:c.numel()]


def block_exponents(x):
    """k of each block of 32"""
    mag = torch.where(torch.isfinite(x), x.abs(), 0.0).clamp(max=1.875 * 2.0 ** 127)
    n = x.numel()
    peak = torch.cat([mag, torch.zeros(-n % BLOCK, dtype=torch.float64)]).view(-1, BLOCK).amax(1)
    k = torch.full(peak.shape, -111, dtype=torch.int64)
    for _ in range(240):
        k += (peak > 448.0 * torch.exp2(k.double())).long()
    return k


def neighbours(x, second):
    """(code below, share of the way to the next code, exponents k) of the finite 64-bit values x"""
    k = block_exponents(x)
    q = x.abs().clamp(max=1.875 * 2.0 ** 127) / torch.exp2(k.double()).repeat_interleave(BLOCK)[:x.numel()]
    grid = magnitudes(second)
    low = (torch.searchsorted(grid, q, right=True) - 1).clamp(max=len(grid) - 2)
    return low, (q - grid[low]) / (grid[low + 1] - grid[low]), k


def codes_of(x, bits, second):
    """(codes, scale bytes) of the 64-bit values x, rounded by 16 random bits each"""
    good = torch.isfinite(x)
    low, share, k = neighbours(torch.where(good, x, 0.0), second)
    k = block_exponents(x)
    code = low + (torch.floor(share * 2.0 ** 20) + 16 * bits.double() + 8 >= 2.0 ** 20).long()
    if second:
        code = torch.where((x > 0) & (code < 1), 1, code)
    else:
        code = code + 128 * torch.signbit(x).long()
    return torch.where(good, code, 255 if second else 127).to(torch.uint8), (k + 127).to(torch.uint8)


def adamw(p, g, m, v, lr, step, betas, eps, decay, grad_scale=1.0):
    """(p, m, v) of float64 tensors, and how far the update of p, taken by parts, reaches"""
    g = g * grad_scale
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    away = lr / (1 - betas[0] ** step) * m / (torch.sqrt(v / (1 - betas[1] ** step)) + eps)
    return p - lr * decay * p - away, m, v
