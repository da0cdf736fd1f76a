"""The training operators from their definitions, in 64 bits and one value after the other's formula;
nothing of the library is used.  Also matrices laid out to catch reads and writes outside them."""
import math

import torch

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def e4m3_magnitudes():
    t = [m / 8 * 2.0 ** -6 for m in range(8)]
    for e in range(1, 16):
        t += [(1 + m / 8) * 2.0 ** (e - 7) for m in range(8)]
    return t[:127]


def keep(x, fmt, dtype):
    """(codes, scale bytes) of the 64-bit values x that come in `dtype`; on the CPU"""
    x = x.double().cpu()
    top = 448.0 if fmt == "e4m3" else 127.0
    most = (1.875 if fmt == "e4m3" else 1.96875) * 2.0 ** (15 if dtype == torch.float16 else 127)
    grid = torch.tensor(e4m3_magnitudes() if fmt == "e4m3" else [float(i) for i in range(128)], dtype=torch.float64)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    codes, scales = torch.zeros(rows, cols, dtype=torch.uint8), torch.zeros(rows, blocks, dtype=torch.uint8)
    for b in range(blocks):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        good = torch.isfinite(part)
        mag = torch.where(good, part.abs(), 0.0).clamp(max=most)
        peak = mag.max(1).values
        k = torch.full((rows,), -111, dtype=torch.int64)
        for _ in range(240):
            k += (peak > top * torch.exp2(k.double())).long()
        scales[:, b] = (k + 127).to(torch.uint8)
        v = mag / torch.exp2(k.double())[:, None]
        # nearest, ties to the even code
        low = (torch.searchsorted(grid, v.contiguous(), right=True) - 1).clamp(max=len(grid) - 2)
        down, up = v - grid[low], grid[low + 1] - v
        code = torch.where((up < down) | ((up == down) & (low % 2 == 1)), low + 1, low)
        negative = torch.signbit(part)
        if fmt == "e4m3":
            c = torch.where(good, code + 128 * negative.long(), 127)
        else:
            c = torch.where(good, torch.where(negative, -code, code) % 256, 128)
        codes[:, b * BLOCK:(b + 1) * BLOCK] = c.to(torch.uint8)
    return codes, scales


def values(codes, scales, fmt):
    """64-bit values of a checkpoint, on the CPU"""
    codes, scales = codes.cpu().long(), scales.cpu()
    if fmt == "e4m3":
        table = torch.tensor(e4m3_magnitudes() + [math.nan], dtype=torch.float64)
        v = table[codes % 128] * torch.where(codes >= 128, -1.0, 1.0).double()
    else:
        signed = torch.where(codes > 127, codes - 256, codes)
        v = torch.where(signed == -128, math.nan, signed.double())
    return v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def same_codes(got, want):
    """equal but for the sign of a zero in int8, which has none, and of NaN"""
    return got.shape == want.shape and bool((got.cpu() == want).all())


def act(u, name):
    if name == "relu":
        return torch.where(u <= 0, 0.0, u)
    if name == "gelu":
        return u * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3))
    if name == "silu":
        return u * torch.sigmoid(u)
    return u


def slope(u, name):
    if name == "none":
        return torch.ones_like(u)
    if name == "relu":
        return torch.where(u <= 0, 0.0, torch.where(u > 0, 1.0, math.nan)).double()
    if name == "silu":
        s = torch.sigmoid(u)
        return s + u * s * torch.sigmoid(-u)
    c = 2 * math.sqrt(2 / math.pi)
    z = c * (u + 0.044715 * u ** 3)
    s = torch.sigmoid(z)
    return s + u * s * torch.sigmoid(-z) * c * (1 + 3 * 0.044715 * u ** 2)


def norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + eps)
    return d * rstd[:, None] * gamma.double() + beta.double(), mean, rstd


def norm_grad(dy, x, gamma, mean, rstd, residual=None):
    dy, x, gamma, mean, rstd = (t.double() for t in (dy, x, gamma, mean, rstd))
    h = (x - mean[:, None]) * rstd[:, None]
    p = dy * gamma
    dx = rstd[:, None] * (p - p.mean(1, keepdim=True) - h * (p * h).mean(1, keepdim=True))
    if residual is not None:
        dx = dx + residual.double()
    return dx, (dy * h).sum(0), dy.sum(0)


class Framed:
    """A matrix inside a larger one that is filled with NaN (bytes: 0x7F, NaN in e4m3 and a scale of
    1): what is read outside it shows, and what is written outside it is found."""

    def __init__(self, rows, cols, dtype, lead=0, pad=0, device="cuda"):
        self.rows, self.cols, self.lead = rows, cols, lead
        self.stride = cols + pad
        fill = 0x7F if dtype == torch.uint8 else math.nan
        self.whole = torch.full((lead + (rows + 2) * self.stride + 64,), fill, dtype=dtype, device=device)
        self.start = lead + self.stride
        self.inner = torch.as_strided(self.whole, (rows, cols), (self.stride, 1), self.start)

    def of(self, x):
        self.inner.copy_(x)
        return self.inner

    def intact(self):
        """nothing but the matrix has changed"""
        out = self.whole.clone()
        torch.as_strided(out, (self.rows, self.cols), (self.stride, 1), self.start).fill_(0x7F if out.dtype == torch.uint8 else math.nan)
        return bool((out == 0x7F).all()) if out.dtype == torch.uint8 else bool(out.isnan().all())
