"""Plain definition, in 64 bits on the CPU, of tensors in 4 bits with a scale byte
for every 32 values of a row."""
import math

import torch

SIZES = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def blocks(Nc):
    return -(-Nc // 32)


def unit(scales):
    """What the scale bytes stand for."""
    return torch.where(scales == 255, torch.tensor(math.nan, dtype=torch.float64),
                       torch.ldexp(torch.ones(scales.shape, dtype=torch.float64), scales.int() - 127))


def values(codes, scales, Nc):
    """Values [.., Nc] of codes [.., 16 Nb] and scales [.., Nb]."""
    c = torch.stack([codes & 15, codes >> 4], -1).long().reshape(*scales.shape, 32)
    v = SIZES[c & 7] * (1 - 2 * (c >> 3)).double() * unit(scales)[..., None]
    return v.reshape(*scales.shape[:-1], -1)[..., :Nc]


def pack(codes):
    """Codes [.., n], one a value, to whole blocks of two a byte."""
    n = codes.shape[-1]
    c = torch.zeros((*codes.shape[:-1], 32 * blocks(n)), dtype=torch.uint8)
    c[..., :n] = codes
    return c[..., ::2] | c[..., 1::2] << 4


def quantize(x, rule):
    """Codes (one a value, of whole blocks) and scales of x [.., Nc]."""
    Nc = x.shape[-1]
    y = torch.zeros((*x.shape[:-1], 32 * blocks(Nc)), dtype=torch.float64)
    y[..., :Nc] = x.double()
    y = y.reshape(*x.shape[:-1], -1, 32)
    top = y.abs().amax(-1)
    bad = ~torch.isfinite(y).all(-1)
    top = torch.where(bad, torch.zeros_like(top), top)
    mantissa, e = torch.frexp(top)  # top = mantissa 2^e, mantissa in [1/2, 1)
    e = e - 3
    if rule == "up":
        e = e + (mantissa > 0.75).int()
    e = torch.where(top == 0, torch.full_like(e, -127), e.clamp_min(-127))
    a = torch.ldexp(y.abs(), -e[..., None])
    away = (a[..., None] - SIZES).abs()
    near = away == away.amin(-1, keepdim=True)  # two of them at a tie
    low = near.int().argmax(-1)
    high = 7 - near.flip(-1).int().argmax(-1)
    code = torch.where(low % 2 == 0, low, high) + 8 * torch.signbit(y).long()
    code = torch.where(bad[..., None], torch.zeros_like(code), code)
    scales = torch.where(bad, torch.full_like(e, 255), e + 127).byte()
    return code.byte().reshape(*x.shape[:-1], -1), scales


def random(gen, *lead, Nc, low=126, high=129):
    """Codes and scales of random values, scale bytes in [low, high)."""
    codes = pack(torch.randint(0, 16, (*lead, Nc), generator=gen).byte())
    return codes, torch.randint(low, high, (*lead, blocks(Nc)), generator=gen).byte()
