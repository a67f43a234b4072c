"""Rows kept in 8 bits and the experts' activation from their definitions, in float64 on the CPU."""
import math

import torch

U32 = 2.0**-24   # half an ulp of float32, relative
UBF = 2.0**-8    # of bf16
BLOCK = 32


def keep(x):
    """(codes int8 (R, 32 B), scales uint8 (R, B)), value by value as the definition has it."""
    R, C = x.shape
    B = -(-C // BLOCK)
    v = torch.zeros(R, B * BLOCK, dtype=torch.float64)
    v[:, :C] = x.double()
    v = v.view(R, B, BLOCK)
    finite = v.isfinite()
    top = torch.where(finite, v.abs(), 0.0).amax(-1)
    scales = torch.ones(R, B, dtype=torch.uint8)
    for b in range(2, 249):   # the smallest byte whose 127.5 2^(b - 127) holds the largest
        scales = torch.where(top > 127.5 * 2.0**(b - 1 - 127), b, scales)
    step = torch.exp2(scales.double() - 127)[..., None]
    q = torch.round(torch.where(finite, v, 0.0) / step).clamp(-127, 127)   # (torch rounds ties to even)
    return torch.where(finite, q, -128.0).to(torch.int8).view(R, -1), scales.to(torch.uint8)


def restore(codes, scales, cols):
    c = codes.double().view(*scales.shape, BLOCK)
    v = torch.where(c == -128, math.nan, c * torch.exp2(scales.double() - 127)[..., None])
    return v.reshape(codes.shape)[:, :cols]


def act(g, kind):
    """(f, f', y): y is what the exponential takes."""
    if kind == "relu":
        return torch.where(g <= 0, 0.0, g), torch.where(g > 0, 1.0, torch.where(g <= 0, 0.0, g)), torch.zeros_like(g)
    k2 = 2 * math.sqrt(2 / math.pi)
    y = g if kind == "silu" else k2 * (g + 0.044715 * g**3)
    s, s1 = torch.sigmoid(y), torch.sigmoid(-y)
    f = torch.where(g == -math.inf, 0.0, g * s)
    slope = 1.0 if kind == "silu" else k2 * (1 + 3 * 0.044715 * g * g)
    more = f * (s1 * slope)
    return f, s + torch.where((s1 == 0) | (s == 0), 0.0, more), y


def act_bound(g, kind):
    """What float32 may be off by: (of f, of f'). The argument y of the exponential is off by 6 half ulps of it (its square,
    cube, sum and constants), exp by 2 of its own, the sums, quotients and products around it by 12 more; f' has two
    such terms, which may cancel. An exponential below float32's smallest is off by less than 2^-126."""
    if kind == "relu":
        return torch.zeros_like(g), torch.zeros_like(g)
    f, _, y = act(g, kind)
    k2 = 2 * math.sqrt(2 / math.pi)
    slope = 1.0 if kind == "silu" else k2 * (1 + 3 * 0.044715 * g * g)
    h = (6 * y.abs().clamp(max=100) + 16) * U32
    s, s1 = torch.sigmoid(y), torch.sigmoid(-y)
    tiny = 2.0**-126
    return h * f.abs() + tiny * (1 + g.abs()), 2 * h * (s + f.abs() * s1 * slope) + tiny * (1 + (g * slope).abs())
