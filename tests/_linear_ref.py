"""The linear layers' operators from their definitions in 64 bits (numpy / torch float64 on the CPU), for the tests."""

import math

import torch

ACTS = ("none", "relu", "gelu", "gelu_tanh", "quick_gelu", "silu")
GROUP = 32


def act(name, h):
    if name == "relu":
        return torch.where(h > 0, h, torch.zeros_like(h))
    if name == "gelu":
        return h * 0.5 * torch.special.erfc(-h / math.sqrt(2.0))
    if name == "gelu_tanh":
        return h * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (h + 0.044715 * h ** 3))
    if name == "quick_gelu":
        return h * torch.sigmoid(1.702 * h)
    if name == "silu":
        return h * torch.sigmoid(h)
    return h


def slope(name, h):
    """act' by its formula."""
    if name == "none":
        return torch.ones_like(h)
    if name == "relu":
        return (h > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-h / math.sqrt(2.0)) + h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = 2.0 * math.sqrt(2.0 / math.pi)
        s = torch.sigmoid(c * (h + 0.044715 * h ** 3))
        return s + h * s * (1 - s) * c * (1 + 3 * 0.044715 * h * h)
    c = 1.702 if name == "quick_gelu" else 1.0
    s = torch.sigmoid(c * h)
    return s + c * h * s * (1 - s)


def pack(x):
    """(q, e) of a float64 matrix of finite values, from the definition: per row and 32 columns the smallest power
    of two from 2^-126 on with which every rounded quotient is at most 127."""
    x = x.double().cpu()
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    v = torch.zeros(rows, groups * GROUP, dtype=torch.float64)
    v[:, :cols] = x
    v = v.view(rows, groups, GROUP)
    top = v.abs().amax(-1)
    e = torch.full((rows, groups), 1, dtype=torch.int64)
    for _ in range(254):
        step = torch.ldexp(torch.ones_like(top), e - 127)
        big = torch.round(top / step) > 127
        if not bool(big.any()):
            break
        e += big
    q = torch.round(v / torch.ldexp(torch.ones_like(top), e - 127).unsqueeze(-1))
    return q.view(rows, groups * GROUP)[:, :cols].to(torch.int8), e.to(torch.uint8)


def unpack(q, e):
    q, e = q.cpu(), e.cpu().to(torch.int64)
    scale = torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e - 127)
    return q.double() * scale.repeat_interleave(GROUP, -1)[..., :q.shape[-1]]


def rounding(dtype):
    """The largest relative error of one rounding to the type: half a unit in the last place of 8 bits (bf16) or 24,
    next to a power of two (1 + 2^-8 lies in the middle of the bf16 numbers 1 and 1 + 2^-7)."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


def sum_error(a_abs, dtype, terms):
    """How far a sum of `terms` products may be off, a_abs being the sum of their magnitudes.

    fp32: one rounding per addition, at most 2^-24 of a partial sum; with probability above 1 - 1e-13 their
    random walk stays under 8 sqrt(terms) 2^-24 of the magnitudes' sum (Higham and Mary's probabilistic bound).
    bf16 on the matrix instructions: the products are exact, 16 of them enter the accumulator at a time and each
    entry may cut off up to one unit in the last place, 2^-23, in one direction; 32 more for joins of shares."""
    if dtype == torch.float32:
        return (8 * math.sqrt(max(terms, 1)) + 4) * 2.0 ** -24 * a_abs
    return (terms / 16 + 32) * 2.0 ** -23 * a_abs
