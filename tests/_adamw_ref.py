"""The AdamW step over many tensors as include/smat.h defines it, in numpy: `step` in fp32, one operation at a time (the same
bits), `step64` in 64 bits; the 8-bit form of moments from its definition."""

import math

import numpy as np

GROUP = 256
f32 = np.float32


def starts(sizes):
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // GROUP) * GROUP
    return out, at


def constants(step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01):
    """fl(...) of the definition"""
    return dict(b1=f32(beta1), omb1=f32(1 - beta1), b2=f32(beta2), omb2=f32(1 - beta2), eps=f32(eps),
                decay=f32(1 - lr * weight_decay), step=f32(lr / -math.expm1(step * math.log(beta1))),
                bc2=f32(math.sqrt(-math.expm1(step * math.log(beta2)))))


def step(p, g, m1, m2, c, scale=1.0):
    """(p, m1, m2, r) in fp32, p before it is rounded to its type"""
    with np.errstate(all="ignore"):
        g = g * f32(scale)
        m1 = c["b1"] * m1 + c["omb1"] * g
        m2 = c["b2"] * m2 + c["omb2"] * (g * g)
        r = np.sqrt(m2)
        p = p * c["decay"] - c["step"] * (m1 / (r / c["bc2"] + c["eps"]))
    for v in (p, m1, m2, r):
        assert v.dtype == np.float32
    return p, m1, m2, r


def mix(h):
    with np.errstate(over="ignore"):
        h = h ^ (h >> np.uint32(16))
        h = h * np.uint32(0x85EBCA6B)
        h = h ^ (h >> np.uint32(13))
        h = h * np.uint32(0xC2B2AE35)
        return h ^ (h >> np.uint32(16))


def numbers(places, t, seed):
    """The 32 bits of each place."""
    key = mix(mix(mix(np.array([seed & 0xFFFFFFFF], np.uint32)) ^ np.uint32(seed >> 32 & 0xFFFFFFFF)) ^ np.uint32(t & 0xFFFFFFFF))
    return mix(np.asarray(places, np.uint64).astype(np.uint32) ^ mix(key))


def codes(v, part, places, less):
    """(bytes, e) of fp32 values v >= 0, whole groups; part: 16 bits each."""
    v = v.reshape(-1, GROUP)
    part = part.reshape(-1, GROUP)
    bad = ~np.isfinite(v).all(1)
    v = np.where(bad[:, None], f32(0), v)
    e = np.maximum((v.max(1).view(np.uint32) >> 23).astype(np.int64) - less, 1)
    f = np.ldexp(v, (127 - e)[:, None].astype(np.int32)).astype(np.float32)
    one = 1 << places
    at = np.where(f >= one, np.frexp(f)[1] - 1 - places, 0)
    u = (part.astype(np.float64) + 0.5) / 65536  # 64 bits hold the sum exactly, but for values far below the unit, which it leaves
    whole = np.floor(np.ldexp(f, -at.astype(np.int32)).astype(np.float64) + u).astype(np.int64)
    q = np.where(bad[:, None], 0, at * one + whole).astype(np.uint8)
    return q.reshape(-1), np.where(bad, 255, e).astype(np.uint8)


def table(places):
    one = 1 << places
    return np.array([float(c) if c < one else (one + c % one) * 2.0 ** (c // one - 1) for c in range(16 * one)])


def values(q, e, places):
    """float64 values of codes (no sign bit); NaN where e = 255"""
    unit = np.where(e == 255, np.nan, np.ldexp(1.0, e.astype(np.int32) - 127))
    return table(places)[q] * np.repeat(unit, GROUP)


def pack(m1, r, t, seed, first=0):
    n = numbers(np.arange(first, first + m1.size), t, seed)
    q1, e1 = codes(np.abs(m1), n & np.uint32(0xFFFF), 3, 16)
    q1 = np.where(np.repeat(e1 == 255, GROUP), 0, q1 | np.where(np.signbit(m1), 128, 0)).astype(np.uint8)
    q2, e2 = codes(r, n >> np.uint32(16), 4, 17)
    return q1, e1, q2, e2


def unpack(q1, e1, q2, e2):
    v = values(q1 & 127, e1, 3)
    return np.where(q1 >= 128, -v, v), values(q2, e2, 4)
