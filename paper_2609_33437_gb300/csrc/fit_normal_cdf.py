"""Fit the polynomial of the normal distribution function that fp32 linear layers use (smat_linear.cuh: normal_cdf).

With a = |h| and t = 1 / (1 + P a), Phi(-a) = exp(-a^2 / 2) t Q(t). Q's degree is 8, its relative error the least in the
largest sense over 0 <= a <= 13.4 (Phi is below 2^-130 there): weighted least squares in Chebyshev polynomials of t, the
weights multiplied by the errors again and again (Lawson's algorithm). The targets are scipy's log_ndtr plus a^2 / 2 in 64
bits. P = 0.35 has the least error of the fp32 evaluation among the multiples of 0.05 from 0.15 to 0.6; degree 7 has 7.0
half units in the last place, 8 has 4.9, 9 has 4.8.

Run: python fit_normal_cdf.py     (prints the coefficients and the errors of the fit and of its fp32 evaluation)
"""

import numpy as np
from scipy.special import log_ndtr

P, DEGREE, A_MAX = 0.35, 8, 13.4


def target(a):
    """Phi(-a) exp(a^2 / 2)"""
    return np.exp(log_ndtr(-a) + a * a / 2)


def fit(nodes=20000, rounds=200):
    """(largest relative error, coefficients from the lowest power)"""
    low = 1 / (1 + P * A_MAX)
    t = low + (1 - low) * 0.5 * (1 - np.cos(np.pi * (np.arange(nodes) + 0.5) / nodes))
    rows = np.polynomial.chebyshev.chebvander(2 * (t - low) / (1 - low) - 1, DEGREE) * (t / target((1 / t - 1) / P))[:, None]
    weight, best = np.ones(nodes) / nodes, None
    for _ in range(rounds):
        root = np.sqrt(weight)
        c = np.linalg.lstsq(rows * root[:, None], root, rcond=None)[0]
        off = np.abs(rows @ c - 1)
        if best is None or off.max() < best[0]:
            best = off.max(), c
        weight = weight * off
        weight /= weight.sum()
    power = np.polynomial.chebyshev.Chebyshev(best[1], domain=[low, 1]).convert(kind=np.polynomial.Polynomial)
    return best[0], power.coef


def evaluate(coef, a):
    """t Q(t) as the device evaluates it in fp32 (with a division rounded to nearest)."""
    def fma(x, y, z):
        return (x.astype(np.float64) * y.astype(np.float64) + np.float64(z)).astype(np.float32)

    a = a.astype(np.float32)
    t = (1 / fma(np.full_like(a, P), a, 1.0).astype(np.float64)).astype(np.float32)
    s = np.full_like(a, coef[-1])
    for c in coef[-2::-1]:
        s = fma(s, t, np.float32(c))
    return s * t


if __name__ == "__main__":
    error, coef = fit()
    coef = coef.astype(np.float32)
    a = np.linspace(0, 13.2, 400001).astype(np.float32)
    off = np.abs(evaluate(coef, a) / target(a.astype(np.float64)) - 1).max()
    print("fit %.2f half units, fp32 evaluation %.2f, at 0: %r" % (error * 2 ** 24, off * 2 ** 24, float(evaluate(coef, a[:1])[0])))
    for c in coef:
        print("%.9gf" % c)
