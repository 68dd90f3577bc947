"""Coefficients of the odd polynomials that stand for tanh on |u| <= 0.4 and |u| <= 0.75 in the attention kernels (attn_dev.cuh).

tanh(u) = u P(u^2): P of degree 3 or 5 fitted to tanh(sqrt s) / sqrt s on s in [0, limit^2] at Chebyshev nodes (within a
factor of two of the best uniform fit; the nearest singularity, u = i pi / 2, lies far enough away for an error that falls by a
factor of about 20 per coefficient on the longer range, 60 on the shorter).  Prints the f32 coefficients, lowest first, and the
largest relative error of the f32 evaluation (Horner, fused multiply-add): 2.1e-7 and 1.4e-7.
"""
import numpy as np
from numpy.polynomial import chebyshev as Ch

RANGES = ((0.4, 3), (0.75, 5))


def fit(LIMIT, DEGREE):
    n = 4000
    s = (np.cos((np.arange(n) + 0.5) * np.pi / n) + 1) / 2 * LIMIT * LIMIT
    u = np.sqrt(s)
    c = Ch.chebfit(2 * s / (LIMIT * LIMIT) - 1, np.tanh(u) / u, DEGREE)
    return Ch.Chebyshev(c, domain=[0, LIMIT * LIMIT]).convert(kind=np.polynomial.Polynomial).coef.astype(np.float32)


def error(p, LIMIT, DEGREE):
    u = np.linspace(1e-4, LIMIT, 200001).astype(np.float32)
    s = u * u
    a = np.full_like(u, p[-1])
    for k in range(DEGREE - 1, -1, -1):
        a = (a.astype(np.float64) * s + p[k]).astype(np.float32)      # one rounding, as in a fused multiply-add
    t = np.tanh(u.astype(np.float64))
    return float(np.max(np.abs((a * u).astype(np.float64) - t) / t))


if __name__ == "__main__":
    for r in RANGES:
        p = fit(*r)
        print(r, ["%.9ef" % x for x in p], error(p, *r))
