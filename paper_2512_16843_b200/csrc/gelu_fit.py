"""Derives the coefficients of the GELU polynomials of the 8-bit products in layer_epi.cuh (not part of the build; run by hand).

GELU(x) = x * phi(x), phi(x) = 1/2 + T(x) with T(x) = erf(x / sqrt 2) / 2, or tanh(sqrt(2 / pi) (x + 0.044715 x^3)) / 2.  phi is taken as
x * Q(x^2) + 1/2 clamped to [0, 1], which is a modifier of the multiply-add.  Q has nine coefficients, so its last one is positive: beyond
the fitted range the polynomial leaves [0, 1] on the right side and the clamp gives the limit itself.  The fit on [0, limit]
minimises the largest error of GELU (the error of T weighted by |x|) with Lawson's reweighted least squares on Chebyshev nodes, and
the script then evaluates the float32 arithmetic of the kernel (Horner, fused multiply-add) up to the largest numbers.
"""
import math

import numpy as np

N_COEF = 9
_erf = np.vectorize(math.erf)
FORMS = {
    "erf": (4.3, lambda u: 0.5 * _erf(u / math.sqrt(2.0))),
    "tanh": (4.2, lambda u: 0.5 * np.tanh(math.sqrt(2.0 / math.pi) * (u + 0.044715 * u ** 3))),
}


def fit(limit, target, iters=120):
    v = (np.cos(np.pi * (np.arange(4000) + 0.5) / 4000) + 1) / 2
    x = v * limit
    y = target(x)
    w = np.ones_like(v)
    A = np.stack([v * (v * v) ** k for k in range(N_COEF)], 1)
    for _ in range(iters):
        wt = w * np.maximum(x, 0.05)
        coef, *_ = np.linalg.lstsq(A * wt[:, None], y * wt, rcond=None)
        e = np.abs(A @ coef - y) * np.maximum(x, 0.05)
        w = w * (0.5 + e / e.max())
        w /= w.mean()
    return np.array([c / limit ** (2 * k + 1) for k, c in enumerate(coef)])     # in powers of x, not of x / limit


def largest_error(coef, target):
    k32 = coef.astype(np.float32)
    far = 10.0 ** np.linspace(0, 38, 400)
    xs = np.concatenate([np.linspace(-12, 12, 600001), far, -far]).astype(np.float32)
    with np.errstate(over="ignore"):
        s = xs * xs
        q = np.full_like(xs, k32[-1])
        for k in range(len(k32) - 2, -1, -1):
            q = (q.astype(np.float64) * s + k32[k]).astype(np.float32)          # one rounding
        phi = np.clip(q.astype(np.float64) * xs + 0.5, 0.0, 1.0).astype(np.float32)
    x = xs.astype(np.float64)
    e = np.abs(phi * xs - x * (0.5 + np.sign(x) * target(np.minimum(np.abs(x), 1e6))))
    return float(np.max(e / np.maximum(1.0, np.abs(x) / 300)))


if __name__ == "__main__":
    for name, (limit, target) in FORMS.items():
        k = fit(limit, target)
        print(name, "on [0, %g], highest power first:" % limit, ", ".join("%.9ef" % t for t in k[::-1].astype(np.float32)))
        print("largest |GELU error| in float32: %.3g" % largest_error(k, target))
