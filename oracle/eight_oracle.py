"""Slow, plain CPU oracle for the operators with 8-bit values and for the rotation by position, in float64.

TEST INFRASTRUCTURE ONLY: imported by the tests; shares no code with the CUDA path and never imports it.

* `norm`: h = x + residual and its root-mean-square or layer norm (or h itself);
* `eight_bits`: a scale per row and the 8-bit values, int8 or e4m3, rounded to nearest even;
* `dense`: act(a_scale w_scale (a w^T) + bias) + residual from the values that the bytes stand for;
* `rotate`: pairs of columns turned by position * inv_freq.

Pins: tests/test_oracle_eight.py.
"""
from __future__ import annotations

import math

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}


def norm(x, kind, gain=None, bias=None, eps=1e-5, residual=None):
    """(h, y) of rows x [rows, cols]."""
    h = np.asarray(x, dtype=np.float64)
    if residual is not None:
        h = h + residual
    if kind == "none":
        return h, h
    mean = h.mean(-1, keepdims=True) if kind == "layer" else 0.0
    y = (h - mean) / np.sqrt(((h - mean) ** 2).mean(-1, keepdims=True) + eps)
    if gain is not None:
        y = y * gain
    return h, y if bias is None else y + bias


def e4m3(x):
    """x rounded to the nearest number of four significant bits with exponents of -6 .. 8 (ties to even), at most 448."""
    x = np.asarray(x, dtype=np.float64)
    size = np.abs(x)
    with np.errstate(divide="ignore"):
        exponent = np.floor(np.log2(np.where(size > 0, size, 1.0)))
    step = 2.0 ** (np.maximum(exponent, -6.0) - 3.0)
    return np.sign(x) * np.minimum(np.rint(size / step) * step, 448.0)


def eight_bits(y, to):
    """(values, scale): scale * values stands for the rows of y."""
    y = np.asarray(y, dtype=np.float64)
    top = np.abs(y).max(-1, initial=0.0)                 # (NaN stays NaN)
    fine = np.isfinite(top)
    some = fine & (top >= 1e-30)
    scale = np.where(fine, np.where(some, top, 0.0) / TOP[to], np.nan)
    with np.errstate(invalid="ignore"):
        v = np.where(some[..., None], y / np.where(some, scale, 1.0)[..., None], 0.0)
    return (np.rint(v) if to == "int8" else e4m3(v)), scale


def gelu(x, act):
    if act == "gelu_erf":
        return x * 0.5 * (1.0 + np.vectorize(math.erf)(x / math.sqrt(2.0)))
    if act == "gelu_tanh":
        return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))
    return x


def dense(a, a_scale, w, w_scale, bias=None, act="none", residual=None):
    """(result, sum in front of the activation); a, w: the values of the bytes."""
    z = (np.asarray(a, np.float64) @ np.asarray(w, np.float64).T) * np.asarray(a_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)[None]
    if bias is not None:
        z = z + bias
    y = gelu(z, act)
    return (y if residual is None else y + residual), z


def rotate(x, position, inv_freq, interleaved=False):
    """x [rows, heads, 64] with its first 2 * len(inv_freq) columns turned by position [rows]."""
    x = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    angle = np.asarray(position, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    first = np.arange(half) * 2 if interleaved else np.arange(half)
    second = first + 1 if interleaved else first + half
    a, b = x[..., first], x[..., second]
    x[..., first], x[..., second] = a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)
    return x
