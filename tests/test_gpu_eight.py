"""Norm with an 8-bit output and product of 8-bit matrices against the float64 oracle.

Tolerances, from the number formats (u = 2^-24, half a step of f32; bf16: 2^-8, e4m3: 2^-4 relative, 2^-10 below 2^-6):
  norm    a row's sums go through at most 32 additions in a thread, 5 in a warp, 16 between warps: 53 u of the sum of magnitudes, in the
          mean (of |h|) and in the mean square; the root, its inverse and two products add 6 u; h itself is rounded once.  An error of
          the mean moves all of y by rstd |gain| times as much.
  q       half a step of the type in units of the scale, which is off by the largest error of y / top and 2 u
  dense   int8: the sum is exact; its conversion, two products and an addition: 4 u of their sizes.  e4m3: at most k u of the sum
          of the products' sizes more.  GELU 3.8e-5: what gelu_fit.py prints for the larger
          of its two polynomials.  One rounding to bf16.
"""
import subprocess
import sys
import textwrap

import numpy as np
import pytest
import torch

from oracle import eight_oracle as E
from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F8 = torch.bfloat16, torch.float8_e4m3fn
U = 2.0 ** -24
TYPE = {"int8": torch.int8, "e4m3": F8}


def f64(t):
    return t.detach().cpu().float().to(torch.float64).numpy()


def rnd(*shape, seed, scale=1.0):
    return synth.randn(shape, seed, DEV, BF, scale)


def filled(rows, ld, cols, dtype, value=7):
    """A matrix of rows that are ld elements apart, and the whole of its memory."""
    whole = torch.full((rows, ld), value, dtype=torch.float32, device=DEV).to(dtype)
    return whole[:, :cols], whole


def norm_bounds(x, r, kind, gain, bias, eps=1e-5):
    """(h, y, bound of y's error) in float64."""
    h, y = E.norm(x, kind, gain, bias, eps, r)
    if kind == "none":
        return h, y, U * np.abs(h)
    g = 1.0 if gain is None else np.abs(gain)
    plain = y if bias is None else y - bias
    mean = h.mean(-1, keepdims=True) if kind == "layer" else 0.0
    rstd = 1.0 / np.sqrt(((h - mean) ** 2).mean(-1, keepdims=True) + eps)
    off_mean = 53 * U * np.abs(h).mean(-1, keepdims=True) if kind == "layer" else 0.0
    # the mean square: relative 53 u and what the mean's error adds (its square, and its product with a sum that is zero up to rounding)
    rel = 30 * U + 6 * U + (rstd * off_mean) ** 2 + 2 * rstd * off_mean * 53 * U
    return h, y, rstd * g * (2 * U * np.abs(h) + off_mean) + rel * np.abs(plain) + 2 * U * np.abs(y)


def check_eight(values, scale, y, tol, to):
    v, s = f64(values), scale.cpu().double().numpy()
    top = np.abs(y).max(-1)
    want = top / E.TOP[to]
    assert np.all(np.abs(s - want) <= tol.max(-1) / E.TOP[to] + 2 * U * want)
    assert np.all(np.abs(v) <= E.TOP[to]) and np.all(np.abs(v).max(-1) == E.TOP[to])
    half = 0.5 * s[:, None] if to == "int8" else np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s[:, None])
    far = np.abs(v * s[:, None] - y) - (half * (1 + 2.0 ** -20) + 2 * tol)
    assert np.all(far <= 0), float(far.max())
    # and the rounding is to the nearest: only values next to a border may differ from the oracle's
    ref, rs = E.eight_bits(y, to)
    other = v != ref
    assert other.mean() < 1e-3 + 1.5 / v.size


NORMS = [
    # rows, cols, kind, residual, total, out, to
    (1, 8, "rms", False, False, True, "int8"),
    (1, 1024, "rms", True, True, False, "e4m3"),
    (5, 64, "layer", True, True, True, "int8"),
    (3, 264, "layer", False, False, True, "e4m3"),
    (9, 520, "none", True, True, True, "int8"),
    (300, 768, "layer", False, False, True, "int8"),
    (2000, 1024, "rms", True, True, True, "e4m3"),
    (7, 1032, "rms", True, False, False, "int8"),            # one piece more than a warp holds
    (1501, 2048, "none", False, False, False, "e4m3"),
    (33, 4096, "layer", True, True, True, "int8"),
    (2, 4104, "rms", True, True, False, "e4m3"),             # one piece more than 128 threads hold
    (700, 5000, "none", False, False, False, "int8"),
    (600, 12296, "rms", False, True, True, "e4m3"),
    (400, 16384, "layer", True, False, True, "int8"),
    (611, 16384, "none", True, False, False, "int8"),
    # rows of 256 threads whose next row waits in shared memory, with 4 to 7 pieces each
    (170, 8192, "rms", False, False, True, "int8"),
    (301, 8200, "layer", True, True, True, "e4m3"),
    (1203, 12280, "rms", True, True, False, "int8"),
    (149, 14000, "layer", False, False, False, "e4m3"),
]


@pytest.mark.parametrize("rows,cols,kind,residual,total,out,to", NORMS)
@pytest.mark.parametrize("padded", [False, True])
def test_norm_against_the_oracle(rows, cols, kind, residual, total, out, to, padded):
    pad = 16 if padded else 0
    x = rnd(rows, cols + pad, seed=rows + cols)[:, :cols]
    x[:, 3::50] *= 6
    r = rnd(rows, cols + pad, seed=5)[:, :cols] if residual else None
    gain = torch.rand(cols, device=DEV) + 0.5 if kind != "none" else None
    bias = torch.randn(cols, device=DEV) * 0.2 if kind == "layer" else None
    t, whole_t = filled(rows, cols + pad, cols, BF) if total else (None, None)
    o, whole_o = filled(rows, cols + pad, cols, BF) if out else (None, None)
    q, whole_q = filled(rows, cols + pad, cols, TYPE[to])
    s = torch.full((rows,), 7.0, device=DEV)
    L.llmcache_norm(x, kind=kind, gain=gain, bias=bias, residual=r, total=t, out=o, q=q, scale=s)
    torch.cuda.synchronize()
    n64 = lambda a: None if a is None else f64(a)
    h, y, tol = norm_bounds(f64(x), n64(r), kind, n64(gain), n64(bias))
    if total:
        assert np.all(np.abs(f64(t) - h) <= 2.0 ** -8 * np.abs(h) * (1 + 2.0 ** -14) + 1e-38)
    if out:
        assert np.all(np.abs(f64(o) - y) <= 2.0 ** -8 * np.abs(y) + tol * (1 + 2.0 ** -8) + 1e-38)
    check_eight(q, s, y, tol, to)
    for whole in (whole_t, whole_o, whole_q):
        if whole is not None and padded:
            assert torch.all(whole[:, cols:].float() == 7)
    # alone, the parts of the output are the same bits
    q2, s2 = torch.zeros_like(q), torch.zeros_like(s)
    L.llmcache_norm(x, kind=kind, gain=gain, bias=bias, residual=r, q=q2, scale=s2)
    assert torch.equal(q2.view(torch.int8), q.contiguous().view(torch.int8)) and torch.equal(s2, s)
    if out:
        o2 = torch.zeros_like(o)
        L.llmcache_norm(x, kind=kind, gain=gain, bias=bias, residual=r, out=o2)
        assert torch.equal(o2, o)


def test_norm_of_a_mean_far_from_zero_and_without_gain():
    x = (rnd(40, 768, seed=3).float() * 0.5 + 60).to(BF)
    o = torch.zeros_like(x)
    L.llmcache_norm(x, kind="layer", out=o, eps=1e-12)
    h, y, tol = norm_bounds(f64(x), None, "layer", None, None, 1e-12)
    assert np.all(np.abs(f64(o) - y) <= 2.0 ** -8 * np.abs(y) + tol * 1.01)
    L.llmcache_norm(x, kind="rms", out=o)
    h, y, tol = norm_bounds(f64(x), None, "rms", None, None)
    assert np.all(np.abs(f64(o) - y) <= 2.0 ** -8 * np.abs(y) + tol * 1.01)


@pytest.mark.parametrize("to", ["int8", "e4m3"])
@pytest.mark.parametrize("cols", [64, 2048, 16384])
def test_rows_that_are_zero_tiny_infinite_or_nan(to, cols):
    x = rnd(8, cols, seed=9)
    x[1] = 0
    x[2] = 1e-31
    x[3, cols - 1] = float("inf")
    x[4, 0] = float("nan")
    x[5] *= 1e-28
    x[6, 5] = float("-inf")
    x[7] = x[7] * 1e30
    q, s = torch.full((8, cols), 7.0, device=DEV).to(TYPE[to]), torch.full((8,), 7.0, device=DEV)
    L.llmcache_norm(x, kind="none", q=q, scale=s)
    v, sc = f64(q), s.cpu()
    assert sc[1] == 0 and sc[2] == 0 and not v[1].any() and not v[2].any()
    assert torch.isnan(sc[[3, 4, 6]]).all() and not v[[3, 4, 6]].any()
    keep = [0, 5, 7]
    y = f64(x)[keep]
    check_eight(q[keep], s[keep], y, U * np.abs(y), to)
    # a normed row of zeros is its bias
    b = torch.randn(cols, device=DEV)
    o = torch.zeros((1, cols), dtype=BF, device=DEV)
    L.llmcache_norm(torch.zeros_like(o), kind="layer", bias=b, out=o)
    assert torch.equal(o[0], b.to(BF))


@pytest.mark.parametrize("rows,cols", [(50, 768), (9, 4096), (3, 16384), (600, 9000)])
def test_norm_in_place_and_with_a_row_count(rows, cols):
    x, r, gain = rnd(rows, cols, seed=11), rnd(rows, cols, seed=12), torch.rand(cols, device=DEV) + 0.5
    t, o = torch.zeros_like(x), torch.zeros_like(x)
    L.llmcache_norm(x, gain=gain, residual=r, total=t, out=o)
    x2, r2 = x.clone(), r.clone()
    L.llmcache_norm(x2, gain=gain, residual=r2, total=r2, out=x2)
    assert torch.equal(r2, t) and torch.equal(x2, o)
    for count in (0, 1, rows - 1, rows + 3):
        part = torch.full_like(x, 7.0)
        q, s = torch.full((rows, cols), 7, dtype=torch.int8, device=DEV), torch.full((rows,), 7.0, device=DEV)
        L.llmcache_norm(x, gain=gain, residual=r, out=part, q=q, scale=s, n_rows_dev=torch.tensor([count], dtype=torch.int32, device=DEV))
        m = min(count, rows)
        assert torch.equal(part[:m], o[:m]) and torch.all(part[m:] == 7) and torch.all(q[m:] == 7) and torch.all(s[m:] == 7)


# ------------------------------------------------------------------------------------------------------------ products
def eight_matrix(rows, k, to, seed, ld=0, finite=True):
    """8-bit values and scales; not finite: e4m3 has a NaN here and there, where a value lies beyond the type."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((rows, max(k, ld)), generator=g, device=DEV) * (40.0 if to == "int8" else 100.0)
    x = x.clamp(-448, 448) if finite else x
    m = (x.round().clamp(-127, 127) if to == "int8" else x).to(TYPE[to])
    return m[:, :k], torch.rand(rows, generator=g, device=DEV) + 0.5


def check_dense(out, a, sa, w, sw, to, bias, act, residual):
    n64 = lambda t: None if t is None else f64(t)
    sa, sw = sa.cpu().double().numpy(), sw.cpu().double().numpy()
    y, z = E.dense(f64(a), sa, f64(w), sw, n64(bias), act, n64(residual))
    b = 0.0 if bias is None else np.abs(f64(bias))
    tol = 3 * U * np.abs(z - (0 if bias is None else f64(bias))) + U * (np.abs(z) + b)
    if to == "e4m3":
        tol = tol + a.shape[1] * U * (np.abs(f64(a)) @ np.abs(f64(w)).T) * sa[:, None] * sw[None]
    tol = 1.13 * tol if act != "none" else tol
    if act != "none":
        tol = tol + 3.8e-5
    tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(y) + 2 * U * np.abs(y) + 1e-38
    got, nan = f64(out), np.isnan(y)
    assert np.array_equal(np.isnan(got), nan)
    far = (np.abs(got - y) - tol)[~nan]
    assert np.all(far <= 0), (float(far.max()), int((far > 0).sum()))


DENSE = [
    # m, n, k, bias, act, residual
    (1, 1, 16, True, "none", False),
    (1, 4096, 1024, True, "gelu_tanh", False),
    (1, 50257, 64, False, "none", False),
    (2, 17, 48, True, "none", True),
    (8, 200, 80, True, "gelu_erf", True),
    (9, 31, 4096, False, "none", True),
    (16, 129, 144, True, "gelu_tanh", True),
    (17, 64, 1040, True, "none", False),
    (32, 72, 96, True, "gelu_erf", True),                    # the last size of the kernel for few rows
    (33, 100, 208, True, "gelu_erf", False),
    (64, 2304, 768, True, "none", False),
    (64, 33, 8192, True, "none", True),
    (65, 40, 32, True, "none", True),
    (65, 1, 16, True, "none", True),
    (128, 64, 128, False, "none", False),
    (129, 95, 144, True, "gelu_erf", True),
    (200, 321, 400, True, "gelu_tanh", False),
    (1000, 2304, 768, True, "none", False),
    (1001, 1999, 272, True, "none", True),
    (2500, 2304, 768, True, "gelu_erf", False),
    (5000, 1024, 4096, True, "none", True),
    (4001, 2047, 1040, True, "gelu_tanh", True),
    # a long k shared by clusters of 8, 4 and 2 blocks
    (100, 33, 8192, True, "gelu_erf", True),
    (70, 2, 2960, False, "none", False),
    (65, 1024, 4096, True, "none", True),
    (300, 500, 3088, False, "gelu_tanh", False),
    (513, 700, 4112, True, "none", True),
    (129, 1983, 3200, True, "gelu_erf", False),
]


@pytest.mark.parametrize("m,n,k,bias,act,residual", DENSE)
@pytest.mark.parametrize("to", ["int8", "e4m3"])
def test_dense_against_the_oracle(m, n, k, bias, act, residual, to):
    a, sa = eight_matrix(m, k, to, m + k, ld=k + 32, finite=False)
    w, sw = eight_matrix(n, k, to, n + k + 1, ld=k + 16, finite=False)
    bits = lambda t: t.contiguous().view(torch.int16)
    sa, sw = sa / (40.0 if to == "int8" else 100.0), sw / ((40.0 if to == "int8" else 100.0) * k ** 0.5)
    b = torch.randn(n, device=DEV) * 0.5 if bias else None
    ld = -(-n // 8) * 8 + 8
    r = rnd(m, ld, seed=3)[:, :n] if residual else None
    out, whole = filled(m, ld, n, BF)
    L.llmcache_dense(a, sa, w, sw, out, bias=b, act=act, residual=r)
    torch.cuda.synchronize()
    assert L.llmcache_dense_status() == L.OK
    assert torch.all(whole[:, n:] == 7)                      # nothing behind a row's end
    check_dense(out, a, sa, w, sw, to, b, act, r)
    again = torch.zeros_like(whole)[:, :n]
    L.llmcache_dense(a, sa, w, sw, again, bias=b, act=act, residual=r)
    assert torch.equal(bits(again), bits(out))
    if residual:                                             # onto the residual itself
        r2 = torch.zeros_like(whole)
        r2[:, :n] = r
        L.llmcache_dense(a, sa, w, sw, r2[:, :n], bias=b, act=act, residual=r2[:, :n])
        assert torch.equal(bits(r2[:, :n]), bits(out))


@pytest.mark.parametrize("n,k", [(777, 1040), (300, 4016)])
def test_int8_rows_do_not_depend_on_how_many_there_are(n, k):
    """Whole-number sums and one arithmetic behind them: all kernels give the same bits."""
    a, sa = eight_matrix(2000, k, "int8", 1)
    w, sw = eight_matrix(n, k, "int8", 2)
    b = torch.randn(n, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    sa, sw, r = sa / 40, sw / (40 * k ** 0.5), rnd(2000, 784, seed=4)[:, :n]
    for act in ("none", "gelu_erf", "gelu_tanh"):
        whole = torch.zeros((2000, 784), dtype=BF, device=DEV)[:, :n]
        L.llmcache_dense(a, sa, w, sw, whole, bias=b, act=act, residual=r)
        for m in (1, 5, 12, 30, 32, 33, 64, 65, 300, 700):
            out = torch.zeros((m, 784), dtype=BF, device=DEV)[:, :n]
            L.llmcache_dense(a[:m], sa[:m], w, sw, out, bias=b, act=act, residual=r[:m])
            assert torch.equal(out, whole[:m]), (act, m)


@pytest.mark.parametrize("m", [3, 40])
def test_largest_sums(m):
    """The longest rows of the largest values: the integer sum reaches 2^31 less a little."""
    k, n = 131056, 70
    a = torch.full((m, k), -128, dtype=torch.int8, device=DEV)
    w = torch.full((n, k), -128, dtype=torch.int8, device=DEV)
    w[1::2] = 127
    one = torch.ones(max(m, n), device=DEV)
    for rows in (m, 80):
        out = torch.zeros((rows, 72), dtype=BF, device=DEV)[:, :n]
        L.llmcache_dense(a[:1].expand(rows, k).contiguous(), one[:1].expand(rows).contiguous(), w, one[:n].contiguous(), out)
        want = torch.tensor([128.0 * 128 * k, -128.0 * 127 * k], device=DEV).to(BF).repeat(n // 2)
        assert torch.equal(out, want.expand(rows, n))


@pytest.mark.parametrize("m,n,k", [(20, 100, 160), (300, 200, 160), (1000, 2304, 160), (300, 200, 4000)])
@pytest.mark.parametrize("to", ["int8", "e4m3"])
def test_dense_with_a_row_count(m, n, k, to):
    a, sa = eight_matrix(m, k, to, 5)
    w, sw = eight_matrix(n, k, to, 6)
    r = rnd(m, n + (-n) % 8, seed=7)[:, :n]
    full = torch.zeros((m, n + (-n) % 8), dtype=BF, device=DEV)[:, :n]
    L.llmcache_dense(a, sa, w, sw, full, residual=r, act="gelu_erf")
    for count in (0, 1, m // 2 + 1, m - 1, m, m + 50):
        out, _ = filled(m, n + (-n) % 8, n, BF)
        L.llmcache_dense(a, sa, w, sw, out, residual=r, act="gelu_erf", n_rows_dev=torch.tensor([count], dtype=torch.int32, device=DEV))
        c = min(count, m)
        assert torch.equal(out[:c], full[:c]) and torch.all(out[c:] == 7), count
    assert L.llmcache_dense_status() == L.OK


def test_scales_of_nan_and_zero():
    for m in (4, 100):
        a, sa = eight_matrix(m, 64, "int8", 8)
        w, sw = eight_matrix(24, 64, "int8", 9)
        sa[1], sa[2] = float("nan"), 0.0
        out = torch.zeros((m, 24), dtype=BF, device=DEV)
        L.llmcache_dense(a, sa, w, sw, out)
        assert torch.isnan(out[1]).all() and not out[2].any() and torch.isfinite(out[[0] + list(range(3, m))]).all()


def test_both_on_another_stream_and_in_a_graph():
    m, d, n = 70, 256, 320
    x, gain = rnd(m, d, seed=21), torch.rand(d, device=DEV) + 0.5
    w, sw = eight_matrix(n, d, "e4m3", 22)
    q, s, out = torch.zeros((m, d), device=DEV).to(F8), torch.zeros(m, device=DEV), torch.zeros((m, n), dtype=BF, device=DEV)

    def step(stream=None):
        L.llmcache_norm(x, gain=gain, q=q, scale=s, stream=stream)
        L.llmcache_dense(q, s, w, sw, out, act="gelu_tanh", stream=stream)

    step()
    torch.cuda.synchronize()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    first = x.clone()
    for seed in (23, 24):
        x.copy_(rnd(m, d, seed=seed))
        step()
        torch.cuda.synchronize()
        eager = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    x.copy_(first)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_two_streams_at_a_time():
    """Calls share nothing but the status word: two chains of them, side by side, give what each gives alone."""
    shapes, chains = ((300, 512, 640), (64, 4096, 1024)), []
    for i, (m, d, n) in enumerate(shapes):
        x, (w, sw) = rnd(m, d, seed=41 + i), eight_matrix(n, d, "int8", 43 + i)
        q, s = torch.zeros((m, d), dtype=torch.int8, device=DEV), torch.zeros(m, device=DEV)
        chains.append((x, w, sw, q, s, [torch.zeros((m, n), dtype=BF, device=DEV) for _ in range(20)], torch.cuda.Stream()))

    def step(c, i, stream):
        x, w, sw, q, s, outs, _ = c
        L.llmcache_norm(x, kind="none", q=q, scale=s, stream=stream)
        L.llmcache_dense(q, s, w, sw, outs[i], act="gelu_erf", stream=stream)

    torch.cuda.synchronize()
    want = []
    for c in chains:
        step(c, 0, None)
        torch.cuda.synchronize()
        want.append(c[5][0].clone())
        c[5][0].zero_()
    torch.cuda.synchronize()
    for i in range(20):
        for c in chains:
            step(c, i, c[6])
    torch.cuda.synchronize()
    for c, w in zip(chains, want):
        assert all(torch.equal(o, w) for o in c[5])
    assert L.llmcache_dense_status() == L.OK


def test_matrices_of_more_than_2_31_elements():
    m, k = 40000, 64
    for n, to in ((60000, "int8"), (60001, "e4m3")):
        a, sa = eight_matrix(m, k, to, 51)
        w, sw = eight_matrix(n, k, to, 52)
        sa, sw = sa / 100, sw / 800
        out, whole = filled(m, 60008, n, BF)
        L.llmcache_dense(a, sa, w, sw, out, residual=out)
        torch.cuda.synchronize()
        rows = [0, 17895, 17896, 35786, 35787, 35791, 35792, m - 129, m - 1]
        check_dense(out[rows], a[rows], sa[rows], w, sw, to, None, "none", torch.full((len(rows), n), 7.0, dtype=BF, device=DEV))
        assert torch.all(whole[:, n:] == 7)
        del out, whole
    rows, cols = 140000, 16384
    x = torch.randn((rows, cols), generator=torch.Generator(device=DEV).manual_seed(53), dtype=BF, device=DEV)
    t, q, s = torch.zeros_like(x), torch.zeros((rows, cols), dtype=torch.int8, device=DEV), torch.zeros(rows, device=DEV)
    L.llmcache_norm(x, total=t, q=q, scale=s)
    torch.cuda.synchronize()
    assert torch.equal(t, x)
    some = [0, 65535, 65536, 131071, 131072, rows - 1]
    _, y, tol = norm_bounds(f64(x[some]), None, "rms", None, None)
    check_eight(q[some], s[some], y, tol, "int8")
    q2, s2 = torch.zeros_like(q[130000:]), torch.zeros_like(s[130000:])
    L.llmcache_norm(x[130000:], q=q2, scale=s2)
    assert torch.equal(q2, q[130000:]) and torch.equal(s2, s[130000:])
    assert L.llmcache_dense_status() == L.OK


def test_norm_and_product_together():
    """Quantised rows through a product: within the quantisation's own error of the product of what was quantised."""
    m, d, n = 300, 512, 384
    x, r, gain = rnd(m, d, seed=31), rnd(m, d, seed=32), torch.rand(d, device=DEV) + 0.5
    wb = rnd(n, d, seed=33, scale=0.05)
    for to in ("int8", "e4m3"):
        w8, ws = torch.zeros((n, d), device=DEV).to(TYPE[to]), torch.zeros(n, device=DEV)
        L.llmcache_norm(wb, kind="none", q=w8, scale=ws)
        q, s, t, out = torch.zeros((m, d), device=DEV).to(TYPE[to]), torch.zeros(m, device=DEV), torch.zeros_like(x), torch.zeros((m, n), dtype=BF, device=DEV)
        L.llmcache_norm(x, gain=gain, residual=r, total=t, q=q, scale=s)
        L.llmcache_dense(q, s, w8, ws, out)
        check_dense(out, q, s, w8, ws, to, None, "none", None)
        _, y = E.norm(f64(x), "rms", f64(gain), residual=f64(r))
        half = lambda v, sc: 0.5 * sc[:, None] * np.ones_like(v) if to == "int8" else np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * sc[:, None])
        ya, wa = np.abs(y), np.abs(f64(wb))
        ey, ew = half(y, f64(s)) * 1.001 + 1e-5 * ya, half(f64(wb), f64(ws)) * 1.001
        want = y @ f64(wb).T
        assert np.all(np.abs(f64(out) - want) <= ya @ ew.T + ey @ wa.T + ey @ ew.T + 2.0 ** -8 * np.abs(want) + 1e-3)


def test_expired_wait_is_reported_and_the_next_call_runs():
    """The loading warp stays idle, so the first wait runs out: the call returns, the status says so, the next call is right.  In a
    process of its own, because the status is sticky."""
    code = textwrap.dedent("""
        import torch
        from paper_2512_16843_b200 import binding as L
        g = torch.Generator(device="cuda").manual_seed(1)
        for dtype, m, n, k in ((torch.int8, 200, 96, 256), (torch.float8_e4m3fn, 5000, 1000, 256), (torch.int8, 200, 96, 4096)):
            a, w = (torch.randn((r, k), generator=g, device="cuda").mul(20).to(dtype) for r in (m, n))
            s = torch.ones(5000, device="cuda")
            r = torch.randn((m, n), generator=g, device="cuda").to(torch.bfloat16)
            call = lambda out: L.llmcache_dense(a, s[:m], w, s[:n], out, residual=r)
            want, out = torch.zeros_like(r), torch.zeros_like(r)
            call(want)
            if dtype is torch.int8 and k == 256:
                assert L.llmcache_dense_status() == L.OK
            L.llmcache_dense_debug_knobs(1_000_000, L.KNOB_PRODUCER_IDLE)
            call(out)
            torch.cuda.synchronize()
            assert L.llmcache_dense_status() == L.ERR_TIMEOUT
            L.llmcache_dense_debug_knobs(0, 0)
            call(out)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert L.llmcache_dense_status() == L.ERR_TIMEOUT            # sticky
        print("fine")
    """)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout + r.stderr
