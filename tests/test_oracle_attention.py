"""Pins of the attention oracle: library softmax attention in float64, hand-worked rows, masks, eviction by hand."""
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A


def rnd(*shape, seed=0):
    return np.random.RandomState(seed).randn(*shape)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,HK", [(4, 4), (4, 2), (3, 1)])
def test_plain_attention_equals_the_librarys_in_float64(causal, H, HK):
    q, k, v = rnd(2, 9, H, 8, seed=1), rnd(2, 9, HK, 8, seed=2), rnd(2, 9, HK, 8, seed=3)
    out, lse, _ = A.attention(q, k, v, A.Mods(causal=causal, scale=8 ** -0.5))
    t = lambda x: torch.from_numpy(np.repeat(x, H // x.shape[2], axis=2)).transpose(1, 2)
    ref = torch.nn.functional.scaled_dot_product_attention(t(q), t(k), t(v), is_causal=causal).transpose(1, 2).numpy()
    assert np.allclose(out, ref, rtol=1e-12, atol=1e-12)


def test_modifiers_on_a_row_worked_by_hand():
    # one query at position 1, three keys; <q, k> = 8, 0, -8 -> scaled 1, 0, -1
    q, k, v = np.array([[8.0]]), np.array([[1.0], [0.0], [-1.0]]), np.array([[1.0], [10.0], [100.0]])
    pos = np.arange(3)
    m = A.Mods(cap=2.0, slopes=np.array([0.5]), table=np.array([[0.25, 0.0, -0.25]]))
    z = [2 * math.tanh(0.5) - 0.5 + 0.25, 0.0, -2 * math.tanh(0.5) - 0.5 - 0.25]
    e = np.exp(z)
    out, lse, p, _ = A.attend(q, k, v, m, 0, np.array([1]), pos, np.ones((1, 3), bool))
    assert np.allclose(p[0], e / e.sum()) and np.isclose(lse[0], math.log(e.sum())) and np.isclose(out[0, 0], (e / e.sum()) @ v[:, 0])


def test_masks_and_rows_that_see_nothing():
    see = A.visible(4, A.Mods(causal=True), np.array([0, 0, 1, -1]), prefix=None)
    assert see.tolist() == [[True, False, False, False], [True, True, False, False], [False, False, True, False], [False] * 4]
    see = A.visible(3, A.Mods(causal=True), None, prefix=2)
    assert see.tolist() == [[True, True, False], [True, True, False], [True, True, True]]
    k = np.full((2, 4), np.nan)
    out, lse, p, _ = A.attend(rnd(1, 4), k, k, A.Mods(), 0, np.zeros(1, int), np.arange(2), np.zeros((1, 2), bool))
    assert not out.any() and lse[0] == -np.inf and not p.any()


def test_chunks_over_the_cache_equal_causal_attention_over_the_whole_sequence():
    n, H, HK, dh, ps = 11, 4, 2, 8, 4
    q, k, v = rnd(1, n, H, dh, seed=4), rnd(1, n, HK, dh, seed=5), rnd(1, n, HK, dh, seed=6)
    m = A.Mods(causal=True, slopes=np.linspace(0.1, 0.4, H))
    ref, lse_ref, _ = A.attention(q, k, v, m)
    c = A.Cache(np.zeros((5, HK, ps, dh)), np.zeros((5, HK, ps, dh)))
    pages, w = np.array([[3, 0, 4]]), np.zeros((1, HK, 12))
    at = 0
    for step in (5, 1, 4, 1):
        rows = slice(at, at + step)
        out, lse, _, written = A.chunk(c, q[0, rows], m, [0, step], [at + step], pages, k[0, rows], v[0, rows], weights=w)
        assert written.all() and np.allclose(out, ref[0, rows]) and np.allclose(lse, lse_ref[0, rows])
        at += step
    assert np.allclose(w.sum(-1), n * H // HK)            # every row's softmax sums to one


def test_eviction_by_hand():
    w = np.array([[[0.5, np.nan, 3.0, 3.0, -1.0, 0.1, 0.2]]])
    assert A.evict([7], w, None, 4, recent=1, sinks=1)[0][0].tolist() == [0, 2, 3, 6]
    assert A.evict([7], w, None, 3, recent=0, sinks=0)[0][0].tolist() == [0, 2, 3]
    assert A.evict([7], w * 0, None, 3, recent=1, sinks=0)[0][0].tolist() == [0, 1, 6]     # ties: the lower slot
    assert A.evict([3], w, None, 4, recent=1, sinks=1)[0][0].tolist() == [0, 1, 2]
    pos = np.array([[[9, 1, 2, 3, 4, 5, 6]]])
    assert A.evict([7], w, pos, 2, recent=1, sinks=0)[0][0].tolist() == [0, 2]             # slot 0 holds the newest
