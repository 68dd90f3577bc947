"""Slow, plain CPU oracle for the attention operators: score modifiers, paged cache, received weights, eviction.

TEST INFRASTRUCTURE ONLY: imported by the tests; shares no code with the CUDA path and never imports it.  float64 over
the exact input values, one query head at a time, nothing rounded.

Definition (heads of dh columns, positions i of the query and j of the key):
    z = scale <q_i, k_j>;  z = cap tanh(z / cap);  z -= slope |i - j|;  z += table[clamp(j - i, -R, R) + R]
    p = softmax of z over the keys that the query sees;  out = sum_j p_j v_j;  lse = log sum_j exp(z_j)
A key that is not seen takes no part, whatever its row holds; a query that sees nothing (or only scores of -inf) has
out = 0, lse = -inf.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional

import numpy as np


@dataclass
class Mods:
    causal: bool = False
    scale: float = 0.125
    cap: float = 0.0
    slopes: Optional[np.ndarray] = None     # [heads]
    table: Optional[np.ndarray] = None      # [heads, 2R + 1]


def scores(q, k, m: Mods, h: int, qpos, kpos) -> np.ndarray:
    """Modified scores [rows, keys] of head h, before any mask."""
    with np.errstate(all="ignore"):
        z = (q @ k.T) * m.scale
        if m.cap:
            z = m.cap * np.tanh(z / m.cap)
        gap = kpos[None, :].astype(np.int64) - qpos[:, None].astype(np.int64)
        if m.slopes is not None:
            z = z - np.float64(m.slopes[h]) * np.abs(gap)
        if m.table is not None:
            R = m.table.shape[1] // 2
            entry = m.table[h].astype(np.float64)[np.clip(gap, -R, R) + R]
            z = np.where(entry == -np.inf, -np.inf, z + entry)      # hidden, whatever the key holds
    return z


def attend(q, k, v, m: Mods, h: int, qpos, kpos, seen):
    """One head: (out [rows, dh], lse [rows], p [rows, keys], spread [rows, dh]); spread = sum_j p_j |v_j|."""
    rows, dh = q.shape
    z = scores(q, k, m, h, qpos, kpos)
    out, lse, p = np.zeros((rows, dh)), np.full(rows, -np.inf), np.zeros((rows, k.shape[0]))
    spread = np.zeros((rows, dh))
    for r in range(rows):
        js = np.nonzero(seen[r])[0]
        if not len(js):
            continue
        zr = z[r, js]
        with np.errstate(all="ignore"):
            top = zr.max() if not np.isnan(zr).any() else np.nan
            if top == -np.inf:
                continue
            e = np.exp(zr - top)
            t = e.sum()
            p[r, js] = e / t
            lse[r] = top + np.log(t)
            used = js[p[r, js] > 0] if not np.isnan(t) else js
            out[r] = p[r, used] @ v[used]
            spread[r] = p[r, used] @ np.abs(v[used])
    return out, lse, p, spread


def visible(n: int, m: Mods, doc=None, prefix: Optional[int] = None) -> np.ndarray:
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    see = np.ones((n, n), dtype=bool)
    if m.causal:
        see = j <= i
        if prefix is not None:
            see = see | (j < prefix)
    if doc is not None:
        see = see & (doc[:, None] == doc[None, :]) & (doc[None, :] >= 0)
    return see


def attention(q, k, v, m: Mods, doc=None, prefix=None):
    """q [S, n, H, dh], k, v [S, n, HK, dh] float64 -> out, lse [S, n, H], spread like out."""
    S, n, H, dh = q.shape
    G = H // k.shape[2]
    out, lse, spread = np.zeros(q.shape), np.zeros((S, n, H)), np.zeros(q.shape)
    pos = np.arange(n)
    for s in range(S):
        see = visible(n, m, None if doc is None else doc[s], None if prefix is None else int(prefix[s]))
        for h in range(H):
            out[s, :, h], lse[s, :, h], _, spread[s, :, h] = attend(q[s, :, h], k[s, :, h // G], v[s, :, h // G], m, h, pos, pos, see)
    return out, lse, spread


@dataclass
class Cache:
    """Pages [num_pages, HK, page_size, dh] (float64 copies), per-sequence side arrays [n_seqs, HK, slots]."""
    k: np.ndarray
    v: np.ndarray

    def place(self, pages, slot):
        ps = self.k.shape[2]
        p = int(pages[slot // ps])
        return (p, slot % ps) if 0 <= p < self.k.shape[0] else (None, None)


def chunk(c: Cache, q, m: Mods, cu, lens, pages, k_new=None, v_new=None, weights=None, decay=1.0, positions=None, first=None,
          longest=None):
    """New rows of a batch over the paged cache; writes c, weights and positions.  q [T, H, dh] -> out, lse, spread, written:
    rows that belong to a sequence and are computed (the first `longest` of it)."""
    T, H, dh = q.shape
    HK, ps = c.k.shape[1], c.k.shape[2]
    G = H // HK
    out, lse, spread, written = np.zeros(q.shape), np.full((T, H), -np.inf), np.zeros(q.shape), np.zeros(T, dtype=bool)
    limit = pages.shape[1] * ps
    for s in range(len(lens)):
        n = min(int(lens[s]), limit)
        r0, r1 = int(cu[s]), int(cu[s + 1])
        for r in range(r0, r1):
            slot = n - (r1 - r)
            if slot < 0:
                continue
            if positions is not None:
                positions[s, :, slot] = (int(first[s]) + r - r0) if first is not None else slot
            if weights is not None:
                weights[s, :, slot] = 0.0
            if k_new is not None:
                p, at = c.place(pages[s], slot)
                if p is not None:
                    c.k[p, :, at], c.v[p, :, at] = k_new[r], v_new[r]
        new, r1 = r1 - r0, r1 if longest is None else min(r1, r0 + longest)
        written[r0:r1] = True
        there = np.array([c.place(pages[s], j)[0] is not None for j in range(n)], dtype=bool)
        slots = np.arange(n)
        mine = n - new + np.arange(r1 - r0)
        see = np.broadcast_to(there[None, :], (r1 - r0, n)).copy()
        if m.causal:
            see &= slots[None, :] <= mine[:, None]
        qpos = mine if first is None else int(first[s]) + np.arange(r1 - r0)
        for hk in range(HK):
            k, v = np.zeros((n, dh)), np.zeros((n, dh))
            for j in range(n):
                p, at = c.place(pages[s], j)
                if p is not None:
                    k[j], v[j] = c.k[p, hk, at], c.v[p, hk, at]
            kpos = slots if positions is None else positions[s, hk, :n]
            got = np.zeros(n)
            for h in range(hk * G, hk * G + G):
                o, l, p, sp = attend(q[r0:r1, h], k, v, m, h, qpos, kpos, see)
                out[r0:r1, h], lse[r0:r1, h], spread[r0:r1, h] = o, l, sp
                got += p.sum(0)
            if weights is not None:
                weights[s, hk, :n] = got if decay == 0 else decay * weights[s, hk, :n] + got
    return out, lse, spread, written


def evict(lens, weights, positions, budget: int, recent: int, sinks: int) -> List[List[np.ndarray]]:
    """Slots kept, ascending, per sequence and head.  weights [n_seqs, HK, slots]; positions likewise or None."""
    kept = []
    for s in range(len(lens)):
        n, row = int(lens[s]), []
        for hk in range(weights.shape[1]):
            pos = np.arange(n) if positions is None else positions[s, hk, :n].astype(np.int64)
            if n <= budget:
                row.append(np.arange(n))
                continue
            w = weights[s, hk, :n].astype(np.float64)
            w = np.where(w > 0, w, 0.0)                       # (NaN > 0 is false)
            safe = (pos < sinks) | (pos > pos.max() - recent)
            order = sorted(range(n), key=lambda j: (not safe[j], 0.0 if safe[j] else -w[j], j))
            row.append(np.sort(np.array(order[:budget])))
        kept.append(row)
    return kept
