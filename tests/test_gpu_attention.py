"""Attention operators against the float64 oracle: score modifiers, paged cache, received weights, eviction.

Tolerances, from the number formats (u = unit roundoff):
  scores    a sum of 64 exact bf16 products in f32: at most 64 * 2^-24 * scale * sum |q_c k_c|; scaling, bias and the base
            change of the exponent add a few 2^-24 |z|, the capped score 2^-20 * cap.  delta = the sum of these bounds.
  weights p exp and division: relative 2 * delta + 2^-20 + n * 2^-24 (sum of n positive terms)
  out       p feeds the product as bf16 (half a step: 2^-8 relative), the sum is f32, the result is bf16 (2^-8):
            |error| <= 2^-8 |out| + (2^-8 + 2 delta + 2^-20 + n 2^-24) * sum_j p_j |v_j|, times (1 + 2^-6) for second order terms
  lse       delta + 2^-20 + n 2^-24 + 2^-22 |lse|
"""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import transformer_oracle as T
from oracle import llmcache_oracle as O
from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def rnd(*shape, seed, scale=1.0):
    return synth.randn(shape, seed, DEV, BF, scale)


def mods_pair(heads, *, causal, cap=0.0, bias=None, scale=0.0, reach=5, seed=3, doc=None, prefix=None):
    """The same modifiers for the library and for the oracle."""
    g = np.random.RandomState(seed)
    slopes = torch.tensor(2.0 ** (-8.0 * (np.arange(heads) + 1) / heads), dtype=torch.float32, device=DEV) if bias == "slopes" else None
    table = torch.tensor(g.randn(heads, 2 * reach + 1), dtype=torch.float32, device=DEV) if bias == "table" else None
    mine = L.make_score_mods(causal=causal, cap=cap, scale=scale, slopes=slopes, table=table, doc=doc, prefix=prefix)
    ref = A.Mods(causal=causal, cap=cap, scale=scale or 0.125, slopes=None if slopes is None else f64(slopes),
                 table=None if table is None else f64(table))
    return mine, ref


def delta(q, k, m: A.Mods, n):
    """Bound of a score's error, from the magnitudes (finite values only)."""
    size = lambda x: np.nanmax(np.where(np.isfinite(x), np.abs(x), 0).reshape(-1, 64), initial=0.0)
    norm = lambda x: np.sqrt(np.max(np.sum(np.where(np.isfinite(x), x, 0).reshape(-1, 64) ** 2, -1), initial=0.0))
    dot = norm(q) * norm(k) * m.scale                     # sum |q_c k_c| <= |q| |k|
    bias = (np.max(m.slopes) * n if m.slopes is not None else 0.0) + (np.max(np.abs(m.table[np.isfinite(m.table)]), initial=0.0) if m.table is not None else 0.0)
    return 64 * 2.0 ** -24 * dot + 6 * 2.0 ** -24 * (dot + bias) + 2.0 ** -20 * m.cap


def check(out, lse, ref_out, ref_lse, spread, d, n, rows=None):
    got, got_lse = f64(out), None if lse is None else f64(lse)
    if rows is not None:
        got, ref_out, spread = got[rows], ref_out[rows], spread[rows]
        if lse is not None:
            got_lse, ref_lse = got_lse[rows], ref_lse[rows]
    rel = 2 * d + 2.0 ** -20 + n * 2.0 ** -24
    tol = (2.0 ** -8 * np.abs(ref_out) + (2.0 ** -8 + rel) * spread) * (1 + 2.0 ** -6)
    fin = np.isfinite(ref_out)
    assert np.array_equal(np.isnan(got), np.isnan(ref_out)) and np.array_equal(got[~fin & ~np.isnan(ref_out)], ref_out[~fin & ~np.isnan(ref_out)])
    bad = np.abs(got - ref_out)[fin] > tol[fin]
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - ref_out)[fin] - tol[fin])))
    if lse is not None:
        fin = np.isfinite(ref_lse)
        assert np.array_equal(np.isnan(got_lse), np.isnan(ref_lse))
        assert np.array_equal(got_lse == -np.inf, ref_lse == -np.inf)
        assert np.all(np.abs(got_lse - ref_lse)[fin] <= d + 2.0 ** -20 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(ref_lse[fin]))


def run_attention(q, k, v, mine, ref, doc=None, prefix=None, n_seqs_dev=None):
    S, n, H, _ = q.shape
    out = torch.full((S, n, H, 64), 7.0, dtype=BF, device=DEV)
    lse = torch.full((S, n, H), 7.0, device=DEV)
    L.llmcache_attention(q, k, v, out, mods=mine, lse=lse, n_seqs_dev=n_seqs_dev)
    torch.cuda.synchronize()
    assert L.llmcache_attention_status() == L.OK
    ro, rl, sp = A.attention(f64(q), f64(k), f64(v), ref, None if doc is None else doc.cpu().numpy(), None if prefix is None else prefix.cpu().numpy())
    return out, lse, ro, rl, sp


def fused(S, n, H, HK, seed):
    m = rnd(S, n, H + 2 * HK, 64, seed=seed)
    m[:, :, :H] *= 2
    return m[:, :, :H], m[:, :, H:H + HK], m[:, :, H + HK:]


def docs(S, n, seed, sorted_ids=True):
    g = np.random.RandomState(seed)
    d = g.randint(-1, 4, (S, n))
    if sorted_ids:
        d = np.where(np.sort(d, 1) == -1, 9, np.sort(d, 1))
        d = np.sort(d, 1)
        d[d == 9] = -1
    return torch.tensor(d, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------ attention, whole sequences
@pytest.mark.parametrize("n", [1, 2, 31, 64, 65, 127, 128, 129, 193, 256, 257, 300])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(n, causal):
    S, H = 2, 3
    q, k, v = fused(S, n, H, H, 10 + n)
    mine, ref = mods_pair(H, causal=causal)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)


@pytest.mark.parametrize("H,HK", [(1, 1), (4, 1), (6, 2), (7, 1), (5, 5), (32, 2)])
@pytest.mark.parametrize("n", [5, 131])
def test_head_layouts(H, HK, n):
    q, k, v = fused(2, n, H, HK, 40 + H)
    mine, ref = mods_pair(H, causal=True, bias="slopes")
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [None, "slopes", "table"])
@pytest.mark.parametrize("cap", [0.0, 30.0, 2.0])
def test_modifiers(causal, bias, cap):
    S, n, H, HK = 2, 150, 4, 2
    q, k, v = fused(S, n, H, HK, 60)
    mine, ref = mods_pair(H, causal=causal, bias=bias, cap=cap, scale=0.2)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)


@pytest.mark.parametrize("reach", [0, 1, 200, 1024])
def test_table_reach(reach):
    S, n, H = 1, 140, 2
    q, k, v = fused(S, n, H, H, 65)
    mine, ref = mods_pair(H, causal=False, bias="table", reach=reach)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)


@pytest.mark.parametrize("causal,prefix,sorted_ids,n", [
    (False, None, True, 200), (False, None, False, 200), (True, None, True, 300), (True, [0, 70, 300], True, 300),
    (True, [1, 129, 500], None, 260), (True, [-3, 0, 128], None, 129)])
def test_documents_prefixes_and_rows_that_see_nothing(causal, prefix, sorted_ids, n):
    S, H, HK = 3, 4, 2
    q, k, v = fused(S, n, H, HK, 70)
    doc = None if sorted_ids is None else docs(S, n, 5, sorted_ids)
    pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=DEV)
    mine, ref = mods_pair(H, causal=causal, bias="slopes", doc=doc, prefix=pre)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref, doc, pre)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)
    if doc is not None:
        empty = (doc < 0)
        assert empty.any() and not out[empty].any() and torch.all(lse[empty] == float("-inf"))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_seen_may_hold_anything(bad):
    """Padding, other documents and the future: values that are not numbers stay with the rows that see them."""
    S, n, H = 1, 200, 2
    q, k, v = fused(S, n, H, H, 80)
    k, v = k.clone(), v.clone()
    doc = torch.zeros((S, n), dtype=torch.int32, device=DEV)
    doc[:, 60:130], doc[:, 130:180], doc[:, 180:] = 1, 2, -1
    k[:, 180:], v[:, 180:] = bad, bad                    # padding
    v[:, 100, :, 7] = bad                                # one value of document 1: its rows from 100 on, its column
    mine, ref = mods_pair(H, causal=True, doc=doc)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref, doc)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)
    assert torch.isfinite(out[:, :100]).all() and torch.isfinite(out[:, 130:]).all() and not torch.isfinite(out[:, 100:130, :, 7]).any()
    k[:, 150, 1] = float("nan")                          # a key that is not a number: every row that sees it, in its head
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref, doc)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)
    assert torch.isnan(out[:, 150:180, 1]).all() and torch.isfinite(out[:, 130:180, 0]).all()


def test_infinite_values_of_both_signs_that_are_seen():
    q, k, v = fused(1, 140, 1, 1, 81)
    v = v.clone()
    v[0, 3, 0, 5], v[0, 70, 0, 5], v[0, 70, 0, 6] = float("inf"), float("-inf"), float("-inf")
    mine, ref = mods_pair(1, causal=True)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, 140), 140)
    assert torch.isinf(out[0, 3:70, 0, 5]).all() and torch.isnan(out[0, 70:, 0, 5]).all()


@pytest.mark.parametrize("low", [float("-inf"), float(torch.finfo(torch.float32).min)])
def test_masks_written_into_the_table(low):
    """Entries of -inf hide a distance; entries of the type's lowest value do unless there is nothing else."""
    n, H = 150, 2
    q, k, v = fused(1, n, H, H, 82)
    table = torch.full((H, 2 * 64 + 1), low, device=DEV)
    table[0, 60:70] = 0.0                                # head 0 sees distances -4 .. 5; head 1 nothing but low entries
    mine = L.make_score_mods(table=table)
    ref = A.Mods(table=f64(table))
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out[:, :, :1], lse[:, :, :1], ro[:, :, :1], rl[:, :, :1], sp[:, :, :1], delta(f64(q), f64(k), A.Mods(), n), n)
    if low == float("-inf"):
        assert not out[:, :, 1].any() and torch.all(lse[:, :, 1] == low)
    else:                                                # f32: every score is the lowest value, so all keys count alike
        mean = f64(v)[0, :, 1].mean(0)
        assert np.all(np.abs(f64(out)[0, :, 1] - mean) <= 2.0 ** -8 * np.abs(mean) + (2.0 ** -8 + 2.0 ** -14) * np.abs(f64(v)[0, :, 1]).mean(0))


def test_growing_scores_and_large_ones():
    """The running maximum grows from tile to tile, by far more than a factor that the sums could hold."""
    n, H = 520, 2
    q, k, v = fused(1, n, H, H, 83)
    k = (k.float() * (1 + torch.arange(n, device=DEV).view(1, n, 1, 1) / 20)).to(BF)
    mine, ref = mods_pair(H, causal=False, scale=1.0)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)
    k = k.flip(1)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)


def test_strides_and_device_side_count():
    S, n, H, HK = 5, 140, 4, 2
    q = rnd(S, H, n, 64, seed=90).transpose(1, 2)                         # [S, H, n, 64] storage
    k = rnd(n, S, HK, 72, seed=91).transpose(0, 1)[..., 8:]               # padded rows, sequences inside tokens
    v = rnd(S, n, 3, HK, 64, seed=92)[:, :, 1]
    mine, ref = mods_pair(H, causal=True)
    for count in (0, 3, 5, 9):
        out = torch.full((S, H, n, 64), 7.0, dtype=BF, device=DEV).transpose(1, 2)
        lse = torch.full((S, n, H), 7.0, device=DEV)
        L.llmcache_attention(q, k, v, out, mods=mine, lse=lse, n_seqs_dev=torch.tensor([count], dtype=torch.int32, device=DEV))
        m = min(count, S)
        if m:
            ro, rl, sp = A.attention(f64(q[:m]), f64(k[:m]), f64(v[:m]), ref)
            check(out[:m], lse[:m], ro, rl, sp, delta(f64(q), f64(k), ref, n), n)
        assert torch.all(out[m:] == 7.0) and torch.all(lse[m:] == 7.0)


def test_other_streams_graphs_and_repetition():
    S, n, H = 2, 200, 4
    q, k, v = fused(S, n, H, H, 95)
    mine, _ = mods_pair(H, causal=True, cap=20.0, bias="table")
    out = torch.zeros((S, n, H, 64), dtype=BF, device=DEV)
    L.llmcache_attention(q, k, v, out, mods=mine)
    torch.cuda.synchronize()
    want = out.clone()
    st = torch.cuda.Stream()
    out.zero_()
    st.wait_stream(torch.cuda.current_stream())
    L.llmcache_attention(q, k, v, out, mods=mine, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.llmcache_attention(q, k, v, out, mods=mine)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)                        # same bits every time


# --------------------------------------------------------------------------------------------------------- paged cache
class Paged:
    """Pages in a shuffled order, a batch with uneven lengths, everything unused set to NaN."""

    def __init__(self, lens, H, HK, page, seed, spare=2, extra=0, interleaved=False):
        self.lens, self.H, self.HK, self.page = lens, H, HK, page
        need = [-(-(n + extra) // page) for n in lens]
        self.num = sum(need) + spare
        ids = np.random.RandomState(seed).permutation(self.num)
        self.width = max(need)
        self.pages = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.pages[b, :m] = ids[at:at + m]
            at += m
        self.free = ids[at:]
        if interleaved:
            both = torch.full((self.num, 2, HK, page, 64), float("nan"), dtype=BF, device=DEV)
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k, self.v = (torch.full((self.num, HK, page, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
        for b, n in enumerate(lens):
            for i, t in enumerate((self.k, self.v)):
                x = rnd(max(n, 1), HK, 64, seed=seed * 100 + b * 2 + i)
                for j0 in range(0, n, page):
                    j1 = min(n, j0 + page)
                    t[int(self.pages[b, j0 // page]), :, :j1 - j0] = x[j0:j1].transpose(0, 1)
        self.pages_dev = torch.tensor(self.pages, device=DEV)

    def oracle(self):
        return A.Cache(f64(self.k), f64(self.v))

    def handle(self, max_rows, **kw):
        return L.KVCache(self.k, self.v, heads=self.H, max_seqs=len(self.lens), max_rows=max_rows, max_len=self.width * self.page, **kw)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def run_chunk(p, rows, mine, ref, *, seed, weights=None, decay=1.0, positions=None, first=None, store=True, tail=0, cache=None,
              longest=None):
    """One call against the oracle; returns (q, out, lse, weights)."""
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    T = int(cu[-1]) + tail
    m = rnd(T, p.H + 2 * p.HK, 64, seed=seed)
    m[:, :p.H] *= 2
    q, kn, vn = m[:, :p.H], m[:, p.H:p.H + p.HK], m[:, p.H + p.HK:]
    out = torch.full((T, p.H, 64), 7.0, dtype=BF, device=DEV)
    lse = torch.full((T, p.H), 7.0, device=DEV)
    c = p.oracle()
    w = None if weights is None else weights.clone()
    pos = None if positions is None else positions.clone()
    kv = cache or p.handle(T)
    kv.attention(q, out, cu_rows=i32(cu), lens=i32(p.lens), pages=p.pages_dev, longest=max(rows) if longest is None else longest,
                 k_new=kn if store else None, v_new=vn if store else None, lse=lse, mods=mine, weights=w, decay=decay,
                 positions=pos, first=None if first is None else i32(first))
    torch.cuda.synchronize()
    assert kv.status() == L.OK
    rw, rp = None if weights is None else f64(weights), None if positions is None else positions.cpu().numpy().copy()
    ro, rl, sp, written = A.chunk(c, f64(q), ref, cu, p.lens, p.pages, f64(kn) if store else None, f64(vn) if store else None,
                                  rw, decay, rp, first)
    n = max(p.lens)
    far = n if positions is None else int(positions.max()) + n + (max(first) if first else 0)
    d = delta(f64(q), c.k, ref, far)
    check(out, lse, ro, rl, sp, d, n, rows=written)
    assert torch.all(out[int(cu[-1]):] == 7.0) and torch.all(lse[int(cu[-1]):] == 7.0)       # rows behind the last sequence
    assert np.array_equal(f64(p.k), c.k, equal_nan=True) and np.array_equal(f64(p.v), c.v, equal_nan=True)
    if positions is not None:
        assert np.array_equal(pos.cpu().numpy(), rp)
    if weights is not None:
        got = f64(w)
        # each of the summed softmax values is relatively exact (see above); decay * w and the sum round once each
        terms = max(rows) * (p.H // p.HK)
        # (f32 has no normal numbers below 2^-126 and the exponential flushes there: each of the `terms` summed values may
        # lose up to 2^-126, so the sum up to terms * 2^-126)
        tol = rw * (2 * d + 2.0 ** -20 + (n + terms) * 2.0 ** -24) + terms * 2.0 ** -126
        assert np.all(np.abs(got - rw) <= tol), float(np.max(np.abs(got - rw) - tol))
    if cache is None:
        kv.close()
    return q, out, lse, w


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("rows", [[1, 1, 1], [5, 1, 40]])
def test_chunk_page_sizes(page, rows):
    p = Paged([1, 130, 291], 4, 2, page, 7, interleaved=page == 64)
    rows = [min(r, n) for r, n in zip(rows, p.lens)]
    mine, ref = mods_pair(4, causal=True)
    run_chunk(p, rows, mine, ref, seed=page)


@pytest.mark.parametrize("H,HK", [(1, 1), (12, 12), (8, 1), (6, 2), (7, 1), (16, 4), (40, 1)])
@pytest.mark.parametrize("rows", [1, 2, 3, 17])
def test_chunk_head_layouts(H, HK, rows):
    p = Paged([140, 64, 77], H, HK, 16, 8)
    mine, ref = mods_pair(H, causal=True, bias="slopes")
    w = torch.zeros((3, HK, p.width * 16), device=DEV)
    run_chunk(p, [rows] * 3, mine, ref, seed=H * 10 + rows, weights=w, decay=0.0)


@pytest.mark.parametrize("rows", [1, 4, 33, 130, 257])
@pytest.mark.parametrize("cap,bias", [(0.0, None), (30.0, "slopes"), (5.0, "table")])
@pytest.mark.parametrize("causal", [True, False])
def test_chunk_modifiers(rows, cap, bias, causal):
    p = Paged([257, 300], 4, 2, 32, 9)
    mine, ref = mods_pair(4, causal=causal, cap=cap, bias=bias)
    w = torch.rand((2, 2, p.width * 32), device=DEV)
    run_chunk(p, [rows, max(1, rows - 1)], mine, ref, seed=rows, weights=w, decay=0.5)


@pytest.mark.parametrize("rows", [1, 9])
def test_chunk_long_cache_is_split_and_joined(rows):
    p = Paged([5003, 1, 2049], 4, 4, 64, 10)
    mine, ref = mods_pair(4, causal=True, cap=50.0)
    w = torch.zeros((3, 4, p.width * 64), device=DEV)
    run_chunk(p, [rows, 1, rows], mine, ref, seed=20 + rows, weights=w, decay=1.0)


@pytest.mark.parametrize("rows", [[0, 3, 0, 1], [2, 0, 0, 0], [0, 0, 0, 5]])
def test_chunk_sequences_without_rows_rows_behind_and_stored_keys(rows):
    p = Paged([4, 90, 17, 33], 4, 2, 16, 11)
    mine, ref = mods_pair(4, causal=True)
    w = torch.rand((4, 2, p.width * 16), device=DEV)
    run_chunk(p, rows, mine, ref, seed=31, tail=6, weights=w, decay=0.25)
    run_chunk(p, rows, mine, ref, seed=32, tail=1, store=False)
    run_chunk(p, rows, None, A.Mods(causal=True), seed=33, longest=0)


@pytest.mark.parametrize("rows", [1, 20])
def test_chunk_positions_after_an_eviction(rows):
    p = Paged([70, 140], 4, 2, 16, 12)
    pos = torch.cumsum(torch.randint(1, 9, (2, 2, p.width * 16), device=DEV), -1).to(torch.int32)
    for bias in ("slopes", "table"):
        mine, ref = mods_pair(4, causal=True, bias=bias, reach=64)
        run_chunk(p, [rows, rows], mine, ref, seed=34, positions=pos, first=[700, 1400])
    run_chunk(p, [rows, rows], mine, ref, seed=35, positions=pos)


@pytest.mark.parametrize("rows", [1, 30, 140])
def test_chunk_pages_that_are_missing_and_shared(rows):
    p = Paged([200, 180], 4, 2, 16, 13)
    p.pages[0, 2], p.pages[0, 5], p.pages[1, 3] = -1, p.num, 2 ** 31 - 1       # nobody sees those slots
    p.pages[1, 0:2] = p.pages[0, 0:2]                                         # a shared prefix
    p.pages_dev = torch.tensor(p.pages, device=DEV)
    mine, ref = mods_pair(4, causal=True)
    w = torch.rand((2, 2, p.width * 16), device=DEV)
    run_chunk(p, [rows, min(rows, 100)], mine, ref, seed=40, weights=w, decay=0.5)


def test_chunk_lengths_beyond_the_table_and_more_rows_than_slots():
    p = Paged([64, 48], 2, 2, 16, 14)
    mine, ref = mods_pair(2, causal=True)
    p.lens = [1000, 48]                                  # taken as the table's four pages
    run_chunk(p, [3, 1], mine, ref, seed=41)
    p.lens = [2, 48]                                     # five rows for two slots: the first three see nothing, are not stored
    q, out, lse, _ = run_chunk(p, [5, 1], mine, ref, seed=42)
    assert not out[:3].any() and torch.all(lse[:3] == float("-inf"))
    p.lens = [0, 48]
    run_chunk(p, [2, 1], mine, ref, seed=43)


def test_chunk_pages_beyond_four_gigabytes():
    H, page = 2, 128
    num = (5 << 30) // (H * page * 128) + 8              # 5 GiB per array: byte and element offsets pass 32 bits
    k, v = (torch.empty((num, H, page, 64), dtype=BF, device=DEV) for _ in range(2))
    lens = [page + 5]
    pages = np.array([[num - 1, num // 2 + 3]], np.int32)
    x = rnd(2, lens[0], H, 64, seed=50)
    for t, src in ((k, x[0]), (v, x[1])):
        t[num - 1] = src[:page].transpose(0, 1)
        t[num // 2 + 3, :, :5] = src[page:].transpose(0, 1)
    for rows in (1, 100):
        q = rnd(rows, H, 64, seed=51)
        out = torch.zeros((rows, H, 64), dtype=BF, device=DEV)
        kv = L.KVCache(k, v, heads=H, max_seqs=1, max_rows=rows, max_len=2 * page)
        w = torch.zeros((1, H, 2 * page), device=DEV)
        kv.attention(q, out, cu_rows=i32([0, rows]), lens=i32(lens), pages=i32(pages), weights=w, decay=0.0)
        c = A.Cache(np.zeros((2, H, page, 64)), np.zeros((2, H, page, 64)))
        for t, dst in ((k, c.k), (v, c.v)):
            dst[0], dst[1, :, :5] = f64(t[num - 1]), f64(t[num // 2 + 3, :, :5])
        rw = np.zeros(w.shape)
        ro, rl, sp, _ = A.chunk(c, f64(q), A.Mods(causal=True), [0, rows], lens, np.array([[0, 1]]), weights=rw)
        d = delta(f64(q), c.k, A.Mods(), lens[0])
        check(out, None, ro, rl, sp, d, lens[0])
        assert np.allclose(f64(w), rw, rtol=2 * d + 2.0 ** -12, atol=0)
        # eviction reads and writes out there, too
        nl = torch.zeros(1, dtype=torch.int32, device=DEV)
        kept = torch.zeros((1, H, 64), dtype=torch.int32, device=DEV)
        kv.evict(lens=i32(lens), pages=i32(pages), weights=w, new_pages=i32([[num - 2]]), new_lens=nl, budget=64, kept=kept)
        torch.cuda.synchronize()
        for h in range(H):
            assert torch.equal(k[num - 2, h, :64], x[0][kept[0, h].long(), h])
        kv.close()


def test_chunk_streams_graphs_and_a_shared_workspace():
    p = Paged([300, 41], 4, 2, 16, 15)
    T = 6
    m = rnd(T, 8, 64, seed=60)
    q, kn, vn = m[:, :4], m[:, 4:6], m[:, 6:]
    kv = p.handle(T)
    ws = torch.zeros(L.llmcache_kv_bytes(kv.desc) + 256, dtype=torch.uint8, device=DEV)
    kv2 = p.handle(T, workspace=ws[(-ws.data_ptr()) % 256:])
    out = torch.zeros((T, 4, 64), dtype=BF, device=DEV)
    w = torch.zeros((2, 2, p.width * 16), device=DEV)
    args = dict(cu_rows=i32([0, 2, 6]), lens=i32(p.lens), pages=p.pages_dev, longest=4, k_new=kn, v_new=vn, weights=w, decay=0.0)
    kv.attention(q, out, **args)
    torch.cuda.synchronize()
    want, want_w = out.clone(), w.clone()
    st = torch.cuda.Stream()
    for cache in (kv, kv2):
        out.zero_()
        st.wait_stream(torch.cuda.current_stream())
        cache.attention(q, out, stream=st, **args)
        st.synchronize()
        assert torch.equal(out, want) and torch.equal(w, want_w)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.attention(q, out, **args)
        out.zero_()
        w.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(w, want_w)
        cache.close()


def test_chunk_refusals():
    p = Paged([30, 20], 4, 2, 16, 16)
    kv = p.handle(8)
    q = rnd(4, 4, 64, seed=61)
    out = torch.zeros_like(q)
    good = dict(cu_rows=i32([0, 2, 4]), lens=i32(p.lens), pages=p.pages_dev)

    def status(q=q, out=out, **kw):
        with pytest.raises(L.LLMCacheError) as e:
            kv.attention(q, out, **{**good, **kw})
        return e.value.status

    big = rnd(9, 4, 64, seed=62)
    assert status(big, torch.zeros_like(big)) == L.ERR_SHAPE                        # more rows than max_rows
    assert status(longest=5) == L.ERR_SHAPE
    assert status(cu_rows=i32([0, 4])) == L.ERR_SHAPE
    assert status(lens=i32([1, 2, 3]), cu_rows=i32([0, 1, 2, 3]), pages=i32([[0]] * 3)) == L.ERR_SHAPE      # more than max_seqs
    assert status(k_new=rnd(4, 2, 64, seed=1)) == L.ERR_ARG
    assert status(k_new=rnd(4, 4, 64, seed=1), v_new=rnd(4, 4, 64, seed=1)) == L.ERR_SHAPE
    assert status(lens=torch.tensor([30, 20], device=DEV)) == L.ERR_ARG             # int64
    assert status(weights=torch.zeros((2, 2, 16), device=DEV)) == L.ERR_SHAPE       # rows shorter than the tables
    assert status(weights=torch.zeros((2, 2, 32), device=DEV), decay=1.5) == L.ERR_ARG
    assert status(weights=torch.zeros((2, 2, 32), device=DEV), decay=float("nan")) == L.ERR_ARG
    assert status(mods=L.make_score_mods(causal=True, doc=torch.zeros((2, 2), dtype=torch.int32, device=DEV))) == L.ERR_UNSUPPORTED
    kv.attention(q[:0], out[:0], **{**good, "cu_rows": i32([0, 0, 0])})             # nothing to do
    assert kv.status() == L.OK
    kv.close()


# ------------------------------------------------------------------------------------------------------------ eviction
@pytest.mark.parametrize("page,budget,recent,sinks,lens", [
    (16, 20, 5, 2, [20, 21, 90, 7]), (32, 1, 0, 0, [40, 1, 2, 200]), (64, 64, 64, 0, [300, 65, 64, 63]), (16, 50, 0, 50, [51, 200, 3, 0]),
    (128, 300, 20, 4, [1500, 1023, 1025, 2500]), (256, 7, 3, 4, [3000, 256, 8, 257])])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(page, budget, recent, sinks, lens, kind):
    HK = 3
    p = Paged(lens, HK, HK, page, 17, spare=len(lens) * (-(-budget // page)) + 2)
    slots = p.width * page
    g = np.random.RandomState(5)
    w = np.exp(g.randn(len(lens), HK, slots)).astype(np.float32)
    if kind == "ties":
        w = g.randint(0, 3, w.shape).astype(np.float32)
    if kind == "odd":
        w[g.rand(*w.shape) < 0.2] = np.nan
        w[g.rand(*w.shape) < 0.2] = -1.0
        w[g.rand(*w.shape) < 0.1] = np.inf
        w[g.rand(*w.shape) < 0.1] = 1e-42
    pos = None if kind == "ties" else np.cumsum(g.randint(1, 4, w.shape), -1).astype(np.int32)[..., ::1 if kind == "spread" else -1].copy()
    new = p.free[:len(lens) * (-(-budget // page))].reshape(len(lens), -1).astype(np.int32).copy()
    kept = A.evict(lens, w, pos, budget, recent, sinks)
    k0, v0 = p.k.clone(), p.v.clone()
    kv = p.handle(8)
    W, lens_dev = torch.tensor(w, device=DEV), i32(lens)
    nw, npos = torch.full((len(lens), HK, budget + 3), 7.0, device=DEV), torch.full((len(lens), HK, budget + 3), 7, dtype=torch.int32, device=DEV)
    got = torch.full((len(lens), HK, budget), 9, dtype=torch.int32, device=DEV)
    kv.evict(lens=lens_dev, pages=p.pages_dev, weights=W, positions=None if pos is None else torch.tensor(pos, device=DEV),
             new_pages=torch.tensor(new, device=DEV), new_lens=lens_dev, budget=budget, recent=recent, sinks=sinks, new_weights=nw,
             new_positions=npos, kept=got)
    torch.cuda.synchronize()
    assert kv.status() == L.OK and lens_dev.tolist() == [min(n, budget) for n in lens]
    ek, ev = k0.clone(), v0.clone()
    for s in range(len(lens)):
        for h in range(HK):
            js = kept[s][h]
            assert got[s, h].tolist() == js.tolist() + [-1] * (budget - len(js))
            want = np.concatenate([w[s, h, js], np.zeros(budget - len(js)), np.full(3, 7)]).astype(np.float32)
            assert np.array_equal(nw[s, h].cpu().numpy(), want, equal_nan=True)
            wp = js if pos is None else pos[s, h, js]
            assert npos[s, h].tolist() == wp.tolist() + [0] * (budget - len(js)) + [7] * 3
            for i, j in enumerate(js):
                src, dst = int(p.pages[s, j // page]), int(new[s, i // page])
                ek[dst, h, i % page], ev[dst, h, i % page] = k0[src, h, j % page], v0[src, h, j % page]
    assert torch.equal(p.k.view(torch.int16), ek.view(torch.int16)) and torch.equal(p.v.view(torch.int16), ev.view(torch.int16))
    kv.close()


def test_evict_more_slots_than_one_block_keeps_in_shared_memory():
    n, HK, page, budget = 60000, 2, 256, 5000
    num = -(-n // page) + -(-budget // page)
    k = rnd(num, HK, page, 64, seed=70)
    v = k.clone()
    kv = L.KVCache(k, v, heads=HK, max_seqs=1, max_rows=1, max_len=n)
    w = torch.rand((1, HK, n), device=DEV)
    kept = torch.zeros((1, HK, budget), dtype=torch.int32, device=DEV)
    nl = torch.zeros(1, dtype=torch.int32, device=DEV)
    kv.evict(lens=i32([n]), pages=i32([list(range(-(-n // page)))]), weights=w, new_pages=i32([list(range(-(-n // page), num))]), new_lens=nl,
             budget=budget, recent=100, sinks=3, kept=kept)
    ref = A.evict([n], f64(w), None, budget, 100, 3)
    for h in range(HK):
        assert np.array_equal(kept[0, h].cpu().numpy(), ref[0][h])
        assert torch.equal(k[-(-n // page) + budget // page, h, budget % page - 1], k[int(kept[0, h, -1]) // page, h, int(kept[0, h, -1]) % page])
    kv.close()


def test_evict_refusals():
    p = Paged([30, 20], 2, 2, 16, 18)
    kv = p.handle(4)
    w, nl = torch.zeros((2, 2, 32), device=DEV), i32([0, 0])
    good = dict(lens=i32(p.lens), pages=p.pages_dev, weights=w, new_pages=i32([[0], [1]]), new_lens=nl, budget=16)

    def status(**kw):
        with pytest.raises(L.LLMCacheError) as e:
            kv.evict(**{**good, **kw})
        return e.value.status

    assert status(budget=0) == L.ERR_SHAPE and status(budget=17) == L.ERR_SHAPE and status(budget=33) == L.ERR_SHAPE
    assert status(recent=10, sinks=7) == L.ERR_SHAPE and status(weights=w[:, :, :16].contiguous()) == L.ERR_SHAPE
    assert status(weights=w[:, :1].contiguous()) == L.ERR_SHAPE and status(weights=w.double()) == L.ERR_ARG
    assert status(new_weights=torch.zeros((2, 2, 15), device=DEV)) == L.ERR_SHAPE
    assert status(kept=torch.zeros((2, 2, 15), dtype=torch.int32, device=DEV)) == L.ERR_SHAPE
    kv.close()


# ---------------------------------------------------------------------------------------------------- used together
def test_prompt_tokens_eviction_and_more_tokens():
    """A prompt with recorded weights, single tokens, an eviction by what they recorded, and tokens after it."""
    H, HK, page, budget = 4, 2, 16, 48
    mine, ref = mods_pair(H, causal=True, bias="slopes", cap=30.0)
    lens = np.array([90, 61])
    num = 40
    k, v = (torch.full((num, HK, page, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    c = A.Cache(f64(k), f64(v))
    ids = np.random.RandomState(3).permutation(num).astype(np.int32)
    pages, fresh = ids[:16].reshape(2, 8), ids[16:24].reshape(2, 4)
    kv = L.KVCache(k, v, heads=H, max_seqs=2, max_rows=200, max_len=128)
    w, rw = torch.zeros((2, HK, 128), device=DEV), np.zeros((2, HK, 128))
    pos, rpos = torch.zeros((2, HK, 128), dtype=torch.int32, device=DEV), np.zeros((2, HK, 128), np.int32)
    seen = np.zeros(2, int)
    cur, cur_w, cur_pos, length = pages, w, pos, np.zeros(2, int)
    for step, rows in enumerate([lens, [1, 1], [1, 1], "evict", [1, 1], [7, 1], [1, 1]]):
        if isinstance(rows, str):
            kept = A.evict(length, rw, rpos, budget, 8, 4)
            nw, npos = torch.zeros((2, HK, 128), device=DEV), torch.zeros((2, HK, 128), dtype=torch.int32, device=DEV)
            got, nl = torch.zeros((2, HK, budget), dtype=torch.int32, device=DEV), i32([0, 0])
            kv.evict(lens=i32(length), pages=i32(cur), weights=cur_w, positions=cur_pos, new_pages=i32(fresh), new_lens=nl, budget=budget, recent=8,
                     sinks=4, new_weights=nw, new_positions=npos, kept=got)
            rw2, rpos2 = np.zeros_like(rw), np.zeros_like(rpos)
            for s in range(2):
                for h in range(HK):
                    # the recorded weights are f32: the order may differ from the oracle's where two are as close as
                    # their rounding, so the oracle continues with what was kept
                    js = got[s, h].cpu().numpy()
                    assert len(set(js.tolist()) & set(kept[s][h].tolist())) >= budget - 1
                    rw2[s, h, :budget], rpos2[s, h, :budget] = rw[s, h, js], rpos[s, h, js]
                    for i, j in enumerate(js):
                        a, b = c.place(cur[s], j), c.place(fresh[s], i)
                        c.k[b[0], h, b[1]], c.v[b[0], h, b[1]] = c.k[a[0], h, a[1]], c.v[a[0], h, a[1]]
            cur, cur_w, cur_pos, rw, rpos = fresh, nw, npos, rw2, rpos2
            length = np.array(nl.tolist())
            assert length.tolist() == [budget, budget]
            continue
        rows = np.array(rows)
        cu = np.concatenate([[0], np.cumsum(rows)])
        length = length + rows
        m = rnd(int(cu[-1]), H + 2 * HK, 64, seed=500 + step)
        q, kn, vn = m[:, :H], m[:, H:H + HK], m[:, H + HK:]
        out, lse = torch.zeros((int(cu[-1]), H, 64), dtype=BF, device=DEV), torch.zeros((int(cu[-1]), H), device=DEV)
        kv.attention(q, out, cu_rows=i32(cu), lens=i32(length), pages=i32(cur), longest=int(rows.max()), k_new=kn, v_new=vn, lse=lse, mods=mine,
                     weights=cur_w, positions=cur_pos, first=i32(seen))
        torch.cuda.synchronize()
        ro, rl, sp, _ = A.chunk(c, f64(q), ref, cu, length, cur, f64(kn), f64(vn), rw, 1.0, rpos, seen)
        d = delta(f64(q), c.k, ref, 128)
        check(out, lse, ro, rl, sp, d, 128)
        assert np.array_equal(cur_pos.cpu().numpy(), rpos)
        seen = seen + rows
    assert kv.status() == L.OK
    kv.close()


def layer_pair(n, d, heads, ffn, S, pre_ln=True, causal=True, seed=21):
    w = synth.layer_weights(d, ffn, seed, DEV)
    for key in ("w_qkv", "w_o", "w_1", "w_2"):
        w[key] = (w[key].float() * 3.0).to(BF)
    return w, L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=causal, tanh_gelu=pre_ln)


def close_layers(a, b):
    """Both keep the same intermediates in bf16 and sum in another order: the tolerance that the layer tests derive."""
    a, b = f64(a), f64(b)
    assert np.sqrt(np.mean((a - b) ** 2)) <= 6e-3 * np.sqrt(np.mean(b ** 2))
    assert np.all(np.abs(a - b) <= 4 * 2.0 ** -8 * np.abs(b) + 0.02 * np.sqrt(np.mean(b ** 2)))


@pytest.mark.parametrize("pre_ln", [True, False])
@pytest.mark.parametrize("page", [16, 64])
def test_layer_extend_equals_the_layer_on_the_whole_sequence(pre_ln, page):
    n, d, heads, S = 130, 192, 3, 2
    _, layer = layer_pair(n, d, heads, 320, S, pre_ln=pre_ln)
    x = rnd(S, n, d, seed=22)
    want = torch.zeros_like(x)
    layer.forward(x, want)
    num = S * (-(-n // page))
    k, v = (torch.full((num, heads, page, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    kv = L.KVCache(k, v, heads=heads, max_seqs=S, max_rows=S * n, max_len=n)
    pages = i32(np.random.RandomState(1).permutation(num).reshape(S, -1))
    got = torch.full((S, n, d), 7.0, dtype=BF, device=DEV)
    at = [0, 0]
    for rows in ([100, 60], [1, 1], [0, 40], [29, 29]):
        cu = np.concatenate([[0], np.cumsum(rows)])
        xs = torch.cat([x[s, at[s]:at[s] + rows[s]] for s in range(S)] + [x[0, :2]])             # two rows behind the last sequence
        out = torch.full_like(xs, 7.0)
        at = [a + r for a, r in zip(at, rows)]
        layer.extend(kv, xs, out, cu_rows=i32(cu), lens=i32(at), pages=pages, longest=max(rows))
        torch.cuda.synchronize()
        assert torch.all(out[int(cu[-1]):] == 7.0)
        for s in range(S):
            got[s, at[s] - rows[s]:at[s]] = out[int(cu[s]):int(cu[s + 1])]
    assert layer.status() == L.OK and kv.status() == L.OK
    close_layers(got, want)
    kv.close()
    layer.close()


@pytest.mark.parametrize("pre_ln", [True, False])
def test_layer_with_score_modifiers(pre_ln):
    """Plain modifiers change nothing; documents packed into a row give each document what it has alone."""
    n, d, heads, S = 130, 192, 3, 2
    _, layer = layer_pair(n, d, heads, 320, S, pre_ln=pre_ln, causal=pre_ln)
    x = rnd(S, n, d, seed=23)
    plain, out = torch.zeros_like(x), torch.zeros_like(x)
    layer.forward(x, plain)
    layer.score_mods(L.make_score_mods(causal=pre_ln))
    layer.forward(x, out)
    torch.cuda.synchronize()
    close_layers(out, plain)
    doc = torch.zeros((S, n), dtype=torch.int32, device=DEV)
    doc[:, 57:] = 1
    doc[1, 120:] = -1
    layer.score_mods(L.make_score_mods(causal=pre_ln, doc=doc))
    layer.forward(x, out)
    _, small = layer_pair(57, d, heads, 320, S, pre_ln=pre_ln, causal=pre_ln)
    alone = torch.zeros((S, 57, d), dtype=BF, device=DEV)
    small.forward(x[:, :57].contiguous(), alone)
    torch.cuda.synchronize()
    close_layers(out[:, :57], alone)
    layer.score_mods(None)
    again = torch.zeros_like(x)
    layer.forward(x, again)
    torch.cuda.synchronize()
    assert torch.equal(again, plain) and layer.status() == L.OK
    with pytest.raises(L.LLMCacheError) as e:
        layer.score_mods(L.make_score_mods(causal=not pre_ln))
    assert e.value.status == L.ERR_ARG
    layer.close()
    small.close()


def test_layer_refusals_where_sequences_change_their_places():
    n, d, heads, S = 16, 128, 2, 4
    _, layer = layer_pair(n, d, heads, 256, S)
    _, enc = layer_pair(n, d, heads, 256, S, pre_ln=False, causal=False)
    bank = L.Bank(capacity=8, seq_len=n, d_model=d, fp_dim=d, max_batch=S)
    bufs = L.ProbeBuffers(S, d, DEV)
    x = rnd(S, n, d, seed=24)
    mk = lambda: torch.zeros_like(x)
    layer.score_mods(L.make_score_mods(causal=True, prefix=torch.zeros(S, dtype=torch.int32, device=DEV)))
    a, b, c, e = mk(), mk(), mk(), mk()
    with pytest.raises(L.LLMCacheError) as err:
        L.llmcache_infer([bank.handle], [layer.handle], x, S, None, a, b, c, e, bufs.io)
    assert err.value.status == L.ERR_UNSUPPORTED
    L.llmcache_infer(None, [layer.handle], x, S, None, a, b, c, e, bufs.io)              # without banks nothing moves
    layer.score_mods(L.make_score_mods(causal=True, cap=20.0))
    L.llmcache_infer([bank.handle], [layer.handle], x, S, None, a, b, c, e, bufs.io)     # the same for every sequence
    k = torch.zeros((4, heads, 16, 64), dtype=BF, device=DEV)
    kv = L.KVCache(k, k.clone(), heads=heads, max_seqs=2, max_rows=8, max_len=32)
    wide = L.KVCache(k, k.clone(), heads=2 * heads, max_seqs=2, max_rows=8, max_len=32)
    call = dict(cu_rows=i32([0, 4]), lens=i32([4]), pages=i32([[0, 1]]))
    rows, out = x[0, :4].contiguous(), torch.zeros((4, d), dtype=BF, device=DEV)
    for lay, cache, status in ((enc, kv, L.ERR_UNSUPPORTED), (layer, wide, L.ERR_SHAPE)):
        with pytest.raises(L.LLMCacheError) as err:
            lay.extend(cache, rows, out, **call)
        assert err.value.status == status
    layer.extend(kv, rows, out, **call)
    torch.cuda.synchronize()
    assert layer.status() == L.OK and kv.status() == L.OK and bank.status() == L.OK
    for o in (layer, enc, kv, wide, bank):
        o.close()
