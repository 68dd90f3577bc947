"""Calls whose `longest` is smaller than a sequence's rows: the rows beyond it are stored, not computed.  Tolerances: see
test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2512_16843_b200 import binding as L
from tests.test_gpu_attention import BF, DEV, Paged, check, close_layers, delta, f64, i32, layer_pair, mods_pair, rnd

pytestmark = pytest.mark.gpu


# (4 heads on 2: up to 8 rows of a sequence are few)
@pytest.mark.parametrize("rows,longest", [([3, 1], 1), ([9, 40], 8), ([150, 7], 20), ([40, 200], 130)])
@pytest.mark.parametrize("bias", [None, "table"])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_beyond_the_longest_are_stored_and_left_alone(rows, longest, bias, causal):
    p = Paged([260, 300], 4, 2, 32, 61)
    mine, ref = mods_pair(4, causal=causal, bias=bias, reach=64)
    cu = np.concatenate([[0], np.cumsum(rows)])
    T = int(cu[-1])
    m = rnd(T, 8, 64, seed=62)
    q, kn, vn = m[:, :4], m[:, 4:6], m[:, 6:]
    out, lse = torch.full((T, 4, 64), 7.0, dtype=BF, device=DEV), torch.full((T, 4), 7.0, device=DEV)
    w = torch.rand((2, 2, p.width * 32), device=DEV)
    g = np.random.RandomState(63)
    pos = torch.tensor(np.cumsum(g.randint(1, 3, w.shape), -1), dtype=torch.int32, device=DEV)
    first = [int(pos.max()) + 1] * 2
    c, rw, rp = p.oracle(), f64(w), pos.cpu().numpy().copy()
    kv = p.handle(T)
    kv.attention(q, out, cu_rows=i32(cu), lens=i32(p.lens), pages=p.pages_dev, longest=longest, k_new=kn, v_new=vn, lse=lse, mods=mine,
                 weights=w, decay=0.5, positions=pos, first=i32(first))
    torch.cuda.synchronize()
    assert kv.status() == L.OK
    ro, rl, sp, written = A.chunk(c, f64(q), ref, cu, p.lens, p.pages, f64(kn), f64(vn), rw, 0.5, rp, first, longest)
    assert written.sum() == sum(min(r, longest) for r in rows) < T
    n = 300
    d = delta(f64(q), c.k, ref, first[0] + n)
    check(out, lse, ro, rl, sp, d, n, rows=written)
    assert torch.all(out[~torch.tensor(written)] == 7.0) and torch.all(lse[~torch.tensor(written)] == 7.0)
    assert np.array_equal(f64(p.k), c.k, equal_nan=True) and np.array_equal(f64(p.v), c.v, equal_nan=True)
    assert np.array_equal(pos.cpu().numpy(), rp)
    terms = longest * 2
    assert np.all(np.abs(f64(w) - rw) <= rw * (2 * d + 2.0 ** -20 + (n + terms) * 2.0 ** -24) + terms * 2.0 ** -126)
    kv.close()


@pytest.mark.parametrize("rows,longest", [([4, 2], 2), ([50, 30], 40)])
def test_layer_extend_keeps_nothing_of_earlier_calls(rows, longest):
    """Rows beyond the longest have the layer's result for an attention of zero, whatever ran before, and later rows see
    their keys and values."""
    n, d, heads, S = 130, 192, 3, 2
    w, layer = layer_pair(n, d, heads, 320, S)
    w0 = dict(w, w_o=torch.zeros_like(w["w_o"]))                       # the same layer without its attention
    plain = L.Layer(w0, heads=heads, seq_len=n, max_seqs=S, pre_ln=True, causal=True, tanh_gelu=True)
    cu = np.concatenate([[0], np.cumsum(rows)])
    T = int(cu[-1])
    x = rnd(S, n, d, seed=64)
    xs = torch.cat([x[s, :rows[s]] for s in range(S)])
    pages = i32(np.arange(2 * S * 9).reshape(2, S, 9))
    after = [r + 1 for r in rows]
    xn = torch.stack([x[s, rows[s]] for s in range(S)])
    outs, nexts = [], []
    for size in (longest, 0):
        layer.forward(x * 3, torch.zeros_like(x))                      # leaves its attention in the layer's scratch
        k, v = (torch.full((S * 9, heads, 16, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
        kv = L.KVCache(k, v, heads=heads, max_seqs=S, max_rows=T, max_len=n)
        out, nxt = torch.full_like(xs, 7.0), torch.full_like(xn, 7.0)
        layer.extend(kv, xs, out, cu_rows=i32(cu), lens=i32(rows), pages=pages[0], longest=size)
        layer.extend(kv, xn, nxt, cu_rows=i32([0, 1, 2]), lens=i32(after), pages=pages[0], longest=1)
        torch.cuda.synchronize()
        assert kv.status() == L.OK
        outs.append(out)
        nexts.append(nxt)
        kv.close()
    base = torch.zeros((S, n, d), dtype=BF, device=DEV)
    plain.forward(x, base)
    torch.cuda.synchronize()
    assert layer.status() == L.OK
    for s in range(S):
        mid, end = int(cu[s]) + min(rows[s], longest), int(cu[s + 1])
        close_layers(outs[0][int(cu[s]):mid], outs[1][int(cu[s]):mid])
        if mid < end:
            close_layers(outs[0][mid:end], base[s, longest:rows[s]])
    assert torch.equal(nexts[0], nexts[1])
    layer.close()
    plain.close()
