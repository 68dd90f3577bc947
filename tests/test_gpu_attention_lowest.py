"""Distance tables whose entries are the type's lowest value, or not numbers: rows, logarithms and received weights.

Beside an entry of -3.4e38 a score is lost in 32 bits and in 64: rows that see nothing else weigh all keys alike.  Where such an
entry stands beside ordinary ones its key has no weight.  So the tolerances are those of the scores without the
table (see test_gpu_attention.py)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2512_16843_b200 import binding as L
from tests.test_gpu_attention import BF, DEV, Paged, check, delta, f64, fused, i32, rnd, run_attention

pytestmark = pytest.mark.gpu
LOWEST = float(torch.finfo(torch.float32).min)


def low_table(low, reach=64):
    """Head 0 sees the last five distances and has low entries beyond, the others have nothing but low entries."""
    t = torch.full((4, 2 * reach + 1), low, device=DEV)
    t[0, reach - 4:reach + 1] = torch.tensor([0.3, -0.2, 0.0, 0.5, 0.1], device=DEV)
    return t


@pytest.mark.parametrize("low", [LOWEST, float(torch.finfo(torch.bfloat16).min), -3e38])
@pytest.mark.parametrize("causal", [True, False])
def test_whole_sequences(low, causal):
    n = 200
    q, k, v = fused(2, n, 4, 2, 801)
    table = low_table(low)
    out, lse, ro, rl, sp = run_attention(q, k, v, L.make_score_mods(causal=causal, table=table), A.Mods(causal=causal, table=f64(table)))
    d = delta(f64(q), f64(k), A.Mods(), n)
    check(out, None, ro, rl, sp, d, n)
    check(out[:, :, :1], lse[:, :, :1], ro[:, :, :1], rl[:, :, :1], sp[:, :, :1], d + 4 * 2.0 ** -24, n)
    assert torch.all(lse[:, :, 1:] == LOWEST)


# (4 heads on 2; 40 rows over 500 keys: a block's halves share the keys; 150: two query tiles)
@pytest.mark.parametrize("rows", [1, 8, 9, 40, 150])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("positions", [False, True])
def test_rows_and_weights_over_a_cache(rows, causal, positions):
    p = Paged([500, 333], 4, 2, 32, 802)
    table = low_table(LOWEST)
    T = 2 * rows
    m = rnd(T, 8, 64, seed=803)
    q, kn, vn = m[:, :4], m[:, 4:6], m[:, 6:]
    out, lse = torch.zeros((T, 4, 64), dtype=BF, device=DEV), torch.zeros((T, 4), device=DEV)
    w = torch.rand((2, 2, p.width * 32), device=DEV)
    pos = torch.arange(p.width * 32, dtype=torch.int32, device=DEV).expand(2, 2, -1).contiguous() if positions else None
    c, rw, cu = p.oracle(), f64(w), [0, rows, T]
    kv = p.handle(T)
    kv.attention(q, out, cu_rows=i32(cu), lens=i32(p.lens), pages=p.pages_dev, longest=rows, k_new=kn, v_new=vn, lse=lse,
                 mods=L.make_score_mods(causal=causal, table=table), weights=w, decay=0.5, positions=pos)
    torch.cuda.synchronize()
    assert kv.status() == L.OK
    ro, rl, sp, _ = A.chunk(c, f64(q), A.Mods(causal=causal, table=f64(table)), cu, p.lens, p.pages, f64(kn), f64(vn), rw, 0.5,
                            None if pos is None else pos.cpu().numpy().copy())
    n, d = 500, delta(f64(q), c.k, A.Mods(), 500) + 4 * 2.0 ** -24
    check(out, None, ro, rl, sp, d, n)
    check(out[:, :1], lse[:, :1], ro[:, :1], rl[:, :1], sp[:, :1], d, n)
    assert torch.all(lse[:, 1:] == LOWEST)
    tol = rw * (2 * d + 2.0 ** -20 + (n + 2 * rows) * 2.0 ** -24) + 2 * rows * 2.0 ** -126
    assert np.all(np.abs(f64(w) - rw) <= tol), float(np.max(np.abs(f64(w) - rw) - tol))
    kv.close()


@pytest.mark.parametrize("rows", [1, 9, 150])
def test_entries_that_are_not_numbers(rows):
    """They reach the rows that see a key at their distance, and no others."""
    n, reach = 200, 70
    table = torch.zeros((2, 2 * reach + 1), device=DEV)
    table[0, reach - 60] = table[1, 0] = float("nan")    # head 0: keys 60 before the query; head 1: 70 and more before it
    mine, ref = L.make_score_mods(causal=True, table=table), A.Mods(causal=True, table=f64(table))
    q, k, v = fused(1, n, 2, 2, 804)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    assert np.isnan(ro[0, 60:, 0]).all() and np.isnan(ro[0, 70:, 1]).all() and np.isfinite(ro[0, :60]).all()
    d = delta(f64(q), f64(k), A.Mods(), n)
    check(out, lse, ro, rl, np.where(np.isfinite(sp), sp, 0), d, n)
    p = Paged([n, 65], 2, 2, 16, 805)
    o, ls = torch.zeros((rows + 1, 2, 64), dtype=BF, device=DEV), torch.zeros((rows + 1, 2), device=DEV)
    qs = rnd(rows + 1, 2, 64, seed=806)
    kv = p.handle(rows + 1)
    kv.attention(qs, o, cu_rows=i32([0, rows, rows + 1]), lens=i32(p.lens), pages=p.pages_dev, longest=rows, lse=ls, mods=mine)
    torch.cuda.synchronize()
    assert kv.status() == L.OK
    ro, rl, sp, _ = A.chunk(p.oracle(), f64(qs), ref, [0, rows, rows + 1], p.lens, p.pages)
    assert np.isnan(ro[-1, 0]).all() and np.isfinite(ro[-1, 1]).all() and np.isnan(ro[rows - 1]).all()
    check(o, ls, ro, rl, np.where(np.isfinite(sp), sp, 0), d, n)
    kv.close()
