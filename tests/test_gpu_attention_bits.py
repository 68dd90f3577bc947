"""Bits of capped scores: a row's result is a function of what the row sees, and of nothing that lies beside it (keys of the future
and of other documents, slots that nobody wrote, places of a tile without a row)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2512_16843_b200 import binding as L
from tests.test_gpu_attention import BF, DEV, Paged, check, delta, f64, fused, i32, mods_pair, rnd, run_attention

pytestmark = pytest.mark.gpu
# factors for keys that are not seen: arguments of the tanh up to about 0.2, 0.6 and 3 at a cap of 30
FACTORS = (1.0, 3.0, 15.0)


def attend(q, k, v, mods):
    out = torch.zeros(q.shape, dtype=BF, device=DEV)
    lse = torch.zeros(q.shape[:3], device=DEV)
    L.llmcache_attention(q, k, v, out, mods=mods, lse=lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("H,HK", [(2, 2), (4, 1), (6, 2)])
@pytest.mark.parametrize("bias", [None, "slopes", "table"])
def test_rows_before_a_change_of_the_future(H, HK, bias):
    n, cut = 300, 200
    q, k, v = (t.clone() for t in fused(2, n, H, HK, 401))
    mine, _ = mods_pair(H, causal=True, cap=30.0, bias=bias, reach=64)
    k0 = k[:, cut:].clone()
    got = []
    for f in FACTORS:
        k[:, cut:] = k0 * f
        got.append(attend(q, k, v, mine))
    k[:, cut:] = float("nan")
    got.append(attend(q, k, v, mine))
    for out, lse in got[1:]:
        assert torch.equal(out[:, :cut], got[0][0][:, :cut]) and torch.equal(lse[:, :cut], got[0][1][:, :cut])
    assert not torch.equal(got[1][1][:, cut:], got[0][1][:, cut:])


@pytest.mark.parametrize("causal", [False, True])
def test_documents_beside_a_change_in_another(causal):
    n, H = 260, 4
    q, k, v = (t.clone() for t in fused(2, n, H, 2, 402))
    doc = torch.zeros((2, n), dtype=torch.int32, device=DEV)
    doc[:, 90:170], doc[:, 170:] = 1, 2
    mine, _ = mods_pair(H, causal=causal, cap=30.0, bias="slopes", doc=doc)
    k0 = k[:, 90:170].clone()
    got = []
    for f in FACTORS:
        k[:, 90:170] = k0 * f
        got.append(attend(q, k, v, mine))
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[90:170] = False
    for out, lse in got[1:]:
        assert torch.equal(out[:, keep], got[0][0][:, keep]) and torch.equal(lse[:, keep], got[0][1][:, keep])


@pytest.mark.parametrize("H,HK,rows", [(4, 2, 3), (4, 2, 40), (6, 2, 40), (4, 4, 150)])
@pytest.mark.parametrize("bias", [None, "slopes"])
def test_slots_behind_the_end_and_later_rows(H, HK, rows, bias):
    """What never-written slots hold changes neither rows nor weights; what the last row brings changes no row before it."""
    lens = [300, 213]
    got = []
    for fill, f in ((float("nan"), 1.0), (0.0, 3.0), (9.0, 15.0), (-3e38, 1.0)):
        p = Paged(lens, H, HK, 32, 403)
        for t in (p.k, p.v):
            t[torch.isnan(t)] = fill
        mine, _ = mods_pair(H, causal=True, cap=30.0, bias=bias)
        m = rnd(2 * rows, H + 2 * HK, 64, seed=404)
        m[:, :H] *= 2
        m[[rows - 1, 2 * rows - 1], H:H + HK] *= f
        out, lse = torch.zeros((2 * rows, H, 64), dtype=BF, device=DEV), torch.zeros((2 * rows, H), device=DEV)
        w = torch.zeros((2, HK, p.width * 32), device=DEV)
        kv = p.handle(2 * rows)
        kv.attention(m[:, :H], out, cu_rows=i32([0, rows, 2 * rows]), lens=i32(lens), pages=p.pages_dev, longest=rows, k_new=m[:, H:H + HK],
                     v_new=m[:, H + HK:], lse=lse, mods=mine, weights=w, decay=0.0)
        torch.cuda.synchronize()
        assert kv.status() == L.OK
        got.append((f, out, lse, w))
        kv.close()
    first = [r for r in range(2 * rows) if r % rows != rows - 1]
    for f, out, lse, w in got[1:]:
        assert torch.equal(out[first], got[0][1][first]) and torch.equal(lse[first], got[0][2][first])
    assert torch.equal(got[3][1], got[0][1]) and torch.equal(got[3][2], got[0][2]) and torch.equal(got[3][3], got[0][3])


@pytest.mark.parametrize("H,HK", [(6, 2), (7, 1), (12, 1), (96, 2)])
def test_groups_that_leave_places_of_a_tile_without_a_row(H, HK):
    """Same bits whatever an earlier call left on the SMs."""
    q, k, v = fused(2, 150, H, HK, 405)
    mine, ref = mods_pair(H, causal=True, cap=30.0, bias="slopes")
    want = attend(q, k, v, mine)
    for f in (0.0, 40.0, 3e38):
        big = rnd(40, 256, 16, 64, seed=406).float().clamp(-1, 1).mul(f).to(BF)        # 40 * 16 blocks of 256 rows
        attend(big, big, big, None)
        out, lse = attend(q, k, v, mine)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bias", [None, "slopes", "table"])
@pytest.mark.parametrize("size", [0.5, 1.5, 4.0])
def test_capped_scores_of_every_size(causal, bias, size):
    """Arguments of the tanh from both polynomials and beyond, mixed in a chunk of keys, for rows and weights."""
    H, HK, n = 4, 2, 200
    q, k, v = (t.clone() for t in fused(1, n, H, HK, 407))
    q *= size
    k[:, ::7] *= 3
    mine, ref = mods_pair(H, causal=causal, cap=12.0, bias=bias, reach=20)
    out, lse, ro, rl, sp = run_attention(q, k, v, mine, ref)
    check(out, lse, ro, rl, sp, delta(f64(q), f64(k), ref, n), n)
    from tests.test_gpu_attention import run_chunk
    p = Paged([260, 300], H, HK, 32, 408)
    p.k[:, :, ::7] *= size * 2
    w = torch.rand((2, HK, p.width * 32), device=DEV)
    run_chunk(p, [40, 150], mine, ref, seed=409, weights=w, decay=0.5)
