"""Calls large enough that a block of the attention kernels has several pieces of work: items of whole sequences and of a paged
cache (one block per SM takes 148 of them at a time), key tiles of few rows (two blocks per SM, one list of tiles for all
sequences), key tiles of received weights (about eight blocks per SM).  Tolerances: see test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2512_16843_b200 import binding as L
from tests.test_gpu_attention import BF, DEV, Paged, docs, f64, fused, i32, mods_pair, rnd, run_chunk

pytestmark = pytest.mark.gpu


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def one_by_one(q, k, v, make):
    """out, lse of the sequences in calls of their own."""
    S, n, H, _ = q.shape
    out, lse = torch.zeros((S, n, H, 64), dtype=BF, device=DEV), torch.zeros((S, n, H), device=DEV)
    for s in range(S):
        L.llmcache_attention(q[s:s + 1], k[s:s + 1], v[s:s + 1], out[s:s + 1], mods=make(slice(s, s + 1)), lse=lse[s:s + 1])
    return out, lse


@pytest.mark.parametrize("kind", ["plain", "causal", "documents", "capped documents", "prefix", "table", "capped"])
def test_items_of_whole_sequences(kind):
    """Same bits as sequence by sequence, where no block has a second item."""
    S, n, H, HK = 41, 300, 16, 8
    assert S * HK * 3 > 3 * sms() and HK * 3 < sms()      # (three pairs of query tiles of 2 * 64 tokens)
    q, k, v = (t.clone() for t in fused(S, n, H, HK, 601))
    doc = docs(S, n, 602)
    doc[5], doc[20, :290] = -1, -1                       # sequences that see nothing, or hardly anything
    v[3, 40, 2, 9], v[17, 290, 1, 60], k[30, 7, 0] = float("nan"), float("inf"), float("nan")
    prefix = i32(np.random.RandomState(603).randint(0, n + 1, S))

    def make(part):
        kw = dict(causal=kind not in ("plain", "documents", "table"))
        if "documents" in kind:
            kw["doc"] = doc[part].contiguous()
        if kind == "prefix":
            kw["prefix"] = prefix[part].contiguous()
        return mods_pair(H, bias="table" if kind == "table" else "slopes" if "capped" in kind else None, cap=30.0 if "capped" in kind else 0.0,
                         reach=64, **kw)[0]

    want, want_lse = one_by_one(q, k, v, make)
    for count in (None, 29, 0):
        out, lse = torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)
        L.llmcache_attention(q, k, v, out, mods=make(slice(0, S)), lse=lse, n_seqs_dev=None if count is None else i32([count]))
        torch.cuda.synchronize()
        assert L.llmcache_attention_status() == L.OK
        m = S if count is None else count
        assert torch.equal(out[:m].view(torch.int16), want[:m].view(torch.int16)) and torch.equal(lse[:m].view(torch.int32), want_lse[:m].view(torch.int32))
        assert torch.all(out[m:] == 7.0) and torch.all(lse[m:] == 7.0)


@pytest.mark.parametrize("rows,lens,cap,bias", [
    (130, (140, 400), 0.0, None), (130, (140, 400), 30.0, "slopes"),         # several query tiles
    (20, (520, 700), 0.0, None), (20, (520, 700), 30.0, "table"),            # rows that fill one: a block's halves share the keys
])
def test_items_of_a_paged_cache(rows, lens, cap, bias):
    B, H, HK = 45, 8, 4
    assert B * HK > sms()
    p = Paged([int(x) for x in np.random.RandomState(604).randint(*lens, B)], H, HK, 32, 605)
    mine, ref = mods_pair(H, causal=True, cap=cap, bias=bias, reach=64)
    w = torch.rand((B, HK, p.width * 32), device=DEV)
    run_chunk(p, [max(0, rows - 3 * (b % 5)) if b % 11 else 0 for b in range(B)], mine, ref, seed=606, weights=w, decay=0.5)


@pytest.mark.parametrize("B,lens,H,HK,page,rows", [
    (64, (1, 1500), 16, 4, 64, 1), (64, (1, 1500), 16, 4, 16, 4),            # segments of many sequences in a block
    (130, (5, 300), 12, 12, 32, 1),
    (2, (39000, 40001), 4, 2, 256, 3),                                       # shares that begin and end inside a sequence
])
@pytest.mark.parametrize("bias", [None, "slopes"])
def test_tiles_of_few_rows(B, lens, H, HK, page, rows, bias):
    lengths = [int(x) for x in np.random.RandomState(607).randint(*lens, B)]
    assert sum(-(-n // 128) for n in lengths) * HK > 4 * sms()
    p = Paged(lengths, H, HK, page, 608)
    mine, ref = mods_pair(H, causal=True, cap=30.0 if bias else 0.0, bias=bias)
    w = torch.rand((B, HK, p.width * page), device=DEV)
    run_chunk(p, [0 if b % 7 == 3 else min(rows, n) for b, n in enumerate(lengths)], mine, ref, seed=609, weights=w, decay=0.5)


@pytest.mark.parametrize("rows,cap,bias", [(20, 0.0, None), (20, 30.0, "slopes"), (150, 0.0, None), (150, 30.0, "table")])
def test_key_tiles_of_received_weights(rows, cap, bias):
    """More key tiles of a sequence and head than blocks for it."""
    B, HK = 16, 8
    lengths = [int(x) for x in np.random.RandomState(610).randint(1500, 2600, B)]
    assert max(lengths) / 128 > 1 + 8 * sms() / (B * HK)
    p = Paged(lengths, HK, HK, 64, 611)
    mine, ref = mods_pair(HK, causal=True, cap=cap, bias=bias, reach=64)
    w = torch.rand((B, HK, p.width * 64), device=DEV)
    run_chunk(p, [rows - b % 3 for b in range(B)], mine, ref, seed=612, weights=w, decay=0.25)


def test_repeated_calls_give_the_same_bits():
    B, H, HK, page = 48, 6, 2, 32
    lengths = [int(x) for x in np.random.RandomState(613).randint(200, 3000, B)]
    p = Paged(lengths, H, HK, page, 614)
    mine, _ = mods_pair(H, causal=True, cap=30.0, bias="slopes")
    for rows in (1, 40):
        T = rows * B
        m = rnd(T, H + 2 * HK, 64, seed=615)
        kv = p.handle(T)
        seen = []
        for _ in range(4):
            out, lse, w = torch.zeros((T, H, 64), dtype=BF, device=DEV), torch.zeros((T, H), device=DEV), torch.zeros((B, HK, p.width * page), device=DEV)
            kv.attention(m[:, :H], out, cu_rows=i32(np.arange(B + 1) * rows), lens=i32(lengths), pages=p.pages_dev, longest=rows, k_new=m[:, H:H + HK],
                         v_new=m[:, H + HK:], lse=lse, mods=mine, weights=w, decay=0.0)
            torch.cuda.synchronize()
            seen.append((out, lse, w))
        assert kv.status() == L.OK
        for other in seen[1:]:
            assert all(torch.equal(a, b) for a, b in zip(other, seen[0]))
        kv.close()
