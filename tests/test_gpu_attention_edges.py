"""Attention operators where kernels meet their limits: hidden keys that hold anything, lists of many sequences, shares of
the keys, scratch that does not suffice, waits that expire, two streams at once.  Tolerances: see test_gpu_attention.py."""
import subprocess
import sys
import textwrap

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2512_16843_b200 import binding as L
from tests.test_gpu_attention import BF, DEV, Paged, check, delta, f64, fused, i32, mods_pair, rnd, run_attention, run_chunk

pytestmark = pytest.mark.gpu
INF = float("inf")


def hiding_table(H, reach, *, ends, seed=11):
    """Random entries, -inf at both ends (all distances from reach on) and one -inf in the middle."""
    t = np.random.RandomState(seed).randn(H, 2 * reach + 1).astype(np.float32)
    if ends:
        t[:, 0] = t[:, -1] = -np.inf
    t[:, reach - 2] = -np.inf
    return torch.tensor(t, device=DEV)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("reach", [3, 140])
def test_keys_hidden_by_the_table_may_hold_anything(causal, reach):
    """Rows that see the odd keys have their values, all others must not notice (the whole tile lies beyond the reach, or some
    of it)."""
    n, H = 400, 2
    q, k, v = (t.clone() for t in fused(1, n, H, H, 300))
    k[0, 5, 0], v[0, 7, 1] = float("nan"), float("nan")
    v[0, 150, 0, 3], v[0, 151, 0, 4], k[0, 230, 1] = INF, -INF, INF
    table = hiding_table(H, reach, ends=True)
    out, lse, ro, rl, sp = run_attention(q, k, v, L.make_score_mods(causal=causal, table=table), A.Mods(causal=causal, table=f64(table)))
    assert np.isfinite(ro).all(-1).any() and not np.isfinite(ro).all()
    check(out, lse, ro, rl, np.where(np.isfinite(sp), sp, 0), delta(f64(q), f64(k), A.Mods(table=f64(table)), n), n)


@pytest.mark.parametrize("rows", [1, 5, 30, 140])
@pytest.mark.parametrize("evicted", [False, True])
def test_cached_keys_hidden_by_the_table_may_hold_anything(rows, evicted):
    p = Paged([500, 333], 4, 2, 32, 31)
    reach = 6                                            # the rows see the last slots only
    for s, n in enumerate(p.lens):
        for slot, what in ((3, float("nan")), (n // 2, INF), (n - rows - 40, -INF)):
            p.k[int(p.pages[s, slot // 32]), :, slot % 32] = what
            p.v[int(p.pages[s, (slot + 1) // 32]), :, (slot + 1) % 32] = what
    table = hiding_table(4, reach, ends=True)
    w = torch.rand((2, 2, p.width * 32), device=DEV)
    pos = first = None
    if evicted:
        g = np.random.RandomState(32)
        pos = torch.tensor(np.cumsum(g.randint(1, 3, (2, 2, p.width * 32)), -1), dtype=torch.int32, device=DEV)
        first = [int(pos[s, :, n - rows - 1].max()) + 1 for s, n in enumerate(p.lens)]
    run_chunk(p, [rows, rows], L.make_score_mods(causal=True, table=table), A.Mods(causal=True, table=f64(table)), seed=301, weights=w,
              decay=0.5, positions=pos, first=first)


@pytest.mark.parametrize("rows,bias", [(1, None), (3, "slopes")])
def test_more_sequences_than_a_warp_has_lanes(rows, bias):
    lens = [int(x) for x in np.random.RandomState(33).randint(rows, 400, 70)]
    lens[5], lens[69], lens[31] = rows, rows, 1000
    p = Paged(lens, 2, 1, 16, 34)
    mine, ref = mods_pair(2, causal=True, bias=bias)
    counts = [rows] * 70
    counts[40] = counts[0] = 0
    run_chunk(p, counts, mine, ref, seed=302, weights=torch.rand((70, 1, p.width * 16), device=DEV), decay=0.25)


@pytest.mark.parametrize("rows", [1, 4])
def test_scores_that_fit_their_scratch_and_scores_that_do_not(rows):
    """The scratch is sized for one token per sequence; four have their scores formed again for the weights."""
    p = Paged([500, 260], 4, 2, 16, 35)
    mine, ref = mods_pair(4, causal=True, cap=8.0, bias="table")
    run_chunk(p, [rows, rows], mine, ref, seed=303, weights=torch.rand((2, 2, p.width * 16), device=DEV), decay=0.5)


@pytest.mark.parametrize("rows", [17, 63, 64, 65, 128, 129])
@pytest.mark.parametrize("H,HK,bias", [(2, 2, "slopes"), (4, 2, None), (3, 1, "table")])
def test_shares_of_the_keys(rows, H, HK, bias):
    """Rows that fill one query tile, and one more; shares that do not divide the key tiles."""
    p = Paged([1100, 385, 129], H, HK, 64, 36)
    mine, ref = mods_pair(H, causal=True, cap=0.0 if bias else 20.0, bias=bias)
    run_chunk(p, [rows, rows, min(rows, 129)], mine, ref, seed=304, weights=torch.rand((3, HK, p.width * 64), device=DEV), decay=1.0)


@pytest.mark.parametrize("n,budget", [(4097, 100), (6001, 6000), (20003, 4096), (49152, 777)])
def test_evict_of_long_lists(n, budget):
    HK, page = 2, 64
    width, fresh = -(-n // page), -(-budget // page)
    k = torch.zeros((1, HK, page, 64), dtype=BF, device=DEV).expand(width + fresh, -1, -1, -1).contiguous()
    kv = L.KVCache(k, k.clone(), heads=HK, max_seqs=1, max_rows=1, max_len=n)
    g = np.random.RandomState(n)
    w = (g.randint(0, 50, (1, HK, n)) / 7).astype(np.float32)                # many equal ones
    pos = np.cumsum(g.randint(1, 3, (1, HK, n)), -1).astype(np.int32)
    kept = torch.zeros((1, HK, budget), dtype=torch.int32, device=DEV)
    kv.evict(lens=i32([n]), pages=i32([list(range(width))]), weights=torch.tensor(w, device=DEV), positions=torch.tensor(pos, device=DEV),
             new_pages=i32([list(range(width, width + fresh))]), new_lens=i32([0]), budget=budget, recent=37, sinks=5, kept=kept)
    ref = A.evict([n], w, pos, budget, 37, 5)
    for h in range(HK):
        assert np.array_equal(kept[0, h].cpu().numpy(), ref[0][h])
    kv.close()


def test_evict_of_slots_without_a_page():
    """A kept slot that has no page becomes a row of zeros."""
    p = Paged([60], 2, 2, 16, 37, spare=4)
    p.pages[0, 1] = -1                                   # slots 16 .. 31
    kv = p.handle(1)
    new = i32([p.free[:3].tolist()])
    kept = torch.zeros((1, 2, 48), dtype=torch.int32, device=DEV)
    k0 = p.k.clone()
    kv.evict(lens=i32([60]), pages=torch.tensor(p.pages, device=DEV), weights=torch.ones((1, 2, 64), device=DEV), new_pages=new,
             new_lens=i32([0]), budget=48, recent=10, kept=kept)
    torch.cuda.synchronize()
    for h in range(2):
        for i, j in enumerate(kept[0, h].tolist()):
            got = p.k[int(new[0, i // 16]), h, i % 16]
            want = torch.zeros_like(got) if 16 <= j < 32 else k0[int(p.pages[0, j // 16]), h, j % 16]
            assert torch.equal(got, want)
    assert ((kept >= 16) & (kept < 32)).any()
    kv.close()


def test_refusals_that_need_a_device():
    def status(fn, *a, **kw):
        with pytest.raises(L.LLMCacheError) as e:
            fn(*a, **kw)
        return e.value.status

    q, k, v = fused(1, 8, 2, 2, 305)
    out = torch.empty((1, 8, 2, 64), dtype=BF, device=DEV)
    host = [t.cpu() for t in (q, k, v, out)]
    assert status(L.llmcache_attention, *host) == L.ERR_ARG                  # all of them on the host
    assert status(L.llmcache_attention, q, host[1], v, out) == L.ERR_ARG
    assert status(L.llmcache_attention, q, k, v, out, mods=L.make_score_mods(slopes=torch.ones(2))) == L.ERR_ARG
    p = Paged([30, 20], 2, 2, 16, 38)
    kv = p.handle(4)
    q, out = rnd(2, 2, 64, seed=306), torch.empty((2, 2, 64), dtype=BF, device=DEV)
    good = dict(cu_rows=i32([0, 1, 2]), lens=i32(p.lens), pages=p.pages_dev)
    assert status(kv.attention, q, out, **good, first=i32([5, 6])) == L.ERR_ARG          # positions of queries, but not of keys
    assert status(kv.attention, q, out, **{**good, "lens": i32(p.lens).cpu()}) == L.ERR_ARG
    assert status(kv.attention, q.cpu(), out, **good) == L.ERR_ARG
    kv.attention(q, out, **good)
    torch.cuda.synchronize()
    assert kv.status() == L.OK
    kv.close()


def test_two_streams_at_once():
    """Caches of their own, and attention without an object, side by side on two streams: the same bits as alone."""
    jobs = []
    for i in range(2):
        p = Paged([700 + 90 * i, 300], 4, 2, 32, 40 + i)
        T = 40
        m = rnd(T, 8, 64, seed=310 + i)
        kv, few = p.handle(T), p.handle(T)
        w, wf = (torch.zeros((2, 2, p.width * 32), device=DEV) for _ in range(2))
        out, outf = (torch.zeros((T, 4, 64), dtype=BF, device=DEV) for _ in range(2))
        long = dict(cu_rows=i32([0, 20, 40]), lens=i32(p.lens), pages=p.pages_dev, longest=20, weights=w, decay=0.0)
        short = dict(cu_rows=i32([0, 1, 3]), lens=i32(p.lens), pages=p.pages_dev, longest=2, weights=wf, decay=0.0)
        a, b, c = fused(2, 300, 4, 2, 320 + i)
        whole = torch.zeros((2, 300, 4, 64), dtype=BF, device=DEV)
        mine, _ = mods_pair(4, causal=True, cap=9.0, bias="slopes")

        def job(st, p=p, m=m, kv=kv, few=few, out=out, outf=outf, long=long, short=short, a=a, b=b, c=c, whole=whole, mine=mine):
            kv.attention(m[:, :4], out, stream=st, **long)
            L.llmcache_attention(a, b, c, whole, mods=mine, stream=st)
            few.attention(m[:, :4], outf, stream=st, **short)

        jobs.append((job, (out, outf, whole, w, wf), (kv, few)))
    torch.cuda.synchronize()
    want = []
    for job, results, _ in jobs:
        job(None)
        torch.cuda.synchronize()
        want.append([t.clone() for t in results])
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (job, _, _) in zip(streams, jobs):
            job(st)
    torch.cuda.synchronize()
    for (_, results, caches), ws in zip(jobs, want):
        assert all(torch.equal(x, y) for x, y in zip(results, ws))
        for kv in caches:
            assert kv.status() == L.OK
            kv.close()


def test_expired_waits_return_and_leave_the_context_usable():
    """The loading warp stays idle, so every wait runs out: the calls return, the status says so, the device goes on.  In a
    process of its own, because the status of llmcache_attention is sticky."""
    code = textwrap.dedent("""
        import torch
        from paper_2512_16843_b200 import binding as L
        BF, DEV = torch.bfloat16, "cuda"
        q = torch.randn(1, 300, 2, 64, device=DEV).to(BF)
        out = torch.zeros_like(q)
        L.llmcache_attention(q, q, q, out)
        assert L.llmcache_attention_status() == L.OK
        L.llmcache_attention_debug_knobs(2_000_000, L.KNOB_PRODUCER_IDLE)
        L.llmcache_attention(q, q, q, out)
        assert L.llmcache_attention_status() == L.ERR_TIMEOUT
        L.llmcache_attention_debug_knobs(0, 0)
        again = torch.zeros_like(q)
        L.llmcache_attention(q, q, q, again)
        torch.cuda.synchronize()
        assert torch.isfinite(again.float()).all() and again.abs().sum() > 0
        assert L.llmcache_attention_status() == L.ERR_TIMEOUT            # sticky
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        for rows in (1, 60):
            k = torch.randn(40, 2, 16, 64, device=DEV).to(BF)
            kv = L.KVCache(k, k.clone(), heads=2, max_seqs=1, max_rows=rows, max_len=640)
            x = torch.randn(rows, 2, 64, device=DEV).to(BF)
            w = torch.zeros(1, 2, 640, device=DEV)
            call = lambda: kv.attention(x, torch.zeros_like(x), cu_rows=i32([0, rows]), lens=i32([600]), pages=i32([list(range(40))]),
                                        longest=rows, weights=w, decay=0.0)
            call()
            assert kv.status() == L.OK
            kv.debug_knobs(2_000_000, L.KNOB_PRODUCER_IDLE)
            call()
            assert kv.status() == L.ERR_TIMEOUT
            kv.close()
        assert float(torch.ones(10, device=DEV).sum()) == 10.0
        print("fine")
    """)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout + r.stderr
