"""Captured calls that are replayed with other contents, calls on other streams, and calls at the ends of their ranges.  Tolerances:
see test_gpu_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2512_16843_b200 import binding as L
from tests.test_gpu_attention import BF, DEV, Paged, check, close_layers, delta, f64, i32, layer_pair, mods_pair, rnd, run_chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 24])
def test_a_captured_step_replayed_over_a_growing_cache(rows):
    """The graph holds addresses only: lengths, positions and rows change between replays."""
    H, HK, page, steps = 4, 2, 16, 5
    mine, ref = mods_pair(H, causal=True, cap=30.0, bias="slopes")
    lens = [100, 3]
    p = Paged(lens, H, HK, page, 901, extra=rows * steps)
    T = 2 * rows
    q, kn, vn = (torch.zeros((T, h, 64), dtype=BF, device=DEV) for h in (H, HK, HK))
    out, lse = torch.zeros_like(q), torch.zeros((T, H), device=DEV)
    w = torch.zeros((2, HK, p.width * page), device=DEV)
    pos = torch.arange(p.width * page, dtype=torch.int32, device=DEV).expand(2, HK, -1).contiguous()
    lens_dev, first = i32(lens), i32(lens)
    kv = p.handle(T)
    c, rw, rp = p.oracle(), f64(w), pos.cpu().numpy().copy()

    def call():
        kv.attention(q, out, cu_rows=cu, lens=lens_dev, pages=p.pages_dev, longest=rows, k_new=kn, v_new=vn, lse=lse, mods=mine, weights=w,
                     decay=0.5, positions=pos, first=first)

    cu = i32([0, rows, T])
    g = torch.cuda.CUDAGraph()
    keep = [t.clone() for t in (w, pos, p.k, p.v)]
    with torch.cuda.graph(g):
        call()
    for t, x in zip((w, pos, p.k, p.v), keep):
        assert torch.equal(t.view(torch.uint8) if t.dtype is not BF else t.view(torch.int16), x.view(torch.uint8) if x.dtype is not BF else x.view(torch.int16))
    for step in range(steps):
        for t, s in ((q, 1), (kn, 2), (vn, 3)):
            t.copy_(rnd(*t.shape, seed=910 + 10 * step + s))
        first.copy_(lens_dev + 7)
        lens_dev += rows
        g.replay()
        torch.cuda.synchronize()
        now = [n + rows * (step + 1) for n in lens]
        ro, rl, sp, _ = A.chunk(c, f64(q), ref, [0, rows, T], now, p.pages, f64(kn), f64(vn), rw, 0.5, rp, [n - rows + 7 for n in now])
        d = delta(f64(q), c.k, ref, 300)
        check(out, lse, ro, rl, sp, d, max(now))
        assert np.array_equal(pos.cpu().numpy(), rp) and np.array_equal(f64(p.k), c.k, equal_nan=True)
        assert np.all(np.abs(f64(w) - rw) <= rw * (2 * d + 2.0 ** -20 + (max(now) + 2 * rows + step) * 2.0 ** -24) + 2 * rows * 2.0 ** -126)
    assert kv.status() == L.OK
    kv.close()


def test_layer_extend_captured_and_on_another_stream():
    n, d, heads, S = 60, 128, 2, 2
    _, layer = layer_pair(n, d, heads, 256, S)
    mine, _ = mods_pair(heads, causal=True, cap=20.0, bias="table")
    layer.score_mods(mine)
    x = rnd(S, n, d, seed=902)
    k, v = (torch.full((S * 4, heads, 16, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    kv = L.KVCache(k, v, heads=heads, max_seqs=S, max_rows=S * n, max_len=64)
    pages, cu, lens = i32(np.arange(8).reshape(2, 4)), i32([0, 1, 2]), i32([0, 0])
    want = torch.zeros_like(x)
    layer.forward(x, want)
    rows, out, got = torch.zeros((2, d), dtype=BF, device=DEV), torch.zeros((2, d), dtype=BF, device=DEV), torch.zeros_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        layer.extend(kv, rows, out, cu_rows=cu, lens=lens, pages=pages, longest=1)
    st = torch.cuda.Stream()
    for t in range(n):
        rows.copy_(x[:, t])
        lens += 1
        if t % 2:
            g.replay()
        else:
            st.wait_stream(torch.cuda.current_stream())
            layer.extend(kv, rows, out, cu_rows=cu, lens=lens, pages=pages, longest=1, stream=st)
            torch.cuda.current_stream().wait_stream(st)
        got[:, t] = out
    torch.cuda.synchronize()
    assert layer.status() == L.OK and kv.status() == L.OK
    close_layers(got, want)
    kv.close()
    layer.close()


@pytest.mark.parametrize("longest", [1, 20, 0])
def test_calls_in_which_no_sequence_has_rows(longest):
    """All rows lie behind the last sequence: nothing is written but the weights, which fade."""
    p = Paged([150, 1, 300], 4, 2, 32, 903)
    mine, ref = mods_pair(4, causal=True, bias="slopes")
    w = torch.rand((3, 2, p.width * 32), device=DEV)
    run_chunk(p, [0, 0, 0], mine, ref, seed=904, tail=24, weights=w, decay=0.25, longest=longest)


@pytest.mark.parametrize("H,HK", [(128, 1), (200, 2), (65, 1), (254, 2)])
@pytest.mark.parametrize("rows", [1, 3])
def test_large_groups(H, HK, rows):
    """A query tile holds one token of more than 64 heads."""
    p = Paged([140, 70], H, HK, 16, 905)
    mine, ref = mods_pair(H, causal=True, cap=30.0, bias="slopes")
    w = torch.rand((2, HK, p.width * 16), device=DEV)
    run_chunk(p, [rows, rows], mine, ref, seed=906, weights=w, decay=0.5)
