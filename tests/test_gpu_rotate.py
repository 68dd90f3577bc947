"""Rotated append to a paged cache against the float64 oracle, and with the attention that follows it.

Tolerance: an angle's turns are exact to 2^-25 (the fraction's rounding to f32) and 2^-52 of the whole turns, its sine and cosine
to 2^-22 more: 2^-21 of each column's size in a rotated pair, 2^-22 for its products and sum, one rounding to bf16 (2^-8)."""
import numpy as np
import pytest
import torch

from oracle import eight_oracle as E
from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def f64(t):
    return t.detach().cpu().float().to(torch.float64).numpy()


def rnd(*shape, seed, scale=1.0):
    return synth.randn(shape, seed, DEV, BF, scale)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def freqs(dims, base=10000.0):
    return torch.tensor(base ** (-np.arange(dims // 2) / (dims // 2)), dtype=torch.float64, device=DEV)


def close(got, want, x):
    """x: the rows before the rotation."""
    size = np.sqrt((x ** 2).sum(-1, keepdims=True))
    far = np.abs(f64(got) - want) - (2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size * (1 + 2.0 ** -8))
    at = np.unravel_index(np.argmax(far), far.shape)
    assert far[at] <= 0, (at, float(far[at]), float(want[at]), int((far > 0).sum()))


class Case:
    """Sequences of uneven lengths in a shuffled page table, with rows for each."""

    def __init__(self, rows, lens, H, HK, page, seed, stride=0, fused=True):
        self.rows, self.lens_host, self.H, self.HK, self.page = rows, lens, H, HK, page
        B, T = len(rows), sum(rows)
        need = [max(1, -(-n // page)) for n in lens]
        self.num = sum(need) + 2
        ids = np.random.RandomState(seed).permutation(self.num)
        self.table = np.full((B, max(need)), -1)
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
        both = torch.full((self.num, 2, HK, page, 64), 7.0, dtype=BF, device=DEV)
        self.k, self.v = (both[:, 0], both[:, 1]) if stride else (both[:, 0].contiguous(), both[:, 1].contiguous())
        self.cu = np.concatenate([[0], np.cumsum(rows)])
        if fused:
            m = rnd(T, H + 2 * HK, 64, seed=seed + 1)
            self.q, self.k_new, self.v_new = m[:, :H], m[:, H:H + HK], m[:, H + HK:]
        else:                                            # heads first
            self.q, self.k_new, self.v_new = (rnd(h, T, 64, seed=seed + 1 + h).transpose(0, 1) for h in (H, HK, HK))
        self.kv = L.KVCache(self.k, self.v, heads=H, max_seqs=B, max_rows=max(T, 1), max_len=max(need) * page)
        self.args = dict(cu_rows=i32(self.cu), lens=i32(lens), pages=i32(self.table))

    def expected(self, first, inv, interleaved):
        """(q, k pages, v pages, sizes of k) after the append."""
        k, v = f64(self.k), f64(self.v)
        before = k.copy()
        pos = np.concatenate([(np.arange(n - r, n) if first is None else first[b] + np.arange(r)) for b, (r, n) in enumerate(zip(self.rows, self.lens_host))])
        turn = (lambda x: E.rotate(x, pos, inv, interleaved)) if inv is not None else (lambda x: x)
        q, kn, vn = turn(f64(self.q)), turn(f64(self.k_new)), f64(self.v_new)
        for b, (r, n) in enumerate(zip(self.rows, self.lens_host)):
            for i in range(r):
                slot = n - r + i
                page = self.table[b, slot // self.page] if 0 <= slot < self.table.shape[1] * self.page else -1
                if 0 <= page < self.num:
                    k[page, :, slot % self.page], v[page, :, slot % self.page] = kn[self.cu[b] + i], vn[self.cu[b] + i]
                    before[page, :, slot % self.page] = f64(self.k_new)[self.cu[b] + i]
        return q, k, v, before


CASES = [
    # rows, lens, H, HK, page
    ([1], [517], 12, 12, 16),
    ([1], [1], 1, 1, 16),
    ([1, 1, 1, 1, 1], [3, 100, 64, 65, 1], 16, 4, 64),
    ([40, 0, 17, 1], [40, 30, 17, 90], 6, 2, 32),
    ([300, 129], [300, 400], 8, 1, 128),
    ([70, 70], [512, 70], 24, 8, 256),
    ([5, 9], [20, 31], 32, 32, 16),
]


@pytest.mark.parametrize("rows,lens,H,HK,page", CASES)
@pytest.mark.parametrize("dims,interleaved", [(64, False), (64, True), (48, False), (32, True), (16, False), (16, True), (0, False)])
def test_append_against_the_oracle(rows, lens, H, HK, page, dims, interleaved):
    odd = dims % 32 == 16
    c = Case(rows, lens, H, HK, page, 7 * H + page, stride=odd, fused=not odd)
    first = [100003 + 911 * b for b in range(len(rows))] if interleaved else None
    inv = freqs(dims) if dims else None
    rot = L.make_rotation(inv, interleaved=interleaved) if dims else None
    q_out = torch.full((sum(rows), H, 64), 7.0, dtype=BF, device=DEV)
    side = torch.full((len(rows), HK, c.table.shape[1] * page), -5, dtype=torch.int32, device=DEV)
    q, k, v, before = c.expected(first, inv.cpu().numpy() if dims else None, interleaved)
    c.kv.append(c.k_new, c.v_new, q=c.q, q_out=q_out, rotation=rot, positions=side, first=None if first is None else i32(first), **c.args)
    torch.cuda.synchronize()
    close(q_out, q, f64(c.q))
    close(c.k, k, before)
    assert np.array_equal(f64(c.v), v)
    want = np.full(side.shape, -5)
    for b, (r, n) in enumerate(zip(rows, lens)):
        want[b, :, n - r:n] = np.arange(n - r, n) if first is None else first[b] + np.arange(r)
    assert np.array_equal(side.cpu().numpy(), want)
    if not dims:
        assert torch.equal(q_out, c.q)
    # in place, and without queries
    both = torch.cat((c.q, c.k_new, c.v_new), 1)
    c.kv.append(both[:, H:H + HK], both[:, H + HK:], q=both[:, :H], q_out=both[:, :H], rotation=rot, first=None if first is None else i32(first), **c.args)
    assert torch.equal(both[:, :H], q_out)
    again = c.k.clone()
    c.k.fill_(7.0)
    c.kv.append(c.k_new, c.v_new, rotation=rot, first=None if first is None else i32(first), **c.args)
    assert torch.equal(c.k, again)
    c.kv.close()


@pytest.mark.parametrize("H,HK,dims,interleaved", [(24, 8, 64, False), (12, 4, 32, True), (33, 11, 48, False)])
def test_long_prompts(H, HK, dims, interleaved):
    """As many rows as fill the device: the lanes of a warp take four heads each."""
    rows = [2500, 2411, 1]
    c = Case(rows, [2600, 2411, 77], H, HK, 64, 13)
    inv = freqs(dims)
    q_out = torch.full((sum(rows), H, 64), 7.0, dtype=BF, device=DEV)
    q, k, v, before = c.expected(None, inv.cpu().numpy(), interleaved)
    c.kv.append(c.k_new, c.v_new, q=c.q, q_out=q_out, rotation=L.make_rotation(inv, interleaved=interleaved), **c.args)
    close(q_out, q, f64(c.q))
    close(c.k, k, before)
    assert np.array_equal(f64(c.v), v)
    c.kv.close()


def test_pages_beyond_2_31_elements():
    HK, page, num, n = 8, 64, 65540, 130                 # 32,768 elements in a page
    k, v = (torch.zeros((num, HK, page, 64), dtype=BF, device=DEV) for _ in range(2))
    kv = L.KVCache(k, v, heads=8, max_seqs=1, max_rows=n, max_len=192)
    kn, vn, table = rnd(n, HK, 64, seed=61), rnd(n, HK, 64, seed=62), [65539, 65535, 65536]
    inv = freqs(64)
    kv.append(kn, vn, rotation=L.make_rotation(inv), cu_rows=i32([0, n]), lens=i32([n]), pages=i32([table]))
    torch.cuda.synchronize()
    flat = lambda t: t[table].transpose(1, 2).reshape(192, HK, 64)
    close(flat(k)[:n], E.rotate(f64(kn), np.arange(n), inv.cpu().numpy()), f64(kn))
    assert torch.equal(flat(v)[:n], vn) and not flat(k)[n:].any()
    k[table], v[table] = 0, 0
    assert not k.any() and not v.any()
    kv.close()


def test_positions_up_to_the_largest():
    """Angles of far positions, where an f32 product would have lost them, and negative ones."""
    B = 6
    c = Case([3] * B, [40] * B, 4, 4, 16, 3)
    first = [0, 2 ** 20 + 1, 10 ** 8 + 7, 2 ** 31 - 3, -1, -12345678]
    inv = freqs(64)
    q_out = torch.zeros((3 * B, 4, 64), dtype=BF, device=DEV)
    q, k, _, before = c.expected(first, inv.cpu().numpy(), False)
    c.kv.append(c.k_new, c.v_new, q=c.q, q_out=q_out, rotation=L.make_rotation(inv), first=i32(first), **c.args)
    close(q_out, q, f64(c.q))
    close(c.k, k, before)
    c.kv.close()


def test_pages_that_do_not_exist_and_rows_behind_the_last_sequence():
    c = Case([20, 30], [60, 50], 4, 2, 16, 5)
    c.table[0, 3], c.table[1, 2] = c.num, -1             # slots 48.. of the first, 32..47 of the second
    c.args["pages"] = i32(c.table)
    q_out = torch.full((50, 4, 64), 7.0, dtype=BF, device=DEV)
    inv = freqs(64)
    q, k, v, before = c.expected(None, inv.cpu().numpy(), False)
    c.kv.append(c.k_new, c.v_new, q=c.q, q_out=q_out, rotation=L.make_rotation(inv), **c.args)
    close(q_out, q, f64(c.q))
    close(c.k, k, before)
    assert np.array_equal(f64(c.v), v)
    # fewer rows belong to sequences than the arrays have; a sequence shorter than what it brings; lengths beyond the table
    c.k.fill_(7.0)
    q_out.fill_(7.0)
    c.args["cu_rows"], c.args["lens"] = i32([0, 10, 30]), i32([4, 1000])
    c.kv.append(c.k_new, c.v_new, q=c.q, q_out=q_out, rotation=L.make_rotation(inv), **c.args)
    torch.cuda.synchronize()
    assert torch.all(q_out[30:] == 7.0)
    pos = np.concatenate([np.arange(-6, 4), np.arange(64 - 20, 64)])
    close(q_out[:30], E.rotate(f64(c.q)[:30], pos, inv.cpu().numpy()), f64(c.q)[:30])
    stored = E.rotate(f64(c.k_new), np.concatenate([pos, np.zeros(20)]), inv.cpu().numpy())
    close(c.k[c.table[0, 0], :, :4].transpose(0, 1), stored[6:10], f64(c.k_new)[6:10])
    assert torch.all(c.k[c.table[0, 0], :, 4:] == 7.0) and torch.all(c.k[c.table[1, 1]] == 7.0)
    c.kv.close()


def test_no_rows_and_no_sequences():
    c = Case([2], [9], 4, 4, 16, 5)
    rot = L.make_rotation(freqs(64))
    c.kv.append(c.k_new[:0], c.v_new[:0], rotation=rot, cu_rows=i32([0, 0]), lens=i32([9]), pages=c.args["pages"])
    c.kv.append(c.k_new, c.v_new, rotation=rot, cu_rows=i32([0]), lens=i32([]), pages=c.args["pages"][:0])
    torch.cuda.synchronize()
    assert torch.all(c.k == 7.0)
    raw = L.KVNew()
    raw.struct_size = 8
    with pytest.raises(L.LLMCacheError) as e:
        L.llmcache_kv_append(c.kv.handle, raw)
    assert e.value.status == L.ERR_ARG
    bad = L.make_rotation(freqs(64))
    bad.dims = 40
    with pytest.raises(L.LLMCacheError) as e:
        c.kv.append(c.k_new, c.v_new, rotation=bad, **c.args)
    assert e.value.status == L.ERR_SHAPE
    bad = L.make_rotation(freqs(64))
    bad.inv_freq = torch.zeros(32, dtype=torch.float64).data_ptr()
    with pytest.raises(L.LLMCacheError) as e:
        c.kv.append(c.k_new, c.v_new, rotation=bad, **c.args)
    assert e.value.status == L.ERR_ARG
    c.kv.close()


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_attention_behind_the_append_equals_attention_that_stores(rows):
    """append + attention without new rows: the same bits as attention that stores the rows which the append gives."""
    H, HK, page, B = 8, 2, 16, 3
    lens = [50, rows, 90]
    a, b = (Case([rows] * B, lens, H, HK, page, 5) for _ in range(2))
    for c in (a, b):
        g = rnd(*c.k.shape, seed=77), rnd(*c.v.shape, seed=78)
        c.k.copy_(g[0])
        c.v.copy_(g[1])
    rot = L.make_rotation(freqs(32), interleaved=True)
    first = i32([1000, 2000, 3000])
    q_out, T = torch.zeros((rows * B, H, 64), dtype=BF, device=DEV), rows * B
    a.kv.append(a.k_new, a.v_new, q=a.q, q_out=q_out, rotation=rot, first=first, **a.args)
    out, weights = torch.zeros_like(q_out), torch.ones((B, HK, a.table.shape[1] * page), device=DEV)
    a.kv.attention(q_out, out, longest=rows, weights=weights, decay=0.5, **a.args)
    torch.cuda.synchronize()
    kn = torch.zeros((T, HK, 64), dtype=BF, device=DEV)
    for s in range(B):
        for i in range(rows):
            slot = lens[s] - rows + i
            kn[s * rows + i] = a.k[int(a.table[s, slot // page]), :, slot % page]
    out2, weights2 = torch.zeros_like(q_out), torch.ones_like(weights)
    b.kv.attention(q_out, out2, k_new=kn, v_new=b.v_new, longest=rows, weights=weights2, decay=0.5, **b.args)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(weights, weights2) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    a.kv.close()
    b.kv.close()


def test_append_captured_on_another_stream():
    c = Case([1, 1], [33, 60], 12, 12, 16, 9)
    rot = L.make_rotation(freqs(64))
    q_out = torch.zeros((2, 12, 64), dtype=BF, device=DEV)
    call = lambda: c.kv.append(c.k_new, c.v_new, q=c.q, q_out=q_out, rotation=rot, **c.args)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in (34, 35):
        c.args["lens"].copy_(i32([n, n + 10]))
        call()
        torch.cuda.synchronize()
        want = q_out.clone(), c.k.clone()
        c.k.fill_(7.0)
        q_out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want[0])
        at = int(c.table[0, (n - 1) // 16]), (n - 1) % 16
        assert torch.equal(c.k[at[0], :, at[1]], want[1][at[0], :, at[1]])
    c.kv.close()
