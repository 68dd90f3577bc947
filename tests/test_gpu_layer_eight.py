"""The layer with 8-bit products, root-mean-square norms and rotation.

Bit for bit against the same steps made one by one through the public entry points (norm, product, rotated append, attention), which
have tests of their own; against a float64 layer; and forward against extend.

Tolerance against float64: the one that the layer's tests derive for its bf16 storage (6e-3 of the output's RMS), and in 8 bits what the
quantisation of weights and activations itself may do: see `eight_error`."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import eight_oracle as E
from oracle import transformer_oracle as T
from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth
from tests.test_gpu_attention import close_layers
from tests.test_gpu_layer import rel_rms

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
TYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def f64(t):
    return t.detach().cpu().float().to(torch.float64).numpy()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def rnd(*shape, seed, scale=1.0):
    return synth.randn(shape, seed, DEV, BF, scale)


def weights(d, ffn, seed):
    w = synth.layer_weights(d, ffn, seed, DEV)
    for k in ("w_qkv", "w_o", "w_1", "w_2"):
        w[k] = (w[k].float() * 3.0).to(BF)
    return w


def rotation(dims, interleaved):
    return L.make_rotation(torch.tensor(10000.0 ** (-np.arange(dims // 2) / (dims // 2)), dtype=torch.float64, device=DEV), interleaved=interleaved)


class Steps:
    """The layer's steps one by one through the public entry points."""

    def __init__(self, w, heads, pre_ln, to, rms, tanh):
        self.w, self.heads, self.pre_ln, self.to, self.kind, self.act = w, heads, pre_ln, to, "rms" if rms else "layer", "gelu_tanh" if tanh else "gelu_erf"
        self.w8 = {k: self.eight(w[k]) for k in ("w_qkv", "w_o", "w_1", "w_2")}

    def eight(self, x):
        q, s = torch.zeros(x.shape, device=DEV).to(TYPE[self.to]), torch.zeros(x.shape[0], device=DEV)
        L.llmcache_norm(x, kind="none", q=q, scale=s)
        return q, s

    def norm(self, x, which):
        q, s, y = torch.zeros(x.shape, device=DEV).to(TYPE[self.to]), torch.zeros(x.shape[0], device=DEV), torch.zeros_like(x)
        L.llmcache_norm(x, kind=self.kind, gain=self.w[f"ln{which}_g"], bias=self.w[f"ln{which}_b"], out=y, q=q, scale=s)
        return y, (q, s)

    def product(self, x8, name, act="none", residual=None):
        n = self.w[f"w_{name}"].shape[0]
        out = torch.zeros((x8[0].shape[0], n), dtype=BF, device=DEV)
        L.llmcache_dense(*x8, *self.w8[f"w_{name}"], out, bias=self.w[f"b_{name}"], act=act, residual=residual)
        return out

    def qkv(self, x):
        return self.product(self.norm(x, 1)[1] if self.pre_ln else self.eight(x), "qkv").view(x.shape[0], 3, self.heads, 64)

    def behind(self, x, a):
        t = self.product(self.eight(a), "o", residual=x)
        y, y8 = self.norm(t, 2 if self.pre_ln else 1)
        f = self.product(y8, "1", act=self.act)
        t = self.product(self.eight(f), "2", residual=t if self.pre_ln else y)
        return t if self.pre_ln else self.norm(t, 2)[0]


LAYERS = [
    # n, d, heads, ffn, S, pre_ln, causal, rms
    (40, 128, 2, 256, 3, False, False, False),
    (130, 192, 3, 320, 2, True, True, True),
    (70, 768, 12, 2048, 2, True, True, False),
    (90, 256, 4, 1152, 1, False, False, True),
    (100, 128, 2, 6400, 2, True, True, True),                # hidden rows that wait in shared memory while others take their place in 8 bits
]


@pytest.mark.parametrize("n,d,heads,ffn,S,pre_ln,causal,rms", LAYERS)
@pytest.mark.parametrize("to", ["int8", "e4m3"])
@pytest.mark.parametrize("dims", [0, 64, 32])
def test_forward_equals_its_steps(n, d, heads, ffn, S, pre_ln, causal, rms, to, dims):
    w = weights(d, ffn, d + n)
    layer = L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=causal, tanh_gelu=pre_ln)
    layer.quantise(to)
    layer.rms(rms)
    rot = rotation(dims, dims == 32) if dims else None
    layer.rotation(rot)
    layer.score_mods(L.make_score_mods(causal=causal))      # the attention that llmcache_attention runs
    x = rnd(S, n, d, seed=7)
    out = torch.full_like(x, 7.0)
    layer.forward(x, out)
    steps = Steps(w, heads, pre_ln, to, rms, pre_ln)
    flat = x.view(S * n, d)
    qkv = steps.qkv(flat)
    if dims:                                             # the rotated rows of a cache with a page table that keeps their order
        k, v = (torch.zeros((S * -(-n // 16), heads, 16, 64), dtype=BF, device=DEV) for _ in range(2))
        kv = L.KVCache(k, v, heads=heads, max_seqs=S, max_rows=S * n, max_len=n)
        kv.append(qkv[:, 1], qkv[:, 2], q=qkv[:, 0], q_out=qkv[:, 0], rotation=rot, cu_rows=i32(np.arange(S + 1) * n), lens=i32([n] * S),
                  pages=i32(np.arange(k.shape[0]).reshape(S, -1)))
        rows = k.view(S, -1, heads, 16, 64).transpose(2, 3).reshape(S, -1, heads, 64)[:, :n]
        qkv[:, 1] = rows.reshape(S * n, heads, 64)
        torch.cuda.synchronize()
        kv.close()
    t = qkv.view(S, n, 3, heads, 64)
    a = torch.zeros((S, n, heads, 64), dtype=BF, device=DEV)
    L.llmcache_attention(t[:, :, 0], t[:, :, 1], t[:, :, 2], a, mods=L.make_score_mods(causal=causal))
    want = steps.behind(flat, a.view(S * n, d)).view(S, n, d)
    torch.cuda.synchronize()
    assert layer.status() == L.OK and torch.equal(out, want)
    # fewer sequences, counted on the device; the rest stays
    if S > 1:
        part = torch.full_like(x, 7.0)
        layer.forward(x, part, n_seqs_dev=i32([1]))
        assert torch.equal(part[:1], out[:1]) and torch.all(part[1:] == 7.0)
    # the attention without modifiers (another kernel) differs by its own roundings
    layer.score_mods(None)
    other = torch.zeros_like(x)
    layer.forward(x, other)
    torch.cuda.synchronize()
    assert rel_rms(f64(other), f64(out)) < (6e-3 if to == "int8" else 2e-2)
    layer.close()


@pytest.mark.parametrize("n,d,heads,ffn,S,pre_ln,causal,rms", [c for c in LAYERS if c[6]] + [(90, 256, 4, 1152, 2, False, True, True)])
@pytest.mark.parametrize("to,dims", [("int8", 64), ("e4m3", 32), ("int8", 0), (None, 64), (None, 48)])
def test_extend_equals_its_steps_and_forward(n, d, heads, ffn, S, pre_ln, causal, rms, to, dims):
    w = weights(d, ffn, d + n + 1)
    layer = L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=True, tanh_gelu=pre_ln)
    layer.quantise(to)
    layer.rms(rms)
    rot = rotation(dims, dims == 32) if dims else None
    layer.rotation(rot)
    x = rnd(S, n, d, seed=8)
    want = torch.zeros_like(x)
    layer.forward(x, want)
    page = 16
    num = S * -(-n // page)
    mk = lambda: L.KVCache(*(torch.full((num, heads, page, 64), 7.0, dtype=BF, device=DEV) for _ in range(2)), heads=heads, max_seqs=S, max_rows=S * n, max_len=n)
    kv, kv2 = mk(), mk()
    pages = i32(np.random.RandomState(2).permutation(num).reshape(S, -1))
    steps = Steps(w, heads, pre_ln, to, rms, pre_ln) if to else None
    got, at = torch.zeros_like(x), [0] * S
    for rows in ([n - 32, n - 38], [1, 1], [30, 36], [1, 1]):
        rows = rows[:S]
        cu = np.concatenate([[0], np.cumsum(rows)])
        xs = torch.cat([x[s, at[s]:at[s] + rows[s]] for s in range(S)])
        at = [p + r for p, r in zip(at, rows)]
        out = torch.full_like(xs, 7.0)
        a = dict(cu_rows=i32(cu), lens=i32(at), pages=pages)
        layer.extend(kv, xs, out, longest=max(rows), **a)
        for s in range(S):
            got[s, at[s] - rows[s]:at[s]] = out[int(cu[s]):int(cu[s + 1])]
        if to:
            qkv = steps.qkv(xs)
            o = torch.zeros((xs.shape[0], heads, 64), dtype=BF, device=DEV)
            if dims:
                kv2.append(qkv[:, 1], qkv[:, 2], q=qkv[:, 0], q_out=qkv[:, 0], rotation=rot, **a)
            kv2.attention(qkv[:, 0], o, longest=max(rows), k_new=None if dims else qkv[:, 1], v_new=None if dims else qkv[:, 2], **a)
            assert torch.equal(out, steps.behind(xs, o.view(-1, d)))
            assert torch.equal(kv.k_pages, kv2.k_pages) and torch.equal(kv.v_pages, kv2.v_pages)
    torch.cuda.synchronize()
    assert at == [n] * S and kv.status() == L.OK and layer.status() == L.OK
    if to == "e4m3":
        assert rel_rms(f64(got), f64(want)) < 2e-2
    elif to == "int8":
        assert rel_rms(f64(got), f64(want)) < 6e-3
    else:
        close_layers(got, want)
    for c in (kv, kv2):
        c.close()
    layer.close()


def oracle_layer(x, w, heads, pre_ln, causal, tanh, to, rms, freq, interleaved):
    """One sequence [n, d] in float64; intermediates that the layer stores in bf16 are rounded to it, products take what the 8
    bits stand for."""
    st = lambda t: T._store(t, True)
    n, d = x.shape
    def eight(v):
        if to is None:
            return v
        q, s = E.eight_bits(v, to)
        return q * s[:, None]
    lin = lambda t, name: eight(t) @ eight(f64(w["w_" + name])).T + f64(w["b_" + name])
    norm = lambda t, i: E.norm(t, "rms" if rms else "layer", f64(w[f"ln{i}_g"]), f64(w[f"ln{i}_b"]))[1]
    act = lambda t: E.gelu(t, "gelu_tanh" if tanh else "gelu_erf")
    keep = st if to is None else (lambda t: t)           # normed rows go to 8 bits from f32
    qkv = st(lin(keep(norm(x, 1)) if pre_ln else x, "qkv")).reshape(n, 3, heads, 64)
    q, k, v = qkv[:, 0], qkv[:, 1], qkv[:, 2]
    if freq is not None:
        q, k = (st(E.rotate(t, np.arange(n), freq, interleaved)) for t in (q, k))
    a, _, _ = A.attention(q[None], k[None], v[None], A.Mods(causal=causal, scale=0.125), None, None)
    t = st(lin(st(a[0].reshape(n, d)), "o") + x)
    y = norm(t, 2 if pre_ln else 1)
    f = st(act(lin(keep(y), "1")))
    t = lin(f, "2") + (t if pre_ln else st(y))
    return t if pre_ln else norm(st(t), 2)


def eight_error(to):
    """RMS error that a stage's rounding to 8 bits may add where its input is off by what bf16 storage may do (6e-3 of the RMS).
    An input that moves by e crosses a border of steps of size h with probability |e| / h and then moves by h: RMS sqrt(e h).  int8:
    h = 4.5 / 127 of the RMS; e4m3: values of the size of the RMS have h = 2^-3 of it.  Two such stages in a row count."""
    return 6e-3 + 2 * (6e-3 * (4.5 / 127 if to == "int8" else 0.125)) ** 0.5 if to else 6e-3


@pytest.mark.parametrize("n,d,heads,ffn,S,pre_ln,causal,rms", LAYERS)
@pytest.mark.parametrize("to,dims,interleaved", [("int8", 64, False), ("e4m3", 32, True), (None, 64, True), (None, 16, False), (None, 0, False)])
def test_forward_against_the_oracle(n, d, heads, ffn, S, pre_ln, causal, rms, to, dims, interleaved):
    w = weights(d, ffn, d + n + 2)
    layer = L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=causal, tanh_gelu=pre_ln)
    x = rnd(S, n, d, seed=9)
    plain, out = torch.zeros_like(x), torch.zeros_like(x)
    layer.forward(x, plain)
    layer.quantise(to)
    layer.rms(rms)
    rot = rotation(dims, interleaved) if dims else None
    layer.rotation(rot)
    layer.forward(x, out)
    torch.cuda.synchronize()
    freq = None if rot is None else rot.tensors[0].cpu().numpy()
    for s in range(S):
        want = oracle_layer(f64(x[s]), w, heads, pre_ln, causal, pre_ln, to, rms, freq, interleaved)
        assert rel_rms(f64(out[s]), want) <= eight_error(to)
        if dims == 64:                                   # and the rotation is there
            without = oracle_layer(f64(x[s]), w, heads, pre_ln, causal, pre_ln, to, rms, None, False)
            assert rel_rms(f64(out[s]), want) < 0.5 * rel_rms(without, want)
    # switched off again: the layer as it was, bit for bit
    layer.quantise(None)
    layer.rms(False)
    layer.rotation(None)
    layer.forward(x, out)
    torch.cuda.synchronize()
    assert torch.equal(out, plain) and layer.status() == L.OK
    layer.close()


def test_rows_beyond_longest_with_a_rotation():
    """They are rotated and stored, and the layer gives for them what it gives for an attention of zero."""
    n, d, heads, S = 64, 128, 2, 2
    w = weights(d, 256, 5)
    x = rnd(60, d, seed=10)
    for rows, longest in (([40, 20], 24), ([50, 10], 20), ([4, 56], 2)):
        results = []
        for rot in (None, rotation(64, False)):
            layer = L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=True, causal=True, tanh_gelu=True)
            layer.rotation(rot)
            kv = L.KVCache(*(torch.full((8, heads, 16, 64), 7.0, dtype=BF, device=DEV) for _ in range(2)), heads=heads, max_seqs=S, max_rows=60, max_len=n)
            a = dict(cu_rows=i32([0, rows[0], 60]), lens=i32(rows), pages=i32(np.arange(8).reshape(2, 4)))
            full, cut = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
            layer.extend(kv, x, full, longest=max(rows), **a)       # leaves other values in the layer's buffers
            pages = kv.k_pages.clone()
            kv.k_pages.fill_(7.0)
            layer.extend(kv, x, cut, longest=longest, **a)
            torch.cuda.synchronize()
            assert torch.equal(kv.k_pages, pages)
            for s, r0 in enumerate((0, rows[0])):
                m = min(longest, rows[s])
                assert rel_rms(f64(cut[r0:r0 + m]), f64(full[r0:r0 + m])) < 6e-3
            results.append(cut)
            kv.close()
            layer.close()
        # an attention of zero does not know of rotations
        for s, r0 in enumerate((0, rows[0])):
            if rows[s] > longest:
                assert torch.equal(results[0][r0 + longest:r0 + rows[s]], results[1][r0 + longest:r0 + rows[s]])


def test_positions_that_run_ahead_of_the_slots():
    """first with and without a positions array: rotary scores depend on distances alone, so a shift of all positions changes
    roundings only."""
    n, d, heads = 48, 128, 2
    w = weights(d, 256, 6)
    layer = L.Layer(w, heads=heads, seq_len=n, max_seqs=1, pre_ln=True, causal=True, tanh_gelu=True)
    layer.rotation(rotation(64, False))
    x = rnd(n, d, seed=11)
    outs = []
    for first, with_positions in ((None, False), (5000, False), (5000, True)):
        kv = L.KVCache(*(torch.full((3, heads, 16, 64), 7.0, dtype=BF, device=DEV) for _ in range(2)), heads=heads, max_seqs=1, max_rows=n, max_len=n)
        side = torch.full((1, heads, 48), -1, dtype=torch.int32, device=DEV) if with_positions else None
        out = torch.zeros_like(x)
        for lo, hi in ((0, 20), (20, 21), (21, 48)):
            layer.extend(kv, x[lo:hi].contiguous(), out[lo:hi], cu_rows=i32([0, hi - lo]), lens=i32([hi]), pages=i32([[2, 0, 1]]),
                         first=None if first is None else i32([first + lo]), positions=side)
        torch.cuda.synchronize()
        if with_positions:
            assert np.array_equal(side.cpu().numpy(), np.broadcast_to(5000 + np.arange(48), (1, heads, 48)))
        outs.append(out)
        kv.close()
    assert rel_rms(f64(outs[1]), f64(outs[0])) < 6e-3 and torch.equal(outs[1], outs[2])
    layer.rotation(None)
    kv = L.KVCache(*(torch.full((3, heads, 16, 64), 7.0, dtype=BF, device=DEV) for _ in range(2)), heads=heads, max_seqs=1, max_rows=n, max_len=n)
    with pytest.raises(L.LLMCacheError) as e:            # without a rotation nobody asks for first alone
        layer.extend(kv, x, torch.zeros_like(x), cu_rows=i32([0, n]), lens=i32([n]), pages=i32([[2, 0, 1]]), first=i32([0]))
    assert e.value.status == L.ERR_ARG
    kv.close()
    layer.close()


def test_quantised_layers_in_the_caching_loop_and_a_workspace():
    n, d, heads, ffn, B, N, k = 32, 128, 2, 256, 6, 16, 64
    ws = [weights(d, ffn, 300 + l) for l in range(2)]
    layers = [L.Layer(w, heads=heads, seq_len=n, max_seqs=B) for w in ws]
    need = L.llmcache_layer_quantise_bytes(layers[0].handle)
    assert need >= (4 * d * d + 2 * d * ffn)
    layers[0].quantise("int8", torch.zeros(need, dtype=torch.uint8, device=DEV))
    layers[1].quantise("e4m3")
    layers[1].rotation(rotation(64, False))
    layers[1].rms()
    for bad, status in ((torch.zeros(need - 1, dtype=torch.uint8, device=DEV), L.ERR_NOMEM), (torch.zeros(need + 16, dtype=torch.uint8, device=DEV)[16:], L.ERR_ARG)):
        with pytest.raises(L.LLMCacheError) as e:
            layers[0].quantise("int8", bad)
        assert e.value.status == status
    banks = [L.Bank(capacity=N, seq_len=n, d_model=d, fp_dim=k, max_batch=B, proj=synth.projection(d, k, 9, DEV), tau=0.9) for _ in range(2)]
    bufs = L.ProbeBuffers(B, k, DEV)
    mk = lambda: torch.zeros((B, n, d), dtype=BF, device=DEV)
    buf_a, buf_b, h_miss, miss_out = mk(), mk(), mk(), mk()
    h0 = rnd(B, n, d, seed=12)

    def run(with_banks):
        at = L.llmcache_infer([b.handle for b in banks] if with_banks else None, [l.handle for l in layers], h0, B, None, buf_a, buf_b, h_miss, miss_out, bufs.io)
        torch.cuda.synchronize()
        return (buf_a if at == buf_a.data_ptr() else buf_b).clone()

    plain = run(False)
    assert torch.equal(run(True), plain) and torch.equal(run(True), plain)       # missed, then served from the banks
    assert [b.stats()["hits"] for b in banks] == [B, B]
    layers[0].quantise("e4m3")                           # replaces the weights
    layers[0].quantise(None)
    layers[1].quantise(None)
    assert not torch.equal(run(False), plain)
    for o in layers + banks:
        o.close()


def test_extend_of_a_quantised_layer_captured():
    n, d, heads = 64, 128, 2
    layer = L.Layer(weights(d, 256, 7), heads=heads, seq_len=n, max_seqs=2, pre_ln=True, causal=True, tanh_gelu=True)
    layer.quantise("int8")
    layer.rms()
    layer.rotation(rotation(64, False))
    kv = L.KVCache(*(torch.zeros((8, heads, 16, 64), dtype=BF, device=DEV) for _ in range(2)), heads=heads, max_seqs=2, max_rows=2, max_len=n)
    x, out, lens, pages = rnd(2, d, seed=13), torch.zeros((2, d), dtype=BF, device=DEV), i32([1, 1]), i32(np.arange(8).reshape(2, 4))
    call = lambda: layer.extend(kv, x, out, cu_rows=cu, lens=lens, pages=pages, longest=1)
    cu = i32([0, 1, 2])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(2, 20):
        lens.fill_(step)
        x.copy_(rnd(2, d, seed=13 + step))
        call()
        torch.cuda.synchronize()
        want = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    kv.close()
    layer.close()


@pytest.mark.parametrize("pre_ln", [False, True])
def test_large_batches_equal_small_ones(pre_ln):
    """Rows of int8 layers do not depend on what else is in the batch, whatever kernels its size takes."""
    n, d, heads, S = 128, 768, 12, 40
    layer = L.Layer(weights(d, 2048, 17), heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=pre_ln, tanh_gelu=pre_ln)
    layer.quantise("int8")
    layer.rms()
    layer.rotation(rotation(64, False))
    x = rnd(S, n, d, seed=71)
    out, part = torch.zeros_like(x), torch.zeros_like(x[:3])
    layer.forward(x, out)
    for s in (0, 17, 37):
        layer.forward(x[s:s + 3].contiguous(), part)
        torch.cuda.synchronize()
        assert torch.equal(part, out[s:s + 3]), s
    assert layer.status() == L.OK
    layer.close()


def test_settings_and_calls_on_another_stream():
    n, d, heads, S = 40, 128, 2, 3
    layer = L.Layer(weights(d, 256, 27), heads=heads, seq_len=n, max_seqs=S)
    x = rnd(S, n, d, seed=81)
    out, want = torch.zeros_like(x), torch.zeros_like(x)
    layer.quantise("int8")
    layer.forward(x, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    layer.quantise(None)
    layer.quantise("int8", stream=side)
    layer.forward(x, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    layer.close()
