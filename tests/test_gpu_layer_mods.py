"""Score modifiers inside the layer: forward against the float64 layer with the modified attention, extend against forward (other
kernels), and a layer served token by token with recorded weights and an eviction between its calls.

Tolerance against float64: the one that the layer's tests derive for its roundings (bf16 storage of the intermediates, which
the oracle rounds at the same places)."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import transformer_oracle as T
from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth
from tests.test_gpu_attention import BF, DEV, close_layers, docs, f64, i32, layer_pair, mods_pair, rnd

pytestmark = pytest.mark.gpu


def oracle_weights(w):
    return T.LayerWeights(**{f.name: synth.bf16_bits(w[f.name]) if f.name.startswith("w_") else w[f.name].float().cpu().numpy()
                             for f in dataclasses.fields(T.LayerWeights)})


def oracle_layer(x, w, heads, m, doc, prefix, pre_ln):
    """One sequence x (bf16 tensor [n, d]): the layer with attention_oracle in place of its attention; intermediates stored
    as bf16.  Also the q|k|v rows."""
    st = lambda t: T._store(t, True)
    v = lambda name: T._v(getattr(w, name))
    lin = lambda t, name: t @ T._w(getattr(w, "w_" + name)).T + v("b_" + name)
    x = f64(x)
    u = st(T.layer_norm(x, v("ln1_g"), v("ln1_b"))) if pre_ln else x
    qkv = st(lin(u, "qkv")).reshape(1, x.shape[0], 3, heads, 64)
    a, _, _ = A.attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], m, None if doc is None else doc[None], None if prefix is None else [prefix])
    a = st(a[0].reshape(x.shape))
    if pre_ln:
        t = st(lin(a, "o") + x)
        f = st(T.gelu_tanh(lin(st(T.layer_norm(t, v("ln2_g"), v("ln2_b"))), "1")))
        return lin(f, "2") + t, qkv[0]
    y = st(T.layer_norm(st(lin(a, "o") + x), v("ln1_g"), v("ln1_b")))
    f = st(T.gelu_erf(lin(y, "1")))
    return T.layer_norm(st(lin(f, "2") + y), v("ln2_g"), v("ln2_b")), qkv[0]


KINDS = [dict(cap=4.0), dict(bias="slopes"), dict(bias="table"), dict(scale=0.3), dict(cap=3.0, bias="table", scale=0.25),
         dict(cap=6.0, bias="slopes")]


def layer_of(n, d, heads, S, pre_ln, causal):
    """A layer whose attention matters: q and k of a size that makes the softmax sharp, so that a lost modifier shows."""
    w, layer = layer_pair(n, d, heads, 320, S, pre_ln=pre_ln, causal=causal)
    layer.close()
    w["w_qkv"] = (w["w_qkv"].float() * 2.0).to(BF)
    w["w_o"] = (w["w_o"].float() * 4.0).to(BF)
    return w, L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=causal, tanh_gelu=pre_ln)


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("pre_ln,masks", [(True, False), (True, True), (False, False), (False, True)])
def test_forward_with_modifiers_against_the_oracle(kind, pre_ln, masks):
    n, d, heads, S = 150, 192, 3, 2
    w, layer = layer_of(n, d, heads, S, pre_ln, pre_ln)
    x = rnd(S, n, d, seed=701)
    doc = docs(S, n, 702) if masks else None
    prefix = i32([40, 0]) if masks and pre_ln else None
    mine, ref = mods_pair(heads, causal=pre_ln, reach=6, doc=doc, prefix=prefix, **KINDS[kind])
    ow = oracle_weights(w)
    plain, out = torch.zeros_like(x), torch.zeros_like(x)
    layer.forward(x, plain)
    layer.score_mods(mine)
    layer.forward(x, out)
    torch.cuda.synchronize()
    assert layer.status() == L.OK
    far = 0.0
    for s in range(S):
        want, _ = oracle_layer(x[s], ow, heads, ref, None if doc is None else doc[s].cpu().numpy(), None if prefix is None else int(prefix[s]), pre_ln)
        close_layers(out[s], torch.tensor(want))
        far = max(far, float(np.sqrt(np.mean((f64(plain[s]) - want) ** 2) / np.mean(want ** 2))))
    assert far > 4 * 6e-3                                # what the modifiers change is larger than the tolerance
    layer.close()


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("pre_ln", [True, False])
def test_extend_with_modifiers_equals_forward(kind, pre_ln):
    n, d, heads, S, page = 150, 192, 3, 2, 16
    _, layer = layer_of(n, d, heads, S, pre_ln, True)
    x = rnd(S, n, d, seed=703)
    mine, _ = mods_pair(heads, causal=True, reach=6, **KINDS[kind])
    plain, want = torch.zeros_like(x), torch.zeros_like(x)
    layer.forward(x, plain)
    layer.score_mods(mine)
    layer.forward(x, want)
    num = S * (-(-n // page))
    k, v = (torch.full((num, heads, page, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    kv = L.KVCache(k, v, heads=heads, max_seqs=S, max_rows=S * n, max_len=n)
    pages = i32(np.random.RandomState(2).permutation(num).reshape(S, -1))
    got, at = torch.full((S, n, d), 7.0, dtype=BF, device=DEV), [0, 0]
    for rows in ([100, 60], [1, 1], [4, 5], [0, 40], [45, 44]):
        cu = np.concatenate([[0], np.cumsum(rows)])
        xs = torch.cat([x[s, at[s]:at[s] + rows[s]] for s in range(S)])
        out = torch.full_like(xs, 7.0)
        at = [a + r for a, r in zip(at, rows)]
        layer.extend(kv, xs, out, cu_rows=i32(cu), lens=i32(at), pages=pages, longest=max(rows))
        torch.cuda.synchronize()
        for s in range(S):
            got[s, at[s] - rows[s]:at[s]] = out[int(cu[s]):int(cu[s + 1])]
    assert at == [n, n] and layer.status() == L.OK and kv.status() == L.OK
    close_layers(got, want)
    assert np.sqrt(np.mean((f64(plain) - f64(want)) ** 2)) > 4 * 6e-3 * np.sqrt(np.mean(f64(want) ** 2))
    kv.close()
    layer.close()


@pytest.mark.parametrize("kind", [0, 1, 4])
def test_extend_with_weights_positions_and_an_eviction(kind):
    """A prompt, tokens, an eviction by what they recorded and more tokens, through the layer; the oracle takes the layer's q|k|v
    rows (stored as bf16) and keeps a cache of its own."""
    n, d, heads, S, page, budget = 160, 192, 3, 2, 16, 48
    w, layer = layer_of(n, d, heads, S, True, True)
    ow = oracle_weights(w)
    mine, ref = mods_pair(heads, causal=True, reach=6, **KINDS[kind])
    layer.score_mods(mine)
    num = 40
    k, v = (torch.full((num, heads, page, 64), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    c = A.Cache(f64(k), f64(v))
    kv = L.KVCache(k, v, heads=heads, max_seqs=S, max_rows=200, max_len=128)
    ids = np.random.RandomState(4).permutation(num).astype(np.int32)
    cur, fresh = ids[:16].reshape(2, 8), ids[16:28].reshape(2, 6)
    W, rw = torch.zeros((S, heads, 128), device=DEV), np.zeros((S, heads, 128))
    pos, rpos = torch.zeros((S, heads, 128), dtype=torch.int32, device=DEV), np.zeros((S, heads, 128), np.int32)
    x = rnd(S, n, d, seed=704)
    seen, length = np.zeros(S, int), np.zeros(S, int)
    for rows in ([90, 61], [1, 1], "evict", [1, 1], [30, 9], [2, 1]):
        if isinstance(rows, str):
            nw, npos = torch.zeros((S, heads, 128), device=DEV), torch.zeros((S, heads, 128), dtype=torch.int32, device=DEV)
            got, nl = torch.zeros((S, heads, budget), dtype=torch.int32, device=DEV), i32([0, 0])
            kv.evict(lens=i32(length), pages=i32(cur), weights=W, positions=pos, new_pages=i32(fresh), new_lens=nl, budget=budget, recent=8, sinks=4,
                     new_weights=nw, new_positions=npos, kept=got)
            rw2, rpos2 = np.zeros_like(rw), np.zeros_like(rpos)
            for s in range(S):
                for h in range(heads):
                    js = got[s, h].cpu().numpy()         # (the oracle goes on with what was kept: weights may be close)
                    assert np.array_equal(js, A.evict(length, f64(W), pos.cpu().numpy(), budget, 8, 4)[s][h])
                    rw2[s, h, :budget], rpos2[s, h, :budget] = rw[s, h, js], rpos[s, h, js]
                    for i, j in enumerate(js):
                        a, b = c.place(cur[s], j), c.place(fresh[s], i)
                        c.k[b[0], h, b[1]], c.v[b[0], h, b[1]] = c.k[a[0], h, a[1]], c.v[a[0], h, a[1]]
            cur, W, pos, rw, rpos, length = fresh, nw, npos, rw2, rpos2, np.array(nl.tolist())
            continue
        rows = np.array(rows)
        cu, length = np.concatenate([[0], np.cumsum(rows)]), length + rows
        xs = torch.cat([x[s, seen[s]:seen[s] + rows[s]] for s in range(S)])
        out = torch.full_like(xs, 7.0)
        layer.extend(kv, xs, out, cu_rows=i32(cu), lens=i32(length), pages=i32(cur), longest=int(rows.max()), weights=W, decay=0.5, positions=pos,
                     first=i32(seen))
        torch.cuda.synchronize()
        assert layer.status() == L.OK and kv.status() == L.OK
        _, qkv = oracle_layer(xs, ow, heads, A.Mods(), None, None, True)
        a, _, _, _ = A.chunk(c, qkv[:, 0], ref, cu, length, cur, qkv[:, 1], qkv[:, 2], rw, 0.5, rpos, seen)
        st, vec = (lambda t: T._store(t, True)), lambda name: T._v(getattr(ow, name))
        lin = lambda t, name: t @ T._w(getattr(ow, "w_" + name)).T + vec("b_" + name)
        t = st(lin(st(a.reshape(xs.shape)), "o") + f64(xs))
        want = lin(st(T.gelu_tanh(lin(st(T.layer_norm(t, vec("ln2_g"), vec("ln2_b"))), "1"))), "2") + t
        close_layers(out, torch.tensor(want))
        assert np.array_equal(pos.cpu().numpy(), rpos)
        # every row and head gives one in all; single weights differ by the roundings of q and k to bf16 in another order
        assert np.all(np.abs(f64(W).sum(-1) - rw.sum(-1)) <= 1e-3 * rw.sum(-1))
        assert np.sqrt(np.mean((f64(W) - rw) ** 2)) <= 6e-3 * np.sqrt(np.mean(rw ** 2))
        seen = seen + rows
    kv.close()
    layer.close()
