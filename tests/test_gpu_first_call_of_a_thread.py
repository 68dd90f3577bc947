"""A thread whose first use of CUDA is a call of the library.

A device that other threads use is not yet current in a new one: the runtime binds it with the thread's first runtime call that
needs it, the driver calls that describe copies do not.  Each call runs on the main thread and then as all that a new thread does."""
import threading

import pytest
import torch

from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def rnd(*shape, seed=1):
    return synth.randn(shape, seed, DEV, BF)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def norm():
    x, q, s = rnd(300, 512), torch.zeros((300, 512), dtype=torch.int8, device=DEV), torch.zeros(300, device=DEV)
    return (lambda st: L.llmcache_norm(x, q=q, scale=s, stream=st)), [q, s]


def dense(m, n, k):
    def make():
        g = torch.Generator(device=DEV).manual_seed(3)
        a, w = (torch.randn((r, k), generator=g, device=DEV).mul(20).to(torch.int8) for r in (m, n))
        one, r, out = torch.ones(max(m, n), device=DEV), rnd(m, n), torch.zeros((m, n), dtype=BF, device=DEV)
        return (lambda st: L.llmcache_dense(a, one[:m], w, one[:n], out, residual=r, stream=st)), [out]
    return make


def attention():
    q, k, v = (rnd(2, 200, 4, 64, seed=i) for i in range(3))
    out = torch.zeros_like(q)
    return (lambda st: L.llmcache_attention(q, k, v, out, stream=st)), [out]


def cache(rows):
    def make():
        kv = L.KVCache(rnd(8, 2, 64, 64, seed=1), rnd(8, 2, 64, 64, seed=2), heads=4, max_seqs=2, max_rows=2 * rows, max_len=256)
        q, k, v = rnd(2 * rows, 4, 64, seed=3), rnd(2 * rows, 2, 64, seed=4), rnd(2 * rows, 2, 64, seed=5)
        out = torch.zeros_like(q)
        a = dict(cu_rows=i32([0, rows, 2 * rows]), lens=i32([250, 200]), pages=i32([[0, 2, 4, 6], [1, 3, 5, 7]]))
        def call(st):
            kv.append(k, v, stream=st, **a)
            kv.attention(q, out, longest=rows, stream=st, **a)
        return call, [out, kv]
    return make


def layer(to, n):
    def make():
        l = L.Layer(synth.layer_weights(128, 256, 5, DEV), heads=2, seq_len=n, max_seqs=3)
        l.quantise(to)
        x = rnd(3, n, 128)
        out = torch.zeros_like(x)
        return (lambda st: l.forward(x, out, stream=st)), [out, l]
    return make


def bank():
    b = L.Bank(capacity=2048, seq_len=16, d_model=128, fp_dim=64, max_batch=64, proj=synth.projection(128, 64, 5, DEV), tau=0.9)
    bufs, h = L.ProbeBuffers(64, 64, DEV), rnd(64, 16, 128)
    out = torch.zeros((64, 16 * 128), dtype=BF, device=DEV)
    return (lambda st: b.probe(h, bufs, h_out=out, stream=st)), [bufs.fp, bufs.hit, b]


CALLS = {
    "norm": norm, "dense by pairs": dense(4000, 1024, 512), "dense by 128 columns": dense(1000, 1024, 256), "dense by 64 columns": dense(64, 2304, 768),
    "dense by clusters": dense(100, 64, 4096), "dense of few rows": dense(4, 512, 256), "attention": attention, "cache, single tokens": cache(1),
    "cache, prompts": cache(150), "layer": layer(None, 40), "layer in 8 bits": layer("int8", 40), "layer of long sequences": layer(None, 300), "bank": bank,
}


@pytest.mark.parametrize("name", CALLS)
def test_the_first_call_of_a_thread(name):
    call, results = CALLS[name]()
    results = [r for r in results if isinstance(r, torch.Tensor)]
    stream = torch.cuda.current_stream().cuda_stream
    call(stream)
    torch.cuda.synchronize()
    want = [r.clone() for r in results]
    for r in results:
        r.zero_()
    torch.cuda.synchronize()
    errors = []

    def run():
        try:
            call(stream)
        except Exception as e:
            errors.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    assert all(torch.equal(r, w) for r, w in zip(results, want))
