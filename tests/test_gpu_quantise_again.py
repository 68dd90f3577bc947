"""A layer whose weights are brought to 8 bits a second time: what a refused call leaves behind, and whose memory the weights use."""
import subprocess
import sys
import textwrap

import pytest
import torch

from paper_2512_16843_b200 import binding as L
from paper_2512_16843_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def make(d=256, ffn=512, n=40, S=2, seed=5):
    layer = L.Layer(synth.layer_weights(d, ffn, seed, DEV), heads=d // 64, seq_len=n, max_seqs=S)
    return layer, synth.randn((S, n, d), seed + 1, DEV, BF)


def forward(layer, x):
    out = torch.zeros_like(x)
    layer.forward(x, out)
    torch.cuda.synchronize()
    return out


def test_a_call_without_memory_leaves_the_layer_as_it_was():
    layer, x = make(d=2048, ffn=16384, n=16, S=1)
    need = L.llmcache_layer_quantise_bytes(layer.handle)
    assert need > 72 << 20
    plain = forward(layer, x)
    results = {}
    for to in ("e4m3", "int8"):                          # every kernel has run before memory gets short
        layer.quantise(to)
        results[to] = forward(layer, x)
    layer.quantise(None)
    spare = torch.zeros(need, dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(x)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    filler = torch.empty(torch.cuda.mem_get_info()[0] - (48 << 20), dtype=torch.uint8, device=DEV)
    try:
        def refused(to):
            with pytest.raises(L.LLMCacheError) as e:
                layer.quantise(to)
            assert e.value.status == L.ERR_NOMEM

        def run():
            layer.forward(x, out)
            torch.cuda.synchronize()
            return out

        refused("int8")                                  # from bf16
        assert torch.equal(run(), plain)
        layer.quantise("int8", spare)
        assert torch.equal(run(), results["int8"])
        refused("e4m3")                                  # from weights in the caller's memory
        assert torch.equal(run(), results["int8"])
        layer.quantise("e4m3", spare)                    # into that memory again
        assert torch.equal(run(), results["e4m3"])
    finally:
        del filler
        torch.cuda.empty_cache()
    layer.quantise("int8")                               # and out of it: the caller may do with it as they please
    spare.fill_(7)
    assert torch.equal(forward(layer, x), results["int8"])
    layer.close()


def test_the_librarys_memory_serves_again():
    layer, x = make(d=2048, ffn=16384, n=16, S=1)
    layer.quantise("e4m3")
    e4m3 = forward(layer, x)
    layer.quantise("int8")
    int8 = forward(layer, x)
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        for to, want in (("e4m3", e4m3), ("int8", int8)):
            layer.quantise(to)
            assert torch.equal(forward(layer, x), want)
    torch.cuda.empty_cache()
    assert abs(torch.cuda.mem_get_info()[0] - free) <= 8 << 20
    layer.quantise(None)
    assert torch.cuda.mem_get_info()[0] - free >= 64 << 20
    layer.close()


def test_refused_workspaces_leave_the_layer_as_it_was():
    layer, x = make()
    need = L.llmcache_layer_quantise_bytes(layer.handle)
    layer.quantise("int8")
    want = forward(layer, x)
    for bad, status in ((torch.zeros(need - 1, dtype=torch.uint8, device=DEV), L.ERR_NOMEM),
                        (torch.zeros(need + 16, dtype=torch.uint8, device=DEV)[16:], L.ERR_ARG),
                        (torch.zeros(need, dtype=torch.uint8), L.ERR_ARG)):
        with pytest.raises(L.LLMCacheError) as e:
            layer.quantise("e4m3", bad)
        assert e.value.status == status
        assert torch.equal(forward(layer, x), want)
    layer.close()


@pytest.mark.parametrize("shift", [0, 256, 4096])
def test_a_workspace_that_overlaps_the_one_before(shift):
    layer, x = make()
    need = L.llmcache_layer_quantise_bytes(layer.handle)
    whole = torch.zeros(need + 8192, dtype=torch.uint8, device=DEV)
    layer.quantise("e4m3")
    want = forward(layer, x)
    layer.quantise("int8", whole[:need])
    other = forward(layer, x)
    layer.quantise("e4m3", whole[shift:shift + need])
    assert torch.equal(forward(layer, x), want) and not torch.equal(want, other)
    layer.close()


def test_first_calls_on_several_threads():
    """In a process of its own: products and layers that are quantised, for the first time and all at once."""
    code = textwrap.dedent("""
        import threading, torch
        from paper_2512_16843_b200 import binding as L
        from paper_2512_16843_b200 import synth
        torch.cuda.init()
        g = torch.Generator(device="cuda").manual_seed(1)
        sizes = [(1000, 1024, 512), (40, 64, 4096), (9, 300, 128), (300, 2000, 784)]
        data = []
        for m, n, k in sizes:
            a, w = (torch.randn((r, k), generator=g, device="cuda").mul(20).to(torch.int8) for r in (m, n))
            data.append((a, torch.ones(m, device="cuda"), w, torch.ones(n, device="cuda"), torch.zeros((m, (n + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")[:, :n]))
        layers = [L.Layer(synth.layer_weights(128, 256, i, "cuda"), heads=2, seq_len=32, max_seqs=2) for i in range(4)]
        x = synth.randn((2, 32, 128), 9, "cuda", torch.bfloat16)
        outs = [torch.zeros_like(x) for _ in layers]
        torch.cuda.synchronize()
        start, errors = threading.Barrier(8), []
        def run(f):
            try:
                start.wait()
                f()
            except Exception as e:
                errors.append(e)
        def product(d):
            def f():
                stream = torch.cuda.Stream()
                for _ in range(50):
                    L.llmcache_dense(*d, stream=stream)
                stream.synchronize()
            return f
        def layer(l, o):
            def f():
                stream = torch.cuda.Stream()
                for _ in range(5):
                    l.quantise("int8", stream=stream)
                    l.forward(x, o, stream=stream)
                stream.synchronize()
            return f
        threads = [threading.Thread(target=run, args=(f,)) for f in [product(d) for d in data] + [layer(l, o) for l, o in zip(layers, outs)]]
        for t in threads: t.start()
        for t in threads: t.join()
        assert not errors, errors
        for a, sa, w, sw, out in data:
            want = (a.double() @ w.double().t()).to(torch.bfloat16)
            assert torch.equal(out, want)
        for l, o in zip(layers, outs):
            again = torch.zeros_like(x)
            l.forward(x, again)
            torch.cuda.synchronize()
            assert torch.equal(o, again)
        print("fine")
    """)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout + r.stderr
