"""Calls captured into a graph whose kernels have not run in the process before.

One call of each operator on the device comes first, as the header asks; the captured ones take other kernels: other widths, kinds and
row counts of the norm, other forms of the product."""
import subprocess
import sys
import textwrap

import pytest

pytestmark = pytest.mark.gpu

HEAD = textwrap.dedent("""
    import torch
    from paper_2512_16843_b200 import binding as L
    BF, DEV = torch.bfloat16, "cuda"
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(BF)
    def norm(rows, cols, kind, residual):
        x, r = rnd(rows, cols), rnd(rows, cols) if residual else None
        gain = torch.rand(cols, generator=g, device=DEV) if kind != "none" else None
        q, s, o = torch.zeros((rows, cols), dtype=torch.int8, device=DEV), torch.zeros(rows, device=DEV), torch.zeros_like(x)
        return (lambda: L.llmcache_norm(x, kind=kind, gain=gain, residual=r, q=q, scale=s, out=o)), [q, s, o]
    def dense(m, n, k, dtype, act, residual):
        a, w = (torch.randn((i, k), generator=g, device=DEV).mul(20).to(dtype) for i in (m, n))
        one, o = torch.ones(max(m, n), device=DEV), torch.zeros((m, n), dtype=BF, device=DEV)
        r = rnd(m, n) if residual else None
        return (lambda: L.llmcache_dense(a, one[:m], w, one[:n], o, act=act, residual=r)), [o]
    def append(rows, interleaved):
        kv = L.KVCache(torch.zeros((8, 2, 64, 64), dtype=BF, device=DEV), torch.zeros((8, 2, 64, 64), dtype=BF, device=DEV), heads=4, max_seqs=1, max_rows=rows, max_len=512)
        q, k, v = rnd(rows, 4, 64), rnd(rows, 2, 64), rnd(rows, 2, 64)
        rot = L.make_rotation(torch.arange(32, dtype=torch.float64, device=DEV) / 32, interleaved=interleaved)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        a = dict(cu_rows=i32([0, rows]), lens=i32([500]), pages=i32([list(range(8))]))
        o = torch.zeros_like(q)
        return (lambda: kv.append(k, v, q=q, q_out=o, rotation=rot, **a)), [o, kv.k_pages, kv]
    def check(calls):
        stream = torch.cuda.Stream()
        graphs = []
        torch.cuda.synchronize()
        for call, outs in calls:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            graphs.append(graph)
        for (call, outs), graph in zip(calls, graphs):
            outs = [o for o in outs if isinstance(o, torch.Tensor)]
            graph.replay()
            torch.cuda.synchronize()
            got = [o.clone() for o in outs]
            assert any(o.float().abs().sum() > 0 for o in outs)
            for o in outs: o.zero_()
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, outs))
        print("fine")
    """)
BODY = {
    "norm": """
norm(4, 64, "rms", False)[0]()
check([norm(r, c, k, res) for r, c, k, res in ((700, 768, "layer", False), (700, 1536, "rms", True), (3, 9000, "rms", False), (300, 9000, "rms", False),
                                               (300, 9000, "layer", True), (300, 16384, "none", False), (1, 8, "none", True), (50, 264, "layer", True))])
""",
    "product": """
dense(100, 64, 64, torch.int8, "none", False)[0]()
check([dense(m, n, k, t, act, res) for m, n, k, t, act, res in ((1, 512, 256, torch.int8, "none", False), (12, 512, 256, torch.float8_e4m3fn, "gelu_erf", True),
      (16, 64, 256, torch.int8, "none", False), (32, 2048, 1024, torch.int8, "none", True), (4000, 1024, 512, torch.float8_e4m3fn, "gelu_tanh", True),
      (100, 64, 4096, torch.int8, "none", True), (1000, 1024, 256, torch.int8, "gelu_erf", False))])
""",
    "append": """
append(1, False)[0]()
check([append(1, True), append(400, False), append(400, True)])
""",
}


@pytest.mark.parametrize("what", BODY)
def test_captured_calls_of_kernels_that_have_not_run(what):
    r = subprocess.run([sys.executable, "-c", HEAD + BODY[what]], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout + r.stderr
