"""Quantised layers whose hidden rows take 8 bits in their own place while the next rows are on their way.

Rows of 4,096 columns and more wait in shared memory (norm.cu), two or three blocks per SM: only with more rows than that does a block ask
for its next row before it writes the one at hand.  Bit for bit against the steps one by one.  (Not for post-norm with layer norms: the last one,
whose output is bf16 alone, is another kernel's, with another order of sums.)"""
import pytest
import torch

from paper_2512_16843_b200 import binding as L
from tests.test_gpu_layer_eight import DEV, Steps, rnd, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ffn", [4096, 6400, 9024, 14336, 16384])
@pytest.mark.parametrize("to,rms,pre_ln", [("int8", True, True), ("e4m3", False, True), ("int8", True, False), ("e4m3", True, False)])
def test_hidden_rows_in_their_own_place(ffn, to, rms, pre_ln):
    n, d, heads, S = 350, 128, 2, 4
    assert n * S > 3 * torch.cuda.get_device_properties(DEV).multi_processor_count * 2
    w = weights(d, ffn, 31)
    layer = L.Layer(w, heads=heads, seq_len=n, max_seqs=S, pre_ln=pre_ln, causal=pre_ln, tanh_gelu=pre_ln)
    layer.quantise(to)
    layer.rms(rms)
    layer.score_mods(L.make_score_mods(causal=pre_ln))
    x = rnd(S, n, d, seed=32)
    out = torch.full_like(x, 7.0)
    layer.forward(x, out)
    steps = Steps(w, heads, pre_ln, to, rms, pre_ln)
    flat = x.view(S * n, d)
    t = steps.qkv(flat).view(S, n, 3, heads, 64)
    a = torch.zeros((S, n, heads, 64), dtype=x.dtype, device=DEV)
    L.llmcache_attention(t[:, :, 0], t[:, :, 1], t[:, :, 2], a, mods=L.make_score_mods(causal=pre_ln))
    want = steps.behind(flat, a.view(S * n, d)).view(S, n, d)
    torch.cuda.synchronize()
    assert layer.status() == L.OK and torch.equal(out, want)
    for _ in range(5):
        layer.forward(x, out)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    layer.close()
