"""Score modifiers that a layer refuses: arrays of another shape or place than its attention would read."""
import ctypes as C

import pytest
import torch

from paper_2512_16843_b200 import binding as L

F32, I32 = torch.float32, torch.int32


def status_of(fn, *a, **kw):
    with pytest.raises(L.LLMCacheError) as e:
        fn(*a, **kw)
    return e.value.status


def layer_stub(heads, seq_len, device):
    """A Layer without its handle: the checks of the wrapper come before the library is called (which refuses a null handle)."""
    layer = L.Layer.__new__(L.Layer)
    layer.desc = L.LayerDesc()
    layer.desc.heads, layer.desc.seq_len, layer.desc.device = heads, seq_len, device
    layer.handle = None
    return layer


@pytest.mark.parametrize("mods", [
    dict(slopes=torch.zeros(3)), dict(slopes=torch.zeros(5)), dict(table=torch.zeros(3, 5)), dict(doc=torch.zeros(2, 9, dtype=I32)),
    dict(doc=torch.zeros(2, 7, dtype=I32)), dict(doc=torch.zeros(0, 8, dtype=I32)), dict(causal=True, prefix=torch.zeros(0, dtype=I32)),
])
def test_shapes_that_the_layer_does_not_have(mods):
    assert status_of(layer_stub(4, 8, -1).score_mods, L.make_score_mods(**mods)) == L.ERR_SHAPE       # (-1: tensors on the host)


@pytest.mark.parametrize("mods", [
    dict(slopes=torch.zeros(4)), dict(table=torch.zeros(4, 5)), dict(doc=torch.zeros(2, 8, dtype=I32)), dict(causal=True, prefix=torch.zeros(2, dtype=I32)),
])
def test_host_tensors(mods):
    assert status_of(layer_stub(4, 8, 0).score_mods, L.make_score_mods(**mods)) == L.ERR_ARG


def test_masks_know_how_many_sequences_they_have():
    doc, prefix = torch.zeros(2, 8, dtype=I32), torch.zeros(3, dtype=I32)
    assert status_of(L.make_score_mods, causal=True, doc=doc, prefix=prefix) == L.ERR_SHAPE
    m = L.make_score_mods(causal=True, doc=doc, prefix=prefix[:2])
    assert m.mask_seqs == 2 and L.make_score_mods(slopes=torch.zeros(4)).mask_seqs == 0
    q = torch.zeros(3, 8, 4, 64, dtype=torch.bfloat16)
    r = C.byref(L.Rows(q.data_ptr(), 8 * 256, 256, 64))
    assert L.lib().llmcache_attention(r, r, r, r, 3, 8, 4, 4, None, C.byref(m), None, None) == L.ERR_SHAPE


@pytest.mark.gpu
def test_layer_calls_with_more_sequences_than_the_masks():
    from tests.test_gpu_attention import BF, DEV, i32, layer_pair, rnd
    n, d, heads, S = 16, 128, 2, 4
    _, layer = layer_pair(n, d, heads, 256, S)
    x = rnd(S, n, d, seed=71)
    out, want = torch.full_like(x, 7.0), torch.zeros_like(x)
    doc = torch.zeros((S, n), dtype=I32, device=DEV)
    for masks in (dict(doc=doc[:2].contiguous()), dict(prefix=i32([3, 5])), dict(doc=doc[:2].contiguous(), prefix=i32([3, 5]))):
        layer.score_mods(L.make_score_mods(causal=True, **masks))
        assert status_of(layer.forward, x, out) == L.ERR_SHAPE
        a, b, c, e = (torch.zeros_like(x) for _ in range(4))
        assert status_of(L.llmcache_infer, None, [layer.handle], x, S, None, a, b, c, e, None) == L.ERR_SHAPE
        layer.forward(x[:2], out[:2])
    torch.cuda.synchronize()
    assert torch.all(out[2:] == 7.0) and torch.isfinite(out[:2].float()).all()
    # a refusal leaves the modifiers that were there
    layer.score_mods(L.make_score_mods(causal=True, slopes=torch.ones(heads, device=DEV)))
    layer.forward(x, want)
    assert status_of(layer.score_mods, L.make_score_mods(causal=True, slopes=torch.ones(heads + 1, device=DEV))) == L.ERR_SHAPE
    assert status_of(layer.score_mods, L.make_score_mods(causal=True, slopes=torch.ones(heads))) == L.ERR_ARG
    layer.forward(x, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # the library itself looks where the arrays are
    raw, near = L.make_score_mods(causal=True), torch.ones(heads)
    raw.slopes = near.data_ptr()
    assert status_of(L.llmcache_layer_score_mods, layer.handle, raw) == L.ERR_ARG
    layer.close()
