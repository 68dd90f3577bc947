"""What the attention operators refuse before anything touches a device (plain host checks: no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2512_16843_b200 import binding as L

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def status_of(fn, *a, **kw):
    with pytest.raises(L.LLMCacheError) as e:
        fn(*a, **kw)
    return e.value.status


def qkv(S=2, n=8, H=4, HK=2):
    return (torch.zeros(S, n, H, 64, dtype=BF), torch.zeros(S, n, HK, 64, dtype=BF), torch.zeros(S, n, HK, 64, dtype=BF),
            torch.zeros(S, n, H, 64, dtype=BF))


@pytest.mark.parametrize("change,status", [
    (dict(q=lambda t: t.float()), L.ERR_ARG),
    (dict(k=lambda t: t.transpose(-1, -2)), L.ERR_SHAPE),
    (dict(k=lambda t: t[:, :, :1].expand(-1, -1, 2, -1)), L.ERR_ARG),            # a stride of zero
    (dict(v=lambda t: t[:, :4]), L.ERR_SHAPE),
    (dict(out=lambda t: t[:, :, :2]), L.ERR_SHAPE),
    (dict(k=lambda t: torch.zeros(2, 8, 3, 64, dtype=BF), v=lambda t: torch.zeros(2, 8, 3, 64, dtype=BF)), L.ERR_SHAPE),
    (dict(q=lambda t: torch.zeros(t.numel() + 4, dtype=BF)[4:].view(t.shape)), L.ERR_ARG),          # 8-byte alignment
    (dict(q=lambda t: torch.zeros(2, 8, 4, 68, dtype=BF)[..., :64]), L.ERR_ARG),                    # a stride of 68
    (dict(lse=torch.zeros(2, 8, 3)), L.ERR_SHAPE),
    (dict(lse=torch.zeros(2, 8, 4, dtype=torch.float64)), L.ERR_ARG),
    (dict(mods=dict(cap=-1.0)), L.ERR_ARG),
    (dict(mods=dict(cap=1e-9)), L.ERR_ARG),
    (dict(mods=dict(cap=float("nan"))), L.ERR_ARG),
    (dict(mods=dict(scale=-0.1)), L.ERR_ARG),
    (dict(mods=dict(scale=float("inf"))), L.ERR_ARG),
    (dict(mods=dict(slopes=torch.zeros(3))), L.ERR_SHAPE),
    (dict(mods=dict(table=torch.zeros(4, 6))), L.ERR_SHAPE),
    (dict(mods=dict(table=torch.zeros(4, 2051))), L.ERR_SHAPE),
    (dict(mods=dict(doc=torch.zeros(2, 9, dtype=I32))), L.ERR_SHAPE),
    (dict(mods=dict(doc=torch.zeros(2, 8, dtype=torch.int64))), L.ERR_ARG),
    (dict(mods=dict(prefix=torch.zeros(2, dtype=I32))), L.ERR_ARG),                                 # only with causal
    (dict(mods=dict(causal=True, prefix=torch.zeros(3, dtype=I32))), L.ERR_SHAPE),
])
def test_attention_refuses(change, status):
    a = dict(zip(("q", "k", "v", "out"), qkv()))
    for name, f in change.items():
        if callable(f):
            a[name] = f(a[name])

    def call():
        m = L.make_score_mods(**change["mods"]) if "mods" in change else None
        L.llmcache_attention(a["q"], a["k"], a["v"], a["out"], mods=m, lse=change.get("lse"), stream=0)

    assert status_of(call) == status


def test_attention_of_an_empty_batch_is_valid_and_null_arguments_are_not():
    q, k, v, out = (t[:0] for t in qkv())
    L.llmcache_attention(q, k, v, out, stream=0)
    lib, r = L.lib(), L.Rows(None, 0, 0, 0)
    p = C.byref(r)
    assert lib.llmcache_attention(None, p, p, p, 1, 1, 1, 1, None, None, None, None) == L.ERR_ARG
    assert lib.llmcache_attention(p, p, p, p, 1, 1, 1, 1, None, None, None, None) == L.ERR_ARG
    assert lib.llmcache_attention(p, p, p, p, 1, 0, 1, 1, None, None, None, None) == L.ERR_SHAPE
    m = L.make_score_mods()
    m.struct_size = 8
    assert lib.llmcache_attention(p, p, p, p, 1, 1, 1, 1, None, C.byref(m), None, None) == L.ERR_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(heads=3), L.ERR_SHAPE), (dict(heads=0), L.ERR_SHAPE), (dict(max_seqs=0), L.ERR_SHAPE), (dict(max_rows=0), L.ERR_SHAPE),
    (dict(max_len=0), L.ERR_SHAPE), (dict(page=8), L.ERR_SHAPE), (dict(page=48), L.ERR_SHAPE), (dict(page=512), L.ERR_SHAPE),
    (dict(dh=128), L.ERR_SHAPE), (dict(max_len=(1 << 30) + 1), L.ERR_SHAPE),
])
def test_cache_descriptions_that_are_refused(kw, status):
    def make(page=16, dh=64, **k):
        a = dict(heads=4, max_seqs=2, max_rows=8, max_len=64)
        a.update(k)
        pages = torch.zeros(4, 2, page, dh, dtype=BF)
        L.llmcache_kv_bytes(L.make_kv_desc(pages, pages.clone(), **a))

    assert status_of(make, **kw) == status


def test_cache_needs_dense_pages_a_large_enough_workspace_and_a_device():
    pages = torch.zeros(4, 2, 16, 64, dtype=BF)
    a = dict(heads=4, max_seqs=2, max_rows=8, max_len=64)
    assert status_of(L.make_kv_desc, pages.transpose(1, 2), pages.transpose(1, 2), **a) == L.ERR_SHAPE
    both = torch.zeros(4, 2, 2, 16, 64, dtype=BF)                     # K and V of a page side by side: a page stride
    need = L.llmcache_kv_bytes(L.make_kv_desc(both[:, 0], both[:, 1], **a))
    assert need > 0
    small = torch.zeros(need // 2, dtype=torch.uint8)
    d = L.make_kv_desc(pages, pages.clone(), **a)
    d.workspace, d.workspace_bytes = (small.data_ptr() + 255) // 256 * 256, need // 4
    assert status_of(L.llmcache_kv_create, d) == L.ERR_NOMEM
    d.workspace = d.workspace + 16
    assert status_of(L.llmcache_kv_create, d) == L.ERR_ARG
    d.struct_size = 4
    assert status_of(L.llmcache_kv_bytes, d) == L.ERR_ARG
    if not torch.cuda.is_available():
        assert status_of(L.llmcache_kv_create, L.make_kv_desc(pages, pages.clone(), **a)) == L.ERR_CUDA
    lib = L.lib()
    assert lib.llmcache_kv_attention(None, None, None) == L.ERR_ARG and lib.llmcache_kv_evict(None, None, None) == L.ERR_ARG
    assert lib.llmcache_kv_destroy(None) == L.ERR_ARG and lib.llmcache_kv_status(None) == L.ERR_ARG
    assert lib.llmcache_layer_extend(None, None, None, None, None, None) == L.ERR_ARG
    assert lib.llmcache_layer_score_mods(None, None) == L.ERR_ARG


def test_struct_layouts_match_the_header():
    assert C.sizeof(L.ScoreMods) == 5 * 4 + 4 + 4 * 8
    assert C.sizeof(L.Rows) == 4 * 8
    assert C.sizeof(L.KVDesc) == 9 * 4 + 4 + 2 * 8 + 8 + 2 * 8
    assert C.sizeof(L.KVChunk) == 4 * 4 + 3 * 8 + 8 + 4 * 32 + 4 * 8 + 8 + 8
    assert C.sizeof(L.KVEviction) == 7 * 4 + 4 + 6 * 8 + 8 + 2 * 8 + 8 + 8
