"""What the 8-bit operators, the rotated append and the layer's settings refuse before anything touches a device (plain host
checks: no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2512_16843_b200 import binding as L

BF, F32, I32, F8 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn


def status_of(fn, *a, **kw):
    with pytest.raises(L.LLMCacheError) as e:
        fn(*a, **kw)
    return e.value.status


def rows(r=4, c=64, dtype=BF):
    return torch.zeros(r, c, dtype=dtype)


@pytest.mark.parametrize("change,status", [
    (dict(x=rows(dtype=F32)), L.ERR_ARG),
    (dict(x=rows()[0]), L.ERR_ARG),
    (dict(x=rows(4, 128)[:, ::2]), L.ERR_SHAPE),
    (dict(x=rows(4, 60), q=None, scale=None, out=rows(4, 60)), L.ERR_SHAPE),                 # a width that is no multiple of 8
    (dict(x=rows(4, 16392), q=None, scale=None, out=rows(4, 16392)), L.ERR_SHAPE),
    (dict(x=rows(4, 68)[:, :64]), L.ERR_SHAPE),                                              # a leading dimension of 68
    (dict(x=rows(1, 64).expand(4, 64)), L.ERR_SHAPE),                                        # a leading dimension of 0
    (dict(x=torch.zeros(4 * 64 + 4, dtype=BF)[4:].view(4, 64)), L.ERR_ARG),                  # 8-byte alignment
    (dict(residual=rows(3)), L.ERR_SHAPE),
    (dict(residual=rows(dtype=F32)), L.ERR_ARG),
    (dict(total=rows(4, 72)), L.ERR_SHAPE),
    (dict(out=rows(5)), L.ERR_SHAPE),
    (dict(q=rows(dtype=torch.uint8)), L.ERR_ARG),
    (dict(q=rows(4, 56, torch.int8)), L.ERR_SHAPE),
    (dict(q=None), L.ERR_ARG),                                                               # a scale without q
    (dict(scale=None), L.ERR_ARG),
    (dict(scale=torch.zeros(3)), L.ERR_SHAPE),
    (dict(q=None, scale=None), L.ERR_ARG),                                                   # nothing to write
    (dict(gain=torch.zeros(63)), L.ERR_SHAPE),
    (dict(gain=torch.zeros(64, dtype=BF)), L.ERR_ARG),
    (dict(kind="none", gain=torch.zeros(64)), L.ERR_ARG),
    (dict(kind="none", bias=torch.zeros(64)), L.ERR_ARG),
    (dict(kind="batch"), L.ERR_ARG),
    (dict(eps=float("nan")), L.ERR_ARG),
    (dict(eps=float("inf")), L.ERR_ARG),
    (dict(eps=1e300), L.ERR_ARG),
    (dict(eps="small"), L.ERR_ARG),
    (dict(n_rows_dev=torch.zeros(1)), L.ERR_ARG),
    (dict(n_rows_dev=torch.zeros(0, dtype=I32)), L.ERR_ARG),
])
def test_norm_refuses(change, status):
    a = dict(x=rows(), q=rows(dtype=torch.int8), scale=torch.zeros(4), stream=0)
    a.update(change)
    assert status_of(L.llmcache_norm, **a) == status


@pytest.mark.parametrize("change,status", [
    (dict(a=rows()), L.ERR_ARG),
    (dict(w=rows(8, 64, F8)), L.ERR_ARG),                                                    # two formats
    (dict(w=rows(8, 48, torch.int8)), L.ERR_SHAPE),
    (dict(a=rows(4, 72, torch.int8), w=rows(8, 72, torch.int8)), L.ERR_SHAPE),               # k no multiple of 16
    (dict(a=rows(4, 72, torch.int8)[:, :64]), L.ERR_SHAPE),                                  # a leading dimension of 72
    (dict(a=rows(4, 131072, torch.int8), w=rows(8, 131072, torch.int8)), L.ERR_SHAPE),
    (dict(a=torch.zeros(4 * 64 + 8, dtype=torch.int8)[8:].view(4, 64)), L.ERR_ARG),          # 8-byte alignment
    (dict(a_scale=None), L.ERR_ARG), (dict(w_scale=None), L.ERR_ARG), (dict(out=None), L.ERR_ARG),
    (dict(a_scale=torch.zeros(5)), L.ERR_SHAPE), (dict(w_scale=torch.zeros(4)), L.ERR_SHAPE),
    (dict(a_scale=torch.zeros(4, dtype=torch.float64)), L.ERR_ARG),
    (dict(bias=torch.zeros(7)), L.ERR_SHAPE), (dict(bias=torch.zeros(8, dtype=BF)), L.ERR_ARG),
    (dict(out=rows(4, 9)), L.ERR_SHAPE), (dict(out=rows(4, 8, F32)), L.ERR_ARG),
    (dict(out=rows(4, 12)[:, :8]), L.ERR_SHAPE),                                             # a leading dimension of 12
    (dict(residual=rows(3, 8)), L.ERR_SHAPE), (dict(residual=rows(4, 12)[:, :8]), L.ERR_SHAPE),
    (dict(w_scale=torch.zeros(9)[1:]), L.ERR_ARG), (dict(bias=torch.zeros(9)[1:]), L.ERR_ARG),     # 4-byte alignment
    (dict(act="relu"), L.ERR_ARG),
    (dict(n_rows_dev=3), L.ERR_ARG),
])
def test_dense_refuses(change, status):
    a = dict(a=rows(4, 64, torch.int8), a_scale=torch.zeros(4), w=rows(8, 64, torch.int8), w_scale=torch.zeros(8), out=rows(4, 8), stream=0)
    a.update(change)
    assert status_of(L.llmcache_dense, **a) == status


def test_calls_without_rows_are_valid_and_null_arguments_are_not():
    e = rows(0)
    L.llmcache_norm(e, q=rows(0, 64, F8), scale=torch.zeros(0), stream=0)
    L.llmcache_dense(rows(0, 64, F8), torch.zeros(0), rows(8, 64, F8), torch.zeros(8), rows(0, 8), stream=0)
    lib = L.lib()
    assert lib.llmcache_norm(None, None) == L.ERR_ARG and lib.llmcache_dense(None, None) == L.ERR_ARG
    n = L.NormArgs()
    assert lib.llmcache_norm(C.addressof(n), None) == L.ERR_ARG                               # struct_size
    n.struct_size, n.n_rows, n.cols = C.sizeof(n), 1, 64
    assert lib.llmcache_norm(C.addressof(n), None) == L.ERR_ARG                               # no x
    n.n_rows = 1 << 31
    assert lib.llmcache_norm(C.addressof(n), None) == L.ERR_SHAPE
    d = L.DenseArgs()
    assert lib.llmcache_dense(C.addressof(d), None) == L.ERR_ARG
    d.struct_size, d.format, d.m, d.n, d.k = C.sizeof(d), L.BF16, 1, 8, 64
    assert lib.llmcache_dense(C.addressof(d), None) == L.ERR_ARG                              # not an 8-bit format
    d.format = L.I8
    assert lib.llmcache_dense(C.addressof(d), None) == L.ERR_ARG                              # no a
    d.m = d.n = (1 << 31) - 1
    assert lib.llmcache_dense(C.addressof(d), None) == L.ERR_SHAPE                            # more tiles than a grid counts
    assert lib.llmcache_kv_append(None, None, None) == L.ERR_ARG
    for f in (lambda: lib.llmcache_layer_rms(None, 1), lambda: lib.llmcache_layer_rotation(None, None),
              lambda: lib.llmcache_layer_quantise(None, L.I8, None, 0, None), lambda: lib.llmcache_layer_quantise_bytes(None, None)):
        assert f() == L.ERR_ARG


@pytest.mark.parametrize("freq,status", [
    (torch.zeros(32), L.ERR_ARG), (torch.zeros(4, 8, dtype=torch.float64), L.ERR_ARG), (torch.zeros(64, dtype=torch.float64)[::2], L.ERR_ARG),
    (torch.zeros(0, dtype=torch.float64), L.ERR_SHAPE), (torch.zeros(12, dtype=torch.float64), L.ERR_SHAPE),
    (torch.zeros(40, dtype=torch.float64), L.ERR_SHAPE), ([1.0] * 32, L.ERR_ARG),
])
def test_rotations_that_are_refused(freq, status):
    assert status_of(L.make_rotation, freq) == status


def stub_cache(heads=4, kv_heads=2):
    """A KVCache on the host without its handle: the wrapper's checks come before the library is called (which refuses the null)."""
    c = L.KVCache.__new__(L.KVCache)
    c.heads, c.kv_heads, c.device, c.handle = heads, kv_heads, -1, None
    return c


@pytest.mark.parametrize("change,status", [
    (dict(k_new=torch.zeros(6, 3, 64, dtype=BF)), L.ERR_SHAPE),
    (dict(k_new=torch.zeros(6, 2, 64)), L.ERR_ARG),
    (dict(v_new=torch.zeros(5, 2, 64, dtype=BF)), L.ERR_SHAPE),
    (dict(v_new=None), L.ERR_ARG),
    (dict(q=torch.zeros(6, 4, 64, dtype=BF)), L.ERR_ARG),                                    # without q_out
    (dict(q=torch.zeros(6, 2, 64, dtype=BF), q_out=torch.zeros(6, 4, 64, dtype=BF)), L.ERR_SHAPE),
    (dict(q=torch.zeros(6, 4, 64, dtype=BF), q_out=torch.zeros(6, 4, 64)), L.ERR_ARG),
    (dict(lens=None), L.ERR_ARG), (dict(pages=None), L.ERR_ARG), (dict(cu_rows=None), L.ERR_ARG),
    (dict(cu_rows=torch.zeros(2, dtype=I32)), L.ERR_SHAPE),
    (dict(first=torch.zeros(3, dtype=I32)), L.ERR_SHAPE),
    (dict(positions=torch.zeros(2, 4, 32, dtype=I32)), L.ERR_SHAPE),
    (dict(rotation=L.make_rotation(torch.zeros(32, dtype=torch.float64))), L.ERR_ARG),       # (what is left: no handle)
])
def test_append_refuses(change, status):
    a = dict(k_new=torch.zeros(6, 2, 64, dtype=BF), v_new=torch.zeros(6, 2, 64, dtype=BF), cu_rows=torch.zeros(3, dtype=I32),
             lens=torch.zeros(2, dtype=I32), pages=torch.zeros(2, 2, dtype=I32), stream=0)
    a.update(change)
    assert status_of(stub_cache().append, **a) == status


def test_struct_layouts_match_the_header():
    assert C.sizeof(L.NormArgs) == L._NORM.size == 7 * 4 + 4 + 8 + 5 * 16 + 3 * 8
    assert C.sizeof(L.DenseArgs) == L._DENSE.size == 7 * 4 + 4 + 8 + 2 * 24 + 8 + 2 * 16
    assert C.sizeof(L.KVNew) == L._NEW.size == 4 * 4 + 3 * 8 + 4 * 32 + 4 * 8
    assert C.sizeof(L.Rotation) == 3 * 4 + 4 + 8


def test_layer_settings_that_the_wrapper_refuses():
    layer = L.Layer.__new__(L.Layer)
    layer.desc = L.LayerDesc()
    layer.desc.device, layer.handle = 0, None
    assert status_of(layer.quantise, "int4") == L.ERR_ARG
    assert status_of(layer.quantise, "int8", torch.zeros(16, dtype=torch.uint8)) == L.ERR_ARG                 # on the host
    assert status_of(layer.rotation, L.make_rotation(torch.zeros(32, dtype=torch.float64))) == L.ERR_ARG      # likewise
