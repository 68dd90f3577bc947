"""Every form of the 8-bit product's kernel on the same odd shapes, whatever the estimated times would choose.

Tolerances: those of test_gpu_eight.py, against the float64 oracle.  Whole-number sums have one value, so in int8 all forms give the same bits."""
import pytest
import torch

from paper_2512_16843_b200 import binding as L
from tests.test_gpu_eight import BF, DEV, check_dense, eight_matrix, filled, rnd

pytestmark = pytest.mark.gpu

FORMS = {"pairs": L.DENSE_PAIRS, "128": L.DENSE_128, "64": L.DENSE_64, "clusters of 2": L.DENSE_CLUSTERS_2, "clusters of 4": L.DENSE_CLUSTERS_4,
         "clusters of 8": L.DENSE_CLUSTERS_8, "few": L.DENSE_FEW}
PARTS = {L.DENSE_CLUSTERS_2: 2, L.DENSE_CLUSTERS_4: 4, L.DENSE_CLUSTERS_8: 8}


@pytest.fixture
def form():
    """Sets a form (0: the rule's) for the test that asks for it."""
    a, sa = eight_matrix(1, 16, "int8", 1)
    L.llmcache_dense(a, sa, a, sa, torch.zeros((1, 8), dtype=BF, device=DEV)[:, :1])      # the device is set up with the first call
    yield lambda f: L.llmcache_dense_debug_knobs(0, L.KNOB_DENSE_FORM * f)
    L.llmcache_dense_debug_knobs(0, 0)


def serves(f, m, k):
    return m <= 32 if f == L.DENSE_FEW else -(-k // 128) >= PARTS.get(f, 1)


def inputs(m, n, k, to, bias, residual):
    a, sa = eight_matrix(m, k, to, m + k, ld=k + 32)
    w, sw = eight_matrix(n, k, to, n + k + 1, ld=k + 16)
    size = 40.0 if to == "int8" else 100.0
    ld = -(-n // 8) * 8 + 8
    g = torch.Generator(device=DEV).manual_seed(m * n)
    b = torch.randn(n, generator=g, device=DEV) * 0.5 if bias else None
    return a, sa / size, w, sw / (size * k ** 0.5), b, rnd(m, ld, seed=3)[:, :n] if residual else None, ld


SHAPES = [
    # m, n, k, bias, act, residual
    (1, 1, 16, True, "none", True),
    (3, 5, 2000, True, "gelu_tanh", False),
    (17, 131, 144, True, "gelu_erf", True),
    (25, 321, 1040, False, "none", True),
    (32, 200, 80, True, "gelu_tanh", True),
    (31, 72, 4112, True, "none", False),
    (33, 100, 208, True, "gelu_erf", False),
    (129, 63, 1040, True, "none", True),
    (257, 259, 272, False, "gelu_tanh", True),
    (300, 1031, 1168, True, "gelu_erf", True),
    (1030, 515, 4016, True, "none", False),
]


@pytest.mark.parametrize("m,n,k,bias,act,residual", SHAPES)
@pytest.mark.parametrize("to", ["int8", "e4m3"])
def test_all_forms_against_the_oracle(form, m, n, k, bias, act, residual, to):
    a, sa, w, sw, b, r, ld = inputs(m, n, k, to, bias, residual)
    ran, first = 0, None
    for name, f in FORMS.items():
        form(f)
        out, whole = filled(m, ld, n, BF)
        call = lambda o, **kw: L.llmcache_dense(a, sa, w, sw, o, bias=b, act=act, residual=r, **kw)
        if not serves(f, m, k):
            with pytest.raises(L.LLMCacheError) as e:
                call(out)
            assert e.value.status == L.ERR_UNSUPPORTED
            continue
        call(out)
        torch.cuda.synchronize()
        check_dense(out, a, sa, w, sw, to, b, act, r)
        assert torch.all(whole[:, n:] == 7), name
        again = torch.zeros_like(whole)[:, :n]
        call(again)
        assert torch.equal(again, out), name
        if first is None:
            first = out
        elif to == "int8":
            assert torch.equal(out, first), name
        for count in {0, 1, m // 2, m - 1, m + 5}:       # rows counted on the device: the others stay
            part, _ = filled(m, ld, n, BF)
            call(part, n_rows_dev=torch.tensor([count], dtype=torch.int32, device=DEV))
            c = min(count, m)
            assert torch.equal(part[:c], out[:c]) and torch.all(part[c:] == 7), (name, count)
        ran += 1
    assert ran >= 3 and L.llmcache_dense_status() == L.OK


@pytest.mark.parametrize("m,n,k", [(17, 2300, 400), (25, 9868, 96), (26, 1048, 432), (31, 25885, 80), (32, 18011, 208)])
@pytest.mark.parametrize("to", ["int8", "e4m3"])
@pytest.mark.parametrize("act,residual", [("none", True), ("gelu_erf", False), ("gelu_tanh", True)])
def test_up_to_32_rows_by_the_rule_and_through_registers(form, m, n, k, to, act, residual):
    """Widths at which the estimates send 17 to 32 rows through registers, e4m3 too."""
    a, sa, w, sw, b, r, ld = inputs(m, n, k, to, True, residual)
    call = lambda o: L.llmcache_dense(a, sa, w, sw, o, bias=b, act=act, residual=r)
    outs = []
    for f in (0, L.DENSE_FEW, L.DENSE_64):
        form(f)
        out, whole = filled(m, ld, n, BF)
        call(out)
        torch.cuda.synchronize()
        check_dense(out, a, sa, w, sw, to, b, act, r)
        assert torch.all(whole[:, n:] == 7)
        outs.append(out)
    if to == "int8":
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_forms_that_are_not_there(form):
    with pytest.raises(L.LLMCacheError) as e:
        form(8)
    assert e.value.status == L.ERR_ARG
    form(L.DENSE_FEW)                                    # and a refused one changes nothing
    with pytest.raises(L.LLMCacheError):
        form(15)
    a, sa, w, sw, b, r, ld = inputs(40, 64, 64, "int8", False, False)
    out = torch.zeros((40, 64), dtype=BF, device=DEV)
    with pytest.raises(L.LLMCacheError) as e:
        L.llmcache_dense(a, sa, w, sw, out)
    assert e.value.status == L.ERR_UNSUPPORTED
    form(0)
    L.llmcache_dense(a, sa, w, sw, out)
    check_dense(out, a, sa, w, sw, "int8", None, "none", None)
