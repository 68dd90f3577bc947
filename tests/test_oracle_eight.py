"""Pins of the oracle of the 8-bit operators and of the rotation: torch's own functions in float64, and cases worked by hand."""
import numpy as np
import pytest
import torch

from oracle import eight_oracle as E


def test_norms_against_torch():
    g = np.random.RandomState(1)
    x, r, gain, bias = g.randn(5, 40) * 3 + 1, g.randn(5, 40), g.rand(40) + 0.5, g.randn(40)
    t = torch.tensor(x + r)
    want = torch.nn.functional.layer_norm(t, (40,), torch.tensor(gain), torch.tensor(bias), 1e-5).numpy()
    assert np.allclose(E.norm(x, "layer", gain, bias, residual=r)[1], want, rtol=1e-12, atol=1e-12)
    want = torch.nn.functional.rms_norm(t, (40,), torch.tensor(gain), 1e-5).numpy()
    assert np.allclose(E.norm(x, "rms", gain, residual=r)[1], want, rtol=1e-12, atol=1e-12)
    h, y = E.norm(x, "none", residual=r)
    assert h is y and np.array_equal(h, x + r)


def test_a_row_by_hand():
    v, s = E.eight_bits([[12.7, -6.4, 0.25, 0.0]], "int8")
    assert np.allclose(s, 0.1) and np.array_equal(v, [[127, -64, 2, 0]])          # 2.5 steps: to even
    v, s = E.eight_bits([[0.0, 0.0], [np.inf, 1.0], [np.nan, 1.0]], "e4m3")
    assert s[0] == 0 and np.isnan(s[1]) and np.isnan(s[2]) and not v.any()


def test_e4m3_against_torch():
    x = np.concatenate([np.linspace(-448, 448, 4001), np.linspace(-0.05, 0.05, 4001), 2.0 ** np.arange(-12, 9), [0.0, 448.0, 464.0]])
    want = torch.tensor(np.clip(x, -448, 448), dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(E.e4m3(np.float32(x)), want)


@pytest.mark.parametrize("act", ["none", "gelu_erf", "gelu_tanh"])
def test_dense_against_torch(act):
    g = np.random.RandomState(2)
    a, w, sa, sw, b, r = g.randint(-127, 128, (3, 32)), g.randint(-127, 128, (7, 32)), g.rand(3) / 100, g.rand(7) / 100, g.randn(7), g.randn(3, 7)
    z = torch.nn.functional.linear(torch.tensor(a * sa[:, None]), torch.tensor(w * sw[:, None]), torch.tensor(b))
    f = {"none": lambda t: t, "gelu_erf": torch.nn.functional.gelu, "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[act]
    y, zz = E.dense(a, sa, w, sw, b, act, r)
    assert np.allclose(y, (f(z) + torch.tensor(r)).numpy(), rtol=1e-12, atol=1e-12) and np.allclose(zz, z.numpy())


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_turns_pairs(interleaved):
    g = np.random.RandomState(3)
    x, f = g.randn(4, 2, 64), 10000.0 ** (-np.arange(16) / 16)
    y = E.rotate(x, [0, 1, 7, 100000], f, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))                        # lengths stay
    a, b = (2, 3) if interleaved else (1, 17)
    z = (x[2, 1, a] + 1j * x[2, 1, b]) * np.exp(7j * f[1])
    assert np.allclose([y[2, 1, a], y[2, 1, b]], [z.real, z.imag])
    # products of queries and keys depend on the distance alone
    q, k = x[:1, :1], x[1:2, 1:]
    dot = lambda p: float((E.rotate(q, [p + 5], f, interleaved) * E.rotate(k, [p], f, interleaved)).sum())
    assert abs(dot(0) - dot(123456)) < 1e-9
