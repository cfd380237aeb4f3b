"""Activations of the linear layer and their derivatives on the GPU, value by value: a layer with one input, one output and the
weight 1 hands z on as it is, so y is act(z) and dx is act'(z)."""
import numpy as np
import pytest

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import TOL32, ULP16, get, rounded, up

pytestmark = pytest.mark.gpu


def _through(z, act, dtype):
    """act(z) and act'(z) as the layer gives them; z in the type's values."""
    need_gpu()
    from paper_1904_03409_amd import head as hd
    r = hd.LinearRun.of(up(z[:, None], dtype), up(np.ones((1, 1)), dtype), act=act, dy=up(np.ones((len(z), 1)), dtype))
    r.forward()
    r.backward()
    return get(r.y)[:, 0], get(r.dx)[:, 0]


@pytest.mark.parametrize("n", [100, 5000])              # a backward in one launch, and in several
def test_gelu_derivative_has_no_bias(n):
    """A constant that is off shifts every value the same way; a rounding does not. Rounded constants of the gate (half a ulp of
    2.3, times z, ln 2 and the derivative's slope of at most 0.2) leave 3e-8, roundings of n values less."""
    for lo, hi in ((1.0, 2.0), (-2.0, -1.0)):
        z = rounded(np.linspace(lo, hi, n), "f32")
        g = _through(z, "gelu", "f32")[1]
        assert abs((g - ref.act_grad(z, "gelu")).mean()) <= 1e-7


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [120, 3000])
def test_tanh_keeps_small_values(n, dtype):
    """Every value against itself, not against the largest: eight roundings of 2^-24 (exp2, 1 - e, 1 + e, its reciprocal, the
    product, each up to one or two of them, over 1 - e of at least 0.39 e)."""
    z = np.geomspace(1e-36, 20.0, n // 2)
    z = rounded(np.concatenate([-z, z]), dtype)
    y, g = _through(z, "tanh", dtype)
    one = ULP16 if dtype == "bf16" else 0.0
    assert (np.abs(y - np.tanh(z)) <= (5e-7 + one) * np.abs(np.tanh(z))).all()
    # the derivative 1 / cosh^2: the exponent's rounding grows with z
    want = 1 / np.cosh(z) ** 2
    assert (np.abs(g - want) <= (1e-6 + 4e-7 * np.abs(z) + one) * want).all()
    assert _through(np.zeros(n), "tanh", dtype)[0].tolist() == [0.0] * n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "tanh", "silu", "gelu"])
@pytest.mark.parametrize("n", [90, 400])
def test_ends_of_the_range(n, act, dtype):
    """Values and derivatives from -40 to 40 and on to the type's largest value, each within the bar of its own size (of 1 for
    smaller ones) and of one rounding to the type."""
    big = np.array([1e3, 1e5, 1e10, 1e18, 2e19, 1e25, 1e30, 3e38])
    z = rounded(np.concatenate([np.linspace(-40, 40, n - 16), -big, big]), dtype)
    y, g = _through(z, act, dtype)
    c = np.clip(z, -1e3, 1e3)                           # (past it the derivative is at its end, and 64 bits overflow in it)
    wy, wg = ref.act(c, act), ref.act_grad(c, act)
    far = np.abs(z) > 1e3
    if act != "tanh":
        wy[far] = np.where((z[far] < 0) & (act != "none"), 0.0, z[far])
    one = ULP16 if dtype == "bf16" else 0.0
    for got, want in ((y, wy), (g, wg)):
        assert (np.abs(got - want) <= TOL32 * np.maximum(1, np.abs(want)) + one * np.abs(want)).all(), act
