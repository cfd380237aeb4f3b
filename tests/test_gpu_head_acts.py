"""Activations of the linear layer and their derivatives on the GPU, value by value: a layer with one input, one output and the
weight 1 hands z on as it is, so y is act(z) and dx is act'(z)."""
import numpy as np
import pytest

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import get, rounded, up

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
