"""The 64-bit references of the operators behind the recurrence against central differences (CPU)."""
import numpy as np
import pytest

from tests import head_ref as ref


def _diff(f, x, g, h=2.0 ** -17):
    """<df/dx, v> against differences for a few directions v."""
    rng = np.random.default_rng(1)
    for _ in range(4):
        v = rng.standard_normal(x.shape)
        num = (f(x + h * v) - f(x - h * v)) / (2 * h)
        # third derivatives of unit size: h^2 of them, and the rounding of f over h
        assert abs(num - (g * v).sum()) <= 1e-6 * max(1.0, abs(num)), (num, (g * v).sum())


@pytest.mark.parametrize("res", [False, True])
def test_norm(res):
    rng = np.random.default_rng(2)
    x, r, ga, be, dy, ds = (rng.standard_normal(s) for s in ((5, 7), (5, 7), (7,), (7,), (5, 7), (5, 7)))
    r = r if res else None
    loss = lambda x, ga, be: (ref.norm_fwd(x, r, ga, be, 1e-5)[1] * dy).sum() + ((ref.norm_fwd(x, r, ga, be, 1e-5)[0] * ds).sum() if res else 0)
    s, _, mu, rstd = ref.norm_fwd(x, r, ga, be, 1e-5)
    dx, dg, db = ref.norm_bwd(s, mu, rstd, ga, dy, ds if res else None)
    _diff(lambda v: loss(v, ga, be), x, dx)
    _diff(lambda v: loss(x, v, be), ga, dg)
    _diff(lambda v: loss(x, ga, v), be, db)


@pytest.mark.parametrize("name", ["none", "relu", "tanh", "silu", "gelu"])
def test_activations(name):
    z = np.random.default_rng(3).standard_normal((4, 9)) * 2
    z[np.abs(z) < 0.01] = 0.5                          # away from the step of relu's derivative
    w = np.random.default_rng(4).standard_normal(z.shape)
    _diff(lambda v: (ref.act(v, name) * w).sum(), z, w * ref.act_grad(z, name))


@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.3), (0.5, 0.0)])
def test_distill(tau, alpha):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 11))
    index = rng.integers(-1, 11, (6, 4))
    index[1] = -1                                      # a row without a teacher
    index[2, :2] = 3                                   # an index twice
    value = rng.standard_normal((6, 4))
    label = np.array([0, 4, -1, 10, 2, 11])
    grad = rng.standard_normal(6)
    _, d = ref.distill(x, index, value, label, grad, tau, alpha)
    _diff(lambda v: (ref.distill(v, index, value, label, grad, tau, alpha)[0] * grad).sum(), x, d)


def test_distill_of_the_full_distribution_is_zero_at_the_teacher():
    x = np.random.default_rng(6).standard_normal((3, 8))
    loss, d = ref.distill(x, np.tile(np.arange(8), (3, 1)), x.copy(), None, np.ones(3), 2.0, 1.0)
    assert np.abs(loss).max() < 1e-14 and np.abs(d).max() < 1e-15


def test_beam_by_hand():
    # two beams, three tokens, probabilities 1/2 1/4 1/4 and 3/4 1/8 1/8: totals log(1/2 * p), the second beam finished
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.75, 0.125, 0.125]]))
    score = np.log(np.array([[0.5, 0.5]]))
    s, parent, token, done = ref.beam(x, None, score, None, eos=0)
    assert parent.tolist() == [[1, 0]] and token.tolist() == [[0, 0]] and done.tolist() == [[1, 1]]
    assert np.allclose(np.exp(s), [[0.375, 0.25]])
    s, parent, token, done = ref.beam(x, None, score, np.array([[0, 1]], np.uint8), eos=2)
    assert parent.tolist() == [[1, 0]] and token.tolist() == [[-1, 0]] and done.tolist() == [[1, 0]]
    # the tie of two quarters goes to the lower token; a beam whose tokens are all forbidden has none
    legal = np.array([[0, 1, 1], [0, 0, 0]], np.uint8)
    s, parent, token, done = ref.beam(x, legal, score, None, eos=-1)
    assert parent.tolist() == [[0, 0]] and token.tolist() == [[1, 2]]
    s, parent, token, done = ref.beam(x, np.zeros((2, 3), np.uint8), score, None, eos=-1)
    assert np.all(s == -np.inf) and parent.tolist() == [[0, 1]] and token.tolist() == [[-1, -1]] and done.all()
