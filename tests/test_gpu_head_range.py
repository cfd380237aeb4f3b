"""Logits and states whose finite values are far from 1 (additive masks of -1e9 and below, the type's lowest value), on the GPU
against 64 bits."""
import numpy as np
import pytest

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import close, get, rng_for, rounded, up

pytestmark = pytest.mark.gpu
LOWEST = float(np.finfo(np.float32).min)
MASKS = [-1e8, -4e8, -1e9, -1.7e9, -3e9, -1e10, -3e10, -1e12, -1e20, -1e25, -1e30, -1e37, LOWEST, 3e8, 1e9, 3e10, 1e12, 1e20, 1e30]


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5, 0.01, 100.0])
@pytest.mark.parametrize("V", [90, 3000, 40000])
def test_distill_of_far_logits(V, tau, dtype):
    """Rows of one far value (every token alike), rows with it in a half, and rows whose largest is far with its neighbours in the
    type beside it."""
    hd = _hd()
    rng = rng_for("far", V, tau, dtype)
    K, kinds = 4, 3
    R = kinds * len(MASKS)
    x = 2 * rng.standard_normal((R, V))
    index = np.tile(np.array([V - 1, V - 3, V - 20, V - 33], np.int32), (R, 1))
    for i, c in enumerate(MASKS):
        x[kinds * i] = c
        if c < 0:
            x[kinds * i + 1, : V // 2] = c
        else:
            x[kinds * i + 1, V // 2:] = c               # (what is asked for is among the largest)
        step = 2.0 ** (np.floor(np.log2(abs(c))) - (23 if dtype == "f32" else 7))
        x[kinds * i + 2] = c - step * rng.integers(0, 3, V) if c != LOWEST else c
        x[kinds * i + 2, V - 1] = c
    x = rounded(x, dtype)
    x[np.isinf(x)] = LOWEST if dtype == "f32" else rounded(np.array([-3.38e38]), dtype)[0]
    value = rng.standard_normal((R, K)).astype(np.float32)
    label = np.full(R, V - 1, np.int32)
    grad = rng.standard_normal(R).astype(np.float32)
    # the loss depends on differences alone; in 64 bits they are taken first
    d64 = x - x.max(1, keepdims=True)
    tau32 = float(np.float32(tau))
    loss, d = ref.distill(d64, index, value.astype(np.float64), label, grad.astype(np.float64), tau32, 0.5)
    r = hd.DistillRun.of(up(x, dtype), up(index), up(value), up(label), up(grad), tau32, 0.5)
    for name in ("step", "apart"):
        r.loss.fill_(7)
        r.dlogits.fill_(7)
        if name == "step":
            r.step()
        else:
            r.forward()
            r.backward()
        got, gd = get(r.loss), get(r.dlogits)
        assert np.isfinite(got).all() and np.isfinite(gd).all(), [MASKS[i // kinds] for i in np.nonzero(~np.isfinite(got))[0]]
        # every row within the bar of its own size; a difference of logits is rounded once, and divided by tau
        bar = 1e-5 * np.maximum(1, np.abs(loss)) + 2.0 ** -22 * 0.5 * tau32 * np.abs(d64[:, index[0]]).max(1)
        assert (np.abs(got - loss) <= bar).all(), np.array(MASKS)[np.nonzero(np.abs(got - loss) > bar)[0] // kinds]
        size = (np.abs(grad) * (0.5 * tau32 + 0.5))[:, None]
        one = 2.0 ** -8 * np.abs(d) if dtype == "bf16" else 0.0
        assert (np.abs(gd - d) <= 1e-5 * size + one).all()


def _beam_of_far_logits(V, B, dtype):
    """Searches of two beams, the second of one far value or with far ranges of a wave's, a thread's or a chunk's tokens."""
    hd = _hd()
    rng = rng_for("bfar", V, B, dtype)
    for c in MASKS[::2] if B * V > 1 << 20 else MASKS:
        x = rounded(2 * rng.standard_normal((2 * B, V)), dtype)
        for b in range(B):
            row = x[2 * b + 1]
            kind = b % 4
            if kind == 0:
                row[:] = c
            elif kind == 1:
                row[: V // 2] = c
            elif kind == 2:
                row[V // 4: V // 4 + max(1, V // 3)] = c
            else:
                row[np.arange(V) % 1024 < 512] = c      # (all that some threads have)
        x = rounded(x, dtype)
        x[np.isinf(x)] = LOWEST if dtype == "f32" else rounded(np.array([-3.38e38]), dtype)[0]
        score = np.tile(np.array([[-30.0, -2.0]], np.float32), (B, 1))
        run = hd.BeamRun.of(up(x, dtype), up(score))
        run.select()
        got = [t.cpu().numpy() for t in (run.score_next, run.parent, run.token)]
        assert np.isfinite(got[0]).all(), (c, got[0])
        few = np.unique(np.r_[np.arange(min(B, 4)), np.arange(max(0, B - 4), B)])
        rows = (2 * few[:, None] + np.arange(2)).reshape(-1)
        want = ref.beam(x[rows].astype(np.float32), None, score[few], None, -1)
        got = [g[few] for g in got]
        close(got[0].astype(np.float64), want[0].astype(np.float64), "f32", f"score_next {c}")
        assert np.array_equal(got[1], want[1]), c
        # (where two totals are within rounding of each other their order is the log sum's)
        apart = np.abs(want[0][:, 0] - want[0][:, 1]) > 1e-5
        equal = want[0][:, 0] == want[0][:, 1]
        far = (few % 4 == 0) | equal
        assert np.array_equal(got[2][apart | far], want[2][apart | far]), c


@pytest.mark.parametrize("V", [50, 700])
def test_beam_of_far_logits_in_a_workgroup(V):
    _beam_of_far_logits(V, 4, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [33000, 131072])
def test_beam_of_far_logits_in_chunks(V, dtype):
    _beam_of_far_logits(V, 4, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", [(4, 5003), (4, 9000), (160, 33000)])
def test_beam_of_far_logits_in_rows(B, V, dtype):
    _beam_of_far_logits(V, B, dtype)


@pytest.mark.parametrize("width", [1, 2, 3, 4, 7, 33, 100, 200, 257, 515, 1030])
def test_norm_backward_of_rows_far_from_zero(width):
    """Rows of one large value: no deviation, so xh is 0 and dx = rstd (g - mean g), whatever mean times rstd would be."""
    hd = _hd()
    rng = rng_for("far rows", width)
    rows, eps = 300, 1e-12
    x = np.tile(2.0 ** 113 * rng.choice([-1.0, 1.0], (rows, 1)), (1, width))
    dy = rounded(rng.standard_normal((rows, width)), "f32")
    r = hd.NormRun.of(up(x, "f32"), up(np.ones(width), "f32"), up(np.zeros(width), "f32"), dy=up(dy, "f32"), eps=eps)
    assert not get(r.forward()).any()
    r.backward()
    rstd = get(r.rstd)
    assert np.array_equal(get(r.mean), x[:, 0])
    want, _, db = ref.norm_bwd(x, x[:, 0], rstd, None, dy, None)
    close(r.dx, want, "f32", "dx", extra=1e-6 * (rstd * np.abs(dy).max())[:, None])
    assert not get(r.dgamma).any()
    close(r.dbeta, db, "f32", "dbeta")


@pytest.mark.parametrize("tau", [1.0, 0.5, 1e-3])
@pytest.mark.parametrize("V", [90, 40000])
def test_teacher_values_at_the_ends_of_the_range(V, tau):
    """p depends on the values' differences: all entries at the lowest value are alike, one of the largest is alone."""
    hd = _hd()
    rng = rng_for("teacher", V, tau)
    top = -LOWEST
    value = np.array([[LOWEST] * 4, [top] * 4, [top, LOWEST, 0, 1e37], [LOWEST, LOWEST, -np.inf, LOWEST], [3e36, 3e36, 1, 2],
                      [0, -1e30, -1e35, LOWEST]], np.float32)
    R, K = value.shape
    x = rounded(rng.standard_normal((R, V)), "f32")
    index = np.tile(np.array([0, 5, V - 2, 7], np.int32), (R, 1))
    grad = np.ones(R, np.float32)
    tau = float(np.float32(tau))
    r = hd.DistillRun.of(up(x, "f32"), up(index), up(value), None, up(grad), tau, 1.0)
    r.step()
    v = value.astype(np.float64)
    loss, d = ref.distill(x, index, v, None, grad.astype(np.float64), tau, 1.0)
    assert (loss != 0).all()
    close(r.loss, loss, "f32", "loss")
    close(r.dlogits, d, "f32", "dlogits")
