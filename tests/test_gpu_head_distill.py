"""Distillation loss on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT, close, get, rng_for, rounded, strided, up

pytestmark = pytest.mark.gpu


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


def _inputs(rng, R, V, K, dtype):
    x = rounded(2 * rng.standard_normal((R, V)), dtype)
    index = np.stack([rng.permutation(V)[:K] if K <= V else rng.integers(0, V, K) for _ in range(R)]).astype(np.int32)
    index[rng.random((R, K)) < 0.2] = -1
    index[rng.random((R, K)) < 0.05] = V                # past the end: not there
    if R > 3:
        index[1] = -1                                   # a row without a teacher
        index[2, : min(3, K)] = V - 1                   # an index several times
    value = (3 * rng.standard_normal((R, K))).astype(np.float32)
    label = rng.integers(-1, V + 1, R).astype(np.int32)
    if R > 4:
        label[1] = 0
        label[3] = index[3, 0]                          # an entry and the label at one place
    grad = np.where(rng.random(R) < 0.2, 0, rng.standard_normal(R)).astype(np.float32)
    return x, index, value, label, grad


# both sides of the lanes and vectors to a row, of rows that are cut, one token, ragged ends
SIZES = [(1, 1, 1), (5, 2, 3), (40, 16, 4), (33, 31, 31), (70, 33, 8), (100, 64, 64), (64, 83, 8), (20, 130, 70), (9, 257, 256),
         (30, 515, 16), (17, 1030, 33), (12, 4099, 64), (600, 4100, 5), (6, 8201, 64), (5, 16385, 17), (3, 32771, 64), (515, 16390, 3),
         (2, 65539, 32), (1, 131071, 64), (520, 33000, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,K", SIZES)
def test_loss_and_gradient(R, V, K, dtype):
    hd = _hd()
    rng = rng_for("distill", R, V, K, dtype)
    x, index, value, label, grad = _inputs(rng, R, V, K, dtype)
    tau, alpha = [(1.0, 0.5), (2.0, 0.3), (1.5, 1.0), (0.7, 0.0)][(R + V + K) % 4]
    tau, alpha = np.float32(tau), np.float32(alpha)
    r = hd.DistillRun.of(up(x, dtype), up(index), up(value), up(label), up(grad), float(tau), float(alpha))
    r.loss.fill_(7)
    r.step()
    few = np.arange(R) if R * V < 2e6 else np.unique(np.r_[0, 1, 2, 3, R - 1, rng.integers(0, R, 8)])
    few = few[few < R]
    loss, d = ref.distill(x[few], index[few], value[few].astype(np.float64), label[few], grad[few].astype(np.float64), float(tau), float(alpha))
    close(get(r.loss)[few], loss, "f32", "loss")
    close(get(r.dlogits)[few], d, dtype, "dlogits", extra=1e-6 * np.abs(grad[few]).max())
    assert not get(r.dlogits)[few][grad[few] == 0].any()
    step = r.dlogits.clone()
    r.dlogits.fill_(7)
    r.forward()
    close(get(r.loss)[few], loss, "f32", "loss of the forward")
    r.backward()
    close(get(r.dlogits)[few], d, dtype, "dlogits of the backward", extra=1e-6 * np.abs(grad[few]).max())
    # in place, and twice the same
    r2 = hd.DistillRun.of(r.logits, r.index, r.value, r.label, r.grad, float(tau), float(alpha))
    r2.dlogits = r2.logits = r.logits.clone()
    r2.step()
    assert torch.equal(r2.dlogits, step)
    r3 = hd.DistillRun.of(r.logits, r.index, r.value, r.label, r.grad, float(tau), float(alpha))
    r3.stats = r.stats
    r3.dlogits = r3.logits = r.logits.clone()
    r3.backward()
    assert torch.equal(r3.dlogits, r.dlogits)


@pytest.mark.parametrize("V", [90, 3000, 40000])
def test_masked_logits_and_rows(V):
    """Logits of -inf and of the type's lowest value, rows that are all masked, teacher values of -inf, NaN in rows that
    nobody looks at."""
    hd = _hd()
    rng = rng_for("masked", V)
    R, K = 8, 5
    x, index, value, label, grad = _inputs(rng, R, V, K, "f32")
    index[:] = np.arange(K) * 7
    label[:] = 3
    grad[:] = 1
    off = rng.random((R, V)) < 0.5
    off[:, list(range(0, 7 * K, 7)) + [3]] = False
    x[0][off[0]] = -np.inf
    x[1][off[1]] = np.finfo(np.float32).min
    x[2, 7] = -np.inf                                   # the teacher wants a masked token: an infinite loss
    value[3, 2] = -np.inf                               # probability 0, and its logit masked: nothing
    x[3, 14] = -np.inf
    value[4] = -np.inf                                  # no teacher
    x[5] = np.nan                                       # padding: no teacher, no label
    index[5], label[5] = -1, -1
    x[6, 11] = np.nan
    x[7] = -np.inf                                      # nothing left, yet asked for
    r = hd.DistillRun.of(up(x, "f32"), up(index), up(value), up(label), up(grad), 2.0, 0.5)
    r.step()
    loss, d = ref.distill(x, index, value.astype(np.float64), label, grad.astype(np.float64), 2.0, 0.5)
    got, gd = get(r.loss), get(r.dlogits)
    assert got[2] == np.inf and np.isnan(got[6]) and np.isnan(got[7])
    assert got[5] == 0 and not gd[5].any()
    close(got[:6], loss[:6], "f32", "loss")
    close(gd[:6], d[:6], "f32", "dlogits")
    assert np.isnan(gd[6]).all() and np.isnan(gd[7]).all()
    # without a weight the teacher's term is nothing, also where it would be infinite
    r0 = hd.DistillRun.of(r.logits, r.index, r.value, r.label, r.grad, 2.0, 0.0)
    assert np.isfinite(get(r0.step())[2])
    # the gradient of a row whose grad is 0 is 0, whatever it holds
    r.grad.zero_()
    r.step()
    assert not r.dlogits.any()
    r.forward()
    r.backward()
    assert not r.dlogits.any()


@pytest.mark.parametrize("R,V", [(50, 83), (4, 33000)])
def test_strides_no_label_no_grad(R, V):
    hd = _hd()
    rng = rng_for("dstride", R, V)
    for dtype in ("f32", "bf16"):
        x, index, value, _, _ = _inputs(rng, R, V, 6, dtype)
        X, D = strided(x, dtype, 5), strided(x, dtype, 1)
        r = hd.DistillRun.of(X, up(index), up(value), tau=2.0, dlogits=D)
        r.step()
        loss, d = ref.distill(x, index, value.astype(np.float64), None, np.ones(R), 2.0, 1.0)
        close(r.loss, loss, "f32", "loss")
        close(D, d, dtype, "dlogits", extra=1e-6)
        keep = torch.ones_like(D._base, dtype=torch.bool)
        keep[:, 1:1 + V] = False
        assert D._base[keep].isnan().all()


def test_differences():
    hd = _hd()
    rng = rng_for("ddiff")
    x, index, value, label, _ = _inputs(rng, 12, 50, 7, "f32")
    grad = rng.standard_normal(12).astype(np.float32)
    run = lambda v: hd.DistillRun.of(up(v, "f32"), up(index), up(value), up(label), up(grad), 2.0, 0.4)
    r = run(x)
    r.step()
    h, v = 2.0 ** -6, rng.standard_normal(x.shape)
    f = lambda p: (get(run(p).forward()) * grad).sum()
    num = (f(x + h * v) - f(x - h * v)) / (2 * h)
    size = np.abs(get(r.dlogits) * v).sum()
    # third derivatives: h^2 of a term's size; fp32's rounding of the losses over h
    assert abs(num - (get(r.dlogits) * v).sum()) <= 10 * h * h * size + 1e-6 / h * np.abs(get(r.loss) * grad).sum()


def test_empty_and_refusals():
    hd = _hd()
    r = hd.DistillRun.of(torch.empty(0, 9, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))
    r.step(), r.forward(), r.backward()
    mk = hd.make_distill_dims
    for bad in (mk(-1, 8, 2), mk(4, 0, 2), mk(4, 8, 0), mk(4, 8, 257), mk(4, 8, 2, 3), mk(4, 8, 2, tau=0.0), mk(4, 8, 2, tau=-1.0),
                mk(4, 8, 2, tau=float("nan")), mk(4, 8, 2, tau=float("inf")), mk(4, 8, 2, alpha=1.5), mk(4, 8, 2, alpha=-0.1),
                mk(4, 8, 2, alpha=float("nan")), mk(4, (1 << 22) + 1, 2), mk(4, 8, 2, ld_logits=7)):
        assert hd.stacklstm_distill_workspace_bytes(bad) == 0
    x = torch.randn(3, 40000, device="cuda")
    i, v = torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, 2, device="cuda")
    loss, st, d = torch.empty(3, device="cuda"), torch.empty(3, 3, device="cuda"), mk(3, 40000, 2)
    small = torch.empty(8, dtype=torch.uint8, device="cuda")
    assert hd.stacklstm_distill_fwd(d, x, i, v, None, loss, st, small, check=False) == 4
    assert hd.stacklstm_distill_fwd(d, x, i, v, None, loss, st, None, check=False) == 1
    for args in ((x, i.long(), v, None, loss, st), (x, i, v.double(), None, loss, st), (x, i[:, :1], v, None, loss, st),
                 (x, i, v, torch.zeros(2, dtype=torch.int32, device="cuda"), loss, st), (x, i, v, None, None, st)):
        with pytest.raises(ValueError):
            hd.stacklstm_distill_fwd(d, *args, small)
