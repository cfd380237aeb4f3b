"""Log probabilities, entropy and best tokens on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import close, get, rng_for, rounded, strided, up

pytestmark = pytest.mark.gpu


def _ly():
    need_gpu()
    from paper_1904_03409_amd import layers
    return layers


def _inputs(rng, R, V, G, dtype):
    x = rounded(2 * rng.standard_normal((R, V)), dtype)
    token = rng.integers(0, V, (R, G)).astype(np.int32)
    token[rng.random((R, G)) < 0.1] = -1
    token[rng.random((R, G)) < 0.05] = V                 # past the end: not there
    if G > 1 and R > 1:
        token[1, :2] = V - 1                             # a token twice
    legal = (rng.random((R, V)) < 0.7).astype(np.uint8) * 3
    legal[:, 0] = 1
    a, h = rng.standard_normal((R, G)).astype(np.float32), rng.standard_normal(R).astype(np.float32)
    if R > 3:
        a[2], h[2] = 0, 0
        h[3] = 0
    return x, token, legal, a, h


def _check(r, rows, want, dtype, a, h, grad=True):
    logp, ent, index, value, d = want
    close(get(r.logp)[rows], logp, "f32", "logp")
    # (a sum of terms of the size of log V)
    close(get(r.entropy)[rows], ent, "f32", "entropy", extra=1e-5)
    if r.index is not None:
        assert np.array_equal(get(r.index)[rows], index), "best tokens"
        close(get(r.value)[rows], value, "f32", "value")
    if grad:
        # what a row's weights can come to, times the bar for 32 bits
        big = (np.abs(a).sum(1) + np.abs(h) * 12)[:, None]
        close(get(r.dlogits)[rows], d, dtype, "dlogits", extra=1e-6 * big)


# both sides of the lanes and vectors to a row, of rows that are cut, one token, ragged ends
SIZES = [(1, 1, 1, 1), (5, 2, 3, 2), (40, 16, 2, 16), (33, 31, 20, 5), (70, 33, 1, 0), (100, 64, 1, 64), (64, 83, 2, 8), (20, 130, 64, 64), (9, 257, 3, 3),
         (30, 515, 2, 0), (17, 1030, 4, 33), (12, 4099, 1, 64), (600, 4100, 1, 5), (6, 8201, 3, 64), (5, 16385, 2, 17), (3, 32771, 1, 64),
         (515, 16390, 1, 0), (2, 65539, 64, 32), (1, 131071, 1, 64), (520, 33000, 1, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,G,N", SIZES)
def test_outputs_and_gradient(R, V, G, N, dtype):
    ly = _ly()
    rng = rng_for("logprob", R, V, G, N, dtype)
    x, token, legal, a, h = _inputs(rng, R, V, G, dtype)
    if (R + V) % 2:
        legal = None
    few = np.arange(R) if R * V < 2e6 else np.unique(np.r_[0, 1, 2, 3, R - 1, rng.integers(0, R, 8)])
    few = few[few < R]
    want = ref.logprob(x[few], token[few], None if legal is None else legal[few], N, a[few].astype(np.float64), h[few].astype(np.float64))
    r = ly.LogProbRun.of(up(x, dtype), up(token), None if legal is None else up(legal), N, up(a), up(h))
    r.step()
    _check(r, few, want, dtype, a[few], h[few])
    step = r.dlogits.clone()
    for t in (r.logp, r.entropy, r.dlogits):
        t.fill_(7)
    if N:
        r.index.fill_(7), r.value.fill_(7)
    r.workspace.fill_(255)
    r.forward()
    _check(r, few, want, dtype, a[few], h[few], grad=False)
    r.backward()
    _check(r, few, want, dtype, a[few], h[few])
    # in place, and twice the same
    for call in ("step", "backward"):
        z = ly.LogProbRun.of(r.logits.clone(), r.token, r.legal, N, r.dlogp, r.dentropy)
        z.dlogits, z.stats = z.logits, r.stats
        getattr(z, call)()
        assert torch.equal(z.dlogits, step if call == "step" else r.dlogits)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [90, 3000, 40000])
def test_masked_and_equal_logits(V, dtype):
    """Rows without allowed tokens, of -inf, of the type's lowest value, of equal logits, with NaN and +inf."""
    ly = _ly()
    rng = rng_for("equal", V, dtype)
    R, N = 10, 12
    x, token, legal, a, h = _inputs(rng, R, V, 2, dtype)
    low = float(torch.finfo({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).min)
    a[:], h[:] = 1, 0.5
    token[:] = [[5, 7]] * R
    legal[:] = 1
    legal[0] = 0                                         # nothing allowed
    x[1] = -np.inf                                       # nothing there
    x[2, rng.random(V) < 0.5] = -np.inf
    x[2, 5] = x[2, 7] = 1
    x[3, 8:] = low
    x[4] = 3                                             # all alike: the lowest tokens
    x[5] = rounded(rng.integers(0, 3, V), dtype)         # many alike
    x[6, 11] = np.nan
    x[7, 11] = np.inf
    legal[8] = 0
    legal[8, 20:25] = 1                                  # fewer than N; the given tokens are not allowed
    x[9] = low
    x[9, ::7] = 0
    want = ref.logprob(x, token, legal, N, a.astype(np.float64), h.astype(np.float64))
    r = ly.LogProbRun.of(up(x, dtype), up(token), up(legal), N, up(a), up(h))
    r.step()
    fine = [0, 2, 3, 4, 5, 8, 9]
    logp, ent, index, value, d = [get(t) for t in (r.logp, r.entropy, r.index, r.value, r.dlogits)]
    assert np.array_equal(index, want[2])
    assert (logp[[0, 1, 8]] == -np.inf).all() and (ent[[0, 1]] == 0).all()
    assert np.isnan(logp[6:8]).all() and np.isnan(ent[6:8]).all()
    assert (index[:2] == -1).all() and (value[:2] == -np.inf).all() and (index[8, 5:] == -1).all()
    assert not d[0].any() and not d[8][legal[8] == 0].any()
    for n, got, w in (("logp", logp, want[0]), ("entropy", ent, want[1]), ("value", value, want[3])):
        close(got[fine], w[fine], "f32", n, extra=1e-5)
    close(d[fine], want[4][fine], dtype, "dlogits", extra=1e-5)
    # without weights the gradient is 0, whatever the row holds
    r.dlogp.zero_(), r.dentropy.zero_()
    r.step()
    assert not r.dlogits.any()
    r.forward(), r.backward()
    assert not r.dlogits.any()


@pytest.mark.parametrize("V", [70, 9000, 70001])
def test_logits_far_from_zero(V):
    """A constant added to a row's logits changes nothing as long as they hold it: 2^20 in steps of 1/8, and 2^100."""
    ly = _ly()
    rng = rng_for("lfar", V)
    x = np.round(8 * 2 * rng.standard_normal((4, V))) / 8
    token, a, h = np.tile(np.arange(3, dtype=np.int32), (4, 1)), np.ones((4, 3), np.float32), np.ones(4, np.float32)
    want = ref.logprob(x, token, None, 5, a.astype(np.float64), h.astype(np.float64))
    for far in (2.0 ** 20, -2.0 ** 20):
        r = ly.LogProbRun.of(up(x + far, "f32"), up(token), None, 5, up(a), up(h))
        r.step()
        _check(r, np.arange(4), want, "f32", a, h)
    x = np.full((4, V), -2.0 ** 100)
    x[:, 1] = 2.0 ** 100
    r = ly.LogProbRun.of(up(x, "f32"), up(token), None, 2, up(a), up(h))
    r.step()
    assert (get(r.logp)[:, 1] == 0).all() and (get(r.entropy) == 0).all() and (get(r.index) == [[1, 0]] * 4).all()
    assert np.isfinite(get(r.dlogits)).all()


@pytest.mark.parametrize("R,V", [(50, 83), (4, 33000)])
def test_strides_and_parts(R, V):
    """Views of wider matrices; no given tokens; no weights of one kind; entropy alone."""
    ly = _ly()
    rng = rng_for("lstride", R, V)
    for dtype in ("f32", "bf16"):
        x, token, _, a, h = _inputs(rng, R, V, 2, dtype)
        X, D = strided(x, dtype, 5), strided(x, dtype, 1)
        r = ly.LogProbRun.of(X, up(token), top=4, dlogp=up(a), dlogits=D)
        r.step()
        want = ref.logprob(x, token, None, 4, a.astype(np.float64), None)
        _check(r, np.arange(R), want, dtype, a, 0 * h)
        keep = torch.ones_like(D._base, dtype=torch.bool)
        keep[:, 1:1 + V] = False
        assert D._base[keep].isnan().all()
        r = ly.LogProbRun.of(X, dentropy=up(h))
        r.step()
        want = ref.logprob(x, token[:, :0], None, 0, None, h.astype(np.float64))
        close(r.entropy, want[1], "f32", "entropy", extra=1e-5)
        close(r.dlogits, want[4], dtype, "dlogits", extra=1e-6 * np.abs(h)[:, None] * 12)
        d = ly.make_logprob_dims(R, V, 2, 0, r.dims.type, r.dims.ld_logits)
        logp = torch.empty(R, 2, device="cuda")
        ly.stacklstm_logprob_fwd(d, X, None, up(token), logp, None, None, None, None, r.workspace)
        close(logp, ref.logprob(x, token)[0], "f32", "logp")


def test_best_tokens_are_a_teacher():
    """index and value go to the distillation loss as they are: the loss of the student against its own best tokens is that
    of a softmax cut off behind them, and 0 where all tokens are kept."""
    ly = _ly()
    from paper_1904_03409_amd import head as hd
    rng = rng_for("teacher")
    x = up(2 * rng.standard_normal((30, 40)), "f32")
    r = ly.LogProbRun.of(x, top=40)
    r.forward()
    loss = hd.DistillRun.of(x, r.index, r.value).step()
    assert float(loss.abs().max()) < 1e-5


def test_differences():
    ly = _ly()
    rng = rng_for("ldiff")
    x, token, legal, a, h = _inputs(rng, 12, 50, 3, "f32")
    np.put_along_axis(legal, np.clip(token, 0, 49), 1, 1)
    run = lambda v: ly.LogProbRun.of(up(v, "f32"), up(token), up(legal), 0, up(a), up(h))
    r = run(x)
    r.step()
    s, v = 2.0 ** -6, rng.standard_normal(x.shape)

    def f(p):
        z = run(p)
        z.forward()
        return (get(z.logp) * a).sum() + (get(z.entropy) * h).sum()
    num, g = (f(x + s * v) - f(x - s * v)) / (2 * s), get(r.dlogits) * v
    # third derivatives: s^2 of a term's size; fp32's rounding of the outputs over s
    assert abs(num - g.sum()) <= 10 * s * s * np.abs(g).sum() + 1e-6 / s * (np.abs(get(r.logp) * a).sum() + np.abs(get(r.entropy) * h).sum())


def test_many_narrow_rows():
    """More rows than one launch has workgroups for."""
    ly = _ly()
    R, V = (1 << 26) + 70, 2
    x = torch.arange(R * V, device="cuda", dtype=torch.int32).remainder_(61).to(torch.bfloat16).view(R, V)
    token = torch.zeros(R, 1, dtype=torch.int32, device="cuda")
    d = ly.make_logprob_dims(R, V, 1, 0, 1)
    logp, ws = torch.full((R, 1), 7e9, device="cuda"), torch.empty(64, dtype=torch.uint8, device="cuda")
    ly.stacklstm_logprob_fwd(d, x, None, token, logp, None, None, None, None, ws)
    gap = (x[:, 1] - x[:, 0]).float()
    assert float((logp[:, 0] + torch.logaddexp(gap, torch.zeros_like(gap))).abs().max()) < 60 * 1e-5
    torch.cuda.empty_cache()


def test_refusals():
    ly = _ly()
    x, t = torch.randn(3, 40000, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    d = ly.make_logprob_dims(3, 40000, 2, 1)
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")
    logp, ent, index, value, small = e(3, 2), e(3), e(3, 1, dtype=torch.int32), e(3, 1), e(8, dtype=torch.uint8)
    assert ly.stacklstm_logprob_fwd(d, x, None, t, logp, ent, index, value, None, small, check=False) == 4
    assert ly.stacklstm_logprob_fwd(d, x, None, t, logp, ent, index, value, None, None, check=False) == 1
    for args in ((x, None, t.long(), logp, ent, index, value), (x, None, t[:, :1], logp, ent, index, value), (x, None, None, logp, ent, index, value),
                 (x, t, t, logp, ent, index, value), (x, None, t, None, ent, index, value), (x, None, t, logp, ent, index.long(), value),
                 (x, None, t, logp, ent, index, None), (x.half(), None, t, logp, ent, index, value)):
        with pytest.raises(ValueError):
            ly.stacklstm_logprob_fwd(d, *args, None, small)
