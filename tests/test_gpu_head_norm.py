"""Layer norm on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT, close, get, rng_for, rounded, strided, up

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


# both sides of every number of lanes and vectors to a row, odd widths, one element, the widest
WIDTHS = [1, 2, 7, 31, 32, 33, 64, 65, 128, 130, 200, 256, 257, 512, 515, 1000, 1024, 1030, 2048, 2049, 4096, 4100, 8191, 8192]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_forward_and_backward(width, dtype):
    hd = _hd()
    rng = rng_for("norm", width, dtype)
    rows = 1 + width % 7 + (300 if width <= 256 else 5)
    res = width % 2 == 0
    a = {k: rounded(rng.standard_normal((rows, width)), dtype) for k in ("x", "res", "dy", "dsum")}
    a["x"] += rounded(rng.standard_normal((rows, 1)), dtype)
    a["x"] = rounded(a["x"], dtype)
    f32 = lambda v: v.astype(np.float32).astype(np.float64)
    gamma, beta = f32(1 + 0.1 * rng.standard_normal(width)), f32(0.1 * rng.standard_normal(width))
    r = hd.NormRun.of(up(a["x"], dtype), up(gamma, "f32"), up(beta, "f32"), res=up(a["res"], dtype) if res else None,
                      dy=up(a["dy"], dtype), dsum=up(a["dsum"], dtype) if res else None, eps=EPS)
    r.forward()
    s, y, mu, rstd = ref.norm_fwd(a["x"], a["res"] if res else None, gamma, beta, EPS)
    # a row of one or two elements has a variance that can be tiny: its rounding is as large as 2^-24 of the mean
    slack = 2.0 ** -22 * (np.abs(s).max(1) + 1) * rstd
    close(r.y, y, dtype, "y", extra=(slack * np.abs(gamma).max() * 4)[:, None])
    close(r.mean, mu, "f32", "mean")
    close(r.rstd, rstd, "f32", "rstd", extra=4 * slack * rstd)
    if res:
        close(r.sum, s, dtype, "sum")
        s = get(r.sum)
    # the backward is a function of what it is given
    mu, rstd = get(r.mean), get(r.rstd)
    r.backward()
    dx, dg, db = ref.norm_bwd(s, mu, rstd, gamma, a["dy"], a["dsum"] if res else None)
    close(r.dx, dx, dtype, "dx", extra=1e-6 * (rstd * np.abs(a["dy"]).max() * 8 * (1 + slack))[:, None])
    close(r.dgamma, dg, "f32", "dgamma")
    close(r.dbeta, db, "f32", "dbeta")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_sum_in_32_bits(dtype):
    hd = _hd()
    rng = rng_for("rows", dtype)
    rows, width = 30011, 96
    x, dy = (rounded(rng.standard_normal((rows, width)) + 0.25, dtype) for _ in range(2))
    r = hd.NormRun.of(up(x, dtype), up(np.ones(width), "f32"), up(np.zeros(width), "f32"), dy=up(dy, dtype))
    r.forward()
    r.backward()
    s, _, mu, rstd = ref.norm_fwd(x, None, None, None, EPS)
    _, dg, db = ref.norm_bwd(s, mu, rstd, None, dy, None)
    close(r.dgamma, dg, "f32", "dgamma")
    close(r.dbeta, db, "f32", "dbeta")
    first = [t.clone() for t in (r.dx, r.dgamma, r.dbeta)]
    r.backward()
    assert all(torch.equal(p, q) for p, q in zip(first, (r.dx, r.dgamma, r.dbeta))), "equal calls differ"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_optional_arguments(dtype):
    hd = _hd()
    rng = rng_for("strides", dtype)
    rows, width = 37, 75
    x, res, dy = (rounded(rng.standard_normal((rows, width)), dtype) for _ in range(3))
    d = hd.make_norm_dims(rows, width, hd.SLSTM_F32 if dtype == "f32" else hd.SLSTM_BF16, EPS, width + 8, width + 4, width + 6)
    y = torch.empty(rows, width, dtype=DT[dtype], device="cuda")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    hd.stacklstm_norm_fwd(d, strided(x, dtype, 5), strided(res, dtype, 1), None, None, None, y, mean, rstd)
    _, want, mu, rs = ref.norm_fwd(x, res, None, None, EPS)
    close(y, want, dtype, "y")
    # without the weights' gradients no work space is asked for
    dx = torch.empty_like(y)
    hd.stacklstm_norm_bwd(d, strided(x, dtype, 5), None, mean, rstd, strided(dy, dtype, 3), None, dx, None, None, None)
    close(dx, ref.norm_bwd(x, get(mean), get(rstd), None, dy, None)[0], dtype, "dx")
    # y alone
    hd.stacklstm_norm_fwd(d, strided(x, dtype, 5), None, None, None, None, y, None, None)
    close(y, ref.norm_fwd(x, None, None, None, EPS)[1], dtype, "y without res")


def test_constant_rows_large_means_and_nonfinite_values():
    hd = _hd()
    x = np.zeros((6, 40))
    x[0] = 3.0                                          # no variance: y = beta
    x[1] = 1e4 + np.arange(40) % 2                      # a mean far larger than the deviation
    x[2, 7] = np.nan
    x[3, 9] = np.inf
    x[4] = 1e19 * (np.arange(40) % 3 - 1)               # squares past fp32's range: rstd 0
    x[5] = np.arange(40)
    r = hd.NormRun.of(up(x, "f32"), up(np.full(40, 2.0), "f32"), up(np.full(40, 0.5), "f32"), dy=up(np.ones((6, 40)), "f32"))
    y = get(r.forward())
    assert np.array_equal(y[0], np.full(40, 0.5))
    want = ref.norm_fwd(x, None, np.full(40, 2.0), np.full(40, 0.5), EPS)[1]
    # the deviations are exact in 32 bits here, the mean is off by a rounding of 1e4
    assert np.abs(y[1] - want[1]).max() < 2 * 2 * 1e4 * 2.0 ** -23
    assert np.isnan(y[2]).all() and np.isnan(y[3]).all() and np.array_equal(y[4], np.full(40, 0.5))
    assert np.abs(y[5] - want[5]).max() < 1e-5 * 4
    r.backward()
    dx = get(r.dx)
    assert np.isnan(dx[2]).all() and np.isnan(dx[3]).all() and np.isfinite(dx[[0, 1, 4, 5]]).all()


def test_empty_and_refusals():
    hd = _hd()
    e = torch.empty(0, 8, device="cuda")
    r = hd.NormRun.of(e, up(np.ones(8), "f32"), up(np.ones(8), "f32"), dy=e)
    r.dgamma.fill_(7)
    r.dbeta.fill_(7)
    r.forward()
    r.backward()
    assert not r.dgamma.any() and not r.dbeta.any()
    x, y = torch.randn(4, 8, device="cuda"), torch.empty(4, 8, device="cuda")
    d = hd.make_norm_dims(4, 8)

    def code(dims, *a, fn=hd.stacklstm_norm_fwd):
        return fn(dims, *a, check=False)
    assert code(d, x, None, None, None, None, y, None, None) == 0
    assert code(hd.make_norm_dims(4, 8, eps=-1.0), x, None, None, None, None, y, None, None) == 1
    assert code(hd.make_norm_dims(4, 8, eps=float("nan")), x, None, None, None, None, y, None, None) == 1
    assert code(d, x, None, None, None, y, y, None, None) == 1                 # a sum without a residual
    for bad in (hd.make_norm_dims(-1, 8), hd.make_norm_dims(4, 0), hd.make_norm_dims(4, 8193), hd.make_norm_dims(4, 8, 2),
                hd.make_norm_dims(4, 8, ld_x=7)):
        assert hd.stacklstm_norm_workspace_bytes(bad) == 0
    g, st = torch.empty(8, device="cuda"), torch.empty(4, device="cuda")
    big = hd.make_norm_dims(4096, 512)
    X = torch.randn(4096, 512, device="cuda")
    S, G, D = torch.ones(4096, device="cuda"), torch.empty(512, device="cuda"), torch.empty(4096, 512, device="cuda")
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    assert hd.stacklstm_norm_bwd(big, X, None, S, S, X, None, D, G, None, small, check=False) == 4
    assert hd.stacklstm_norm_bwd(big, X, None, S, S, X, None, D, G, None, None, check=False) == 1
    with pytest.raises(hd.StackLSTMError):
        hd.stacklstm_norm_bwd(big, X, None, S, S, X, None, D, G, None, small)
    for args in ((x.half(), None, None, None, None, y, None, None), (x.t(), None, None, None, None, y, None, None),
                 (x, None, g.double(), None, None, y, None, None), (x, None, None, None, None, y[:3], None, None),
                 (x, None, None, None, None, None, None, None), (x, None, None, None, None, y, st[:2], None),
                 (x.cpu(), None, None, None, None, y, None, None)):
        with pytest.raises(ValueError):
            hd.stacklstm_norm_fwd(d, *args)
    with pytest.raises(ValueError):
        hd.NormRun.of(x.double())


def test_another_stream():
    hd = _hd()
    x = torch.randn(5000, 300, device="cuda")
    a = hd.NormRun.of(x, train=False)
    a.forward()
    s = torch.cuda.Stream()
    b = hd.NormRun.of(x, train=False)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.forward()
    c = hd.NormRun.of(x, train=False)
    c.forward(stream=s)
    s.synchronize()
    assert torch.equal(a.y, b.y) and torch.equal(a.y, c.y)
