"""Linear layer on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT, TOL32, close, get, rng_for, rounded, strided, up

pytestmark = pytest.mark.gpu


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


# single rows, odd and ragged sizes, whole tiles and one more, sums split and not
SIZES = [(1, 1, 1), (1, 512, 83), (3, 7, 5), (8, 64, 64), (17, 33, 65), (64, 1024, 200), (64, 72, 2000), (65, 128, 64),
         (127, 96, 136), (128, 128, 128), (130, 250, 129), (257, 264, 272), (300, 40, 1000), (2000, 24, 16), (5000, 136, 72),
         (1024, 768, 1032), (4096, 320, 264), (1, 3000, 8), (2, 16, 4104)]
ACTS = ["none", "relu", "tanh", "silu", "gelu"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward_and_backward(M, K, N, dtype):
    hd = _hd()
    rng = rng_for("linear", M, K, N, dtype)
    act = ACTS[(M + K + N) % 5]
    res = (M + N) % 2 == 0
    x, dy, r0 = (rounded(rng.standard_normal(s), dtype) for s in ((M, K), (M, N), (M, N)))
    W, b = rounded(rng.standard_normal((K, N)) / np.sqrt(K), dtype), rounded(rng.standard_normal(N), dtype)
    r = hd.LinearRun.of(up(x, dtype), up(W, dtype), up(b, dtype), res=up(r0, dtype) if res else None, act=act, dy=up(dy, dtype))
    r.forward()
    z = x @ W + b
    y = ref.act(z, act) + (r0 if res else 0)
    close(r.y, y, dtype, "y")
    if act != "none":
        close(r.z, z, dtype, "z")
        z = get(r.z)
    r.backward()
    dz = dy * ref.act_grad(z, act)
    # 16 bits: dz is rounded for the products
    e = (lambda p: 2.0 ** -8 * p) if dtype == "bf16" and act != "none" else (lambda p: 0.0)
    # (32-bit sums over many terms of both signs: the bar is on the sum of their sizes)
    s = lambda p: TOL32 * p.max()
    dzx, dzw = np.abs(dz) @ np.abs(W).T, np.abs(x).T @ np.abs(dz)
    close(r.dx, dz @ W.T, dtype, "dx", extra=e(dzx) + 0.1 * s(dzx))
    close(r.dW, x.T @ dz, dtype, "dW", extra=e(dzw) + 0.1 * s(dzw))
    close(r.db, dz.sum(0), dtype, "db")


# a backward of few rows in one launch, up to its ends and past them; dx and dW in one launch, sums of dW split and not; db in
# strips narrow and wide, of several blocks of rows; rows that end in every place of a vector, or have less than one
LAUNCHES = [(128, 512, 256), (128, 512, 260), (128, 300, 257), (100, 300, 300), (128, 70, 3), (5, 1, 513), (77, 65, 7), (33, 301, 302),
            (129, 85, 46), (200, 512, 512), (660, 413, 23), (700, 333, 5), (1000, 500, 333), (2048, 200, 31), (2049, 96, 516),
            (2100, 300, 1100), (6000, 176, 416), (9000, 9, 11)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", LAUNCHES)
def test_launches(M, K, N, dtype):
    test_forward_and_backward(M, K, N, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [3, 8])
def test_strides(dtype, pad):
    """Views of wider matrices, at aligned and odd places; what lies between the rows is NaN and stays."""
    hd = _hd()
    rng = rng_for("strides", dtype, pad)
    M, K, N = 200, 72, 144
    t = hd.SLSTM_F32 if dtype == "f32" else hd.SLSTM_BF16
    x, W, r0, dy = (rounded(rng.standard_normal(s), dtype) for s in ((M, K), (K, N), (M, N), (M, N)))
    W = rounded(W / 8, dtype)
    X, Wd, R, D, Y = (strided(v, dtype, pad) for v in (x, W, r0, dy, r0))
    d = hd.make_linear_dims(M, K, N, t, hd.ACTS["silu"], X.stride(0), Wd.stride(0), R.stride(0), Y.stride(0), D.stride(0))
    n = max(hd.stacklstm_linear_fwd_workspace_bytes(d), hd.stacklstm_linear_bwd_workspace_bytes(d))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    z = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    hd.stacklstm_linear_fwd(d, X, Wd, None, R, Y, z, ws)
    close(Y, ref.act(x @ W, "silu") + r0, dtype, "y")
    base = Y._base
    keep = torch.ones_like(base, dtype=torch.bool)
    keep[:, pad:pad + N] = False
    assert base[keep].isnan().all(), "written between the rows"
    # y in place of the residual
    hd.stacklstm_linear_fwd(hd.make_linear_dims(M, K, N, t, hd.ACTS["silu"], X.stride(0), Wd.stride(0), Y.stride(0), Y.stride(0)),
                            X, Wd, None, Y, Y, None, ws)
    y1 = rounded(ref.act(x @ W, "silu") + r0, dtype)
    close(Y, ref.act(x @ W, "silu") + y1, dtype, "y over res", extra=2.0 ** -7 * np.abs(y1) if dtype == "bf16" else 1e-6)
    dx, dW = torch.empty(M, K, dtype=DT[dtype], device="cuda"), torch.empty(K, N, dtype=DT[dtype], device="cuda")
    hd.stacklstm_linear_bwd(d, X, Wd, z, D, dx, dW, None, ws)
    dz = dy * ref.act_grad(get(z), "silu")
    e = 2.0 ** -8 if dtype == "bf16" else 1e-6
    close(dx, dz @ W.T, dtype, "dx", extra=e * (np.abs(dz) @ np.abs(W).T))
    close(dW, x.T @ dz, dtype, "dW", extra=e * (np.abs(x).T @ np.abs(dz)))
    # each gradient alone gives the same bits
    for k in range(3):
        out = [torch.empty_like(dx), torch.empty_like(dW), torch.empty(N, dtype=DT[dtype], device="cuda")]
        hd.stacklstm_linear_bwd(d, X, Wd, z, D, *[o if i == k else None for i, o in enumerate(out)], ws)
        if k < 2:
            assert torch.equal(out[k], (dx, dW)[k])
        else:
            close(out[2], dz.sum(0), dtype, "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_at_their_ends(act, dtype):
    """z from -40 to 40 and infinite through a weight of one: values and derivatives, at 0 too."""
    hd = _hd()
    zs = np.concatenate([np.linspace(-40, 40, 161), [-1e30, 1e30, 0.0, 1e-30]])
    zs = rounded(zs, dtype)
    M = len(zs)
    x, W, dy = zs[:, None], np.ones((1, 8)), np.ones((M, 8))
    r = hd.LinearRun.of(up(x, dtype), up(W, dtype), act=act, dy=up(dy, dtype))
    r.forward()
    with np.errstate(all="ignore"):
        want = np.nan_to_num(ref.act(np.repeat(x, 8, 1), act), nan=0.0)
        g = np.repeat(ref.act_grad(np.clip(x, -50, 50), act), 8, 1)
    big = np.abs(x[:, 0]) > 1e20
    y = get(r.y)
    assert np.abs(y[~big] - want[~big]).max() <= 40 * (TOL32 + (2.0 ** -8 if dtype == "bf16" else 0))
    assert np.array_equal(np.sign(np.round(y[big], 3)), np.sign(np.round(want[big], 3)))
    r.backward()
    dx = get(r.dx)[:, 0]
    ok = ~big
    assert np.abs(dx[ok] - g[ok].sum(1)).max() <= 8 * 1.2 * (TOL32 + (2.0 ** -7 if dtype == "bf16" else 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nonfinite_inputs_stay_in_their_rows(dtype):
    hd = _hd()
    rng = rng_for("nonfinite", dtype)
    x = rounded(rng.standard_normal((140, 96)), dtype)
    x[3, 5], x[70, 9] = np.nan, np.inf
    W = rounded(np.abs(rng.standard_normal((96, 80))) + 0.1, dtype)
    y = get(hd.LinearRun.of(up(x, dtype), up(W, dtype)).forward())
    assert np.isnan(y[3]).all() and (y[70] == np.inf).all()
    other = np.ones(140, bool)
    other[[3, 70]] = False
    assert np.isfinite(y[other]).all()


def test_differences():
    """The gradients against differences of the forward itself, in directions."""
    hd = _hd()
    rng = rng_for("differences")
    M, K, N = 20, 30, 25
    x, W, b, dy = (rng.standard_normal(s) for s in ((M, K), (K, N), (N,), (M, N)))
    W /= 6
    up64 = lambda v: up(v, "f32")
    r = hd.LinearRun.of(up64(x), up64(W), up64(b), act="gelu", dy=up64(dy))
    r.forward()
    r.backward()
    loss = lambda x, W, b: (get(hd.LinearRun.of(up64(x), up64(W), up64(b), act="gelu").forward()) * dy).sum()
    h = 2.0 ** -8
    for k, (v, g) in enumerate(((x, r.dx), (W, r.dW), (b, r.db))):
        d = rng.standard_normal(v.shape)
        args = [[x, W, b], [x, W, b]]
        args[0][k], args[1][k] = v + h * d, v - h * d
        num = (loss(*args[0]) - loss(*args[1])) / (2 * h)
        size = np.abs(get(g) * d).sum()
        # third derivatives: h^2 of a term's size; fp32's rounding of the loss's terms over h
        assert abs(num - (get(g) * d).sum()) <= (10 * h * h + 1e-6 / h) * size


def test_empty_and_refusals():
    hd = _hd()
    x0, dy0 = torch.empty(0, 16, device="cuda"), torch.empty(0, 8, device="cuda")
    W, b = torch.randn(16, 8, device="cuda"), torch.randn(8, device="cuda")
    for act in ("none", "gelu"):
        r = hd.LinearRun.of(x0, W, b, act=act, dy=dy0)
        r.dW.fill_(3)
        r.db.fill_(3)
        r.forward()
        r.backward()
        assert not r.dW.any() and not r.db.any()
    for bad in (hd.make_linear_dims(-1, 4, 4), hd.make_linear_dims(4, 0, 4), hd.make_linear_dims(4, 4, 0), hd.make_linear_dims(4, 4, 4, 2),
                hd.make_linear_dims(4, 4, 4, 0, 5), hd.make_linear_dims(4, 4, 4, 0, 0, 3), hd.make_linear_dims(4, 1 << 25, 4),
                hd.make_linear_dims((1 << 30) + 1, 4, 4)):
        assert hd.stacklstm_linear_fwd_workspace_bytes(bad) == 0 and hd.stacklstm_linear_bwd_workspace_bytes(bad) == 0
    x, y = torch.randn(64, 1024, device="cuda"), torch.empty(64, 64, device="cuda")
    W = torch.randn(1024, 64, device="cuda")
    d = hd.make_linear_dims(64, 1024, 64, 0, hd.ACTS["tanh"])
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    assert hd.stacklstm_linear_fwd_workspace_bytes(d) > 64
    assert hd.stacklstm_linear_fwd(d, x, W, None, None, y, None, small, check=False) == 4
    assert hd.stacklstm_linear_fwd(d, x, W, None, None, y, None, None, check=False) == 1
    ws = torch.empty(hd.stacklstm_linear_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)
    assert hd.stacklstm_linear_bwd(d, x, W, None, y, dx, None, None, ws, check=False) == 1        # no z
    assert hd.stacklstm_linear_bwd(d, x, W, y, y, dx, None, None, small, check=False) == 4
    for args in ((x, W.t().contiguous(), None, None, y, None), (x, W.bfloat16(), None, None, y, None),
                 (x, W, torch.randn(63, device="cuda"), None, y, None), (x[:, ::2], W, None, None, y, None)):
        with pytest.raises(ValueError):
            hd.stacklstm_linear_fwd(d, *args, ws)
