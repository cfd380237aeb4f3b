"""The linear layer's 16-bit backward with dz in two planes (GPU, against 64 bits)."""
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


def _want(x, W, z, dy, act):
    g = ref.act_grad(z, act)
    dz = dy * g
    # 2^-18 of dz is left of it (two roundings to 8 bits), act' is within 2e-6, sums are 32-bit
    ex = (2.0 ** -17 * np.abs(dz) + 2e-6 * np.abs(dy)) @ np.abs(W).T + 1e-6 * (np.abs(dz) @ np.abs(W).T)
    ew = np.abs(x).T @ (2.0 ** -17 * np.abs(dz) + 2e-6 * np.abs(dy)) + 1e-6 * (np.abs(x).T @ np.abs(dz))
    return dz, (dz @ W.T, ex), (x.T @ dz, ew)


@pytest.mark.parametrize("act", ["relu", "tanh", "silu", "gelu"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 72), (50, 75, 141), (128, 200, 256), (100, 72, 640), (200, 72, 144), (200, 75, 141), (700, 264, 520),
                                   (3000, 512, 768), (9000, 48, 100)])
def test_two_planes(M, K, N, act):
    hd = _hd()
    rng = rng_for("wide", M, K, N, act)
    x, dy = (rounded(rng.standard_normal(s), "bf16") for s in ((M, K), (M, N)))
    W, b = rounded(rng.standard_normal((K, N)) / np.sqrt(K), "bf16"), rounded(rng.standard_normal(N), "bf16")
    args = [up(v, "bf16") for v in (x, W, b)]
    r = hd.LinearRun.of(*args, act=act, dy=up(dy, "bf16"), wide_dz=True)
    one = hd.LinearRun.of(*args, act=act, dy=up(dy, "bf16"))
    assert torch.equal(r.forward(), one.forward()) and torch.equal(r.z, one.z)
    r.backward()
    one.backward()
    dz, (dx, ex), (dW, ew) = _want(x, W, get(r.z), dy, act)
    close(r.dx, dx, "bf16", "dx", extra=ex)
    close(r.dW, dW, "bf16", "dW", extra=ew)
    assert torch.equal(r.db, one.db)
    # what is left is the outputs' own rounding; with one plane it is a good deal more, where sums have terms to show it
    err = lambda t, w: np.linalg.norm((get(t) if isinstance(t, torch.Tensor) else t) - w)
    for got, other, want in ((r.dx, one.dx, dx), (r.dW, one.dW, dW)):
        if want.size > 1000:
            assert err(got, want) <= 1.05 * err(rounded(want, "bf16"), want)
            assert act == "relu" or M < 2 or err(other, want) >= 1.15 * err(got, want)
    # each alone, and again, the same bits
    first = [t.clone() for t in (r.dx, r.dW)]
    for k in range(2):
        out = [torch.full_like(t, 7.0) if i == k else None for i, t in enumerate(first)]
        hd.stacklstm_linear_bwd(r.dims, r.x, r.W, r.z, r.dy, *out, None, r.workspace)
        assert torch.equal(out[k], first[k])


def test_strides_infinities_and_types():
    hd = _hd()
    rng = rng_for("wide strides")
    M, K, N = 300, 72, 144
    x, W, dy = (rounded(rng.standard_normal(s), "bf16") for s in ((M, K), (K, N), (M, N)))
    for pad in (3, 8):
        X, Wd, D = strided(x, "bf16", pad), strided(W, "bf16", pad), strided(dy, "bf16", pad)
        r = hd.LinearRun.of(X, Wd, act="tanh", dy=D, wide_dz=True)
        r.forward(), r.backward()
        dz, (dx, ex), (dW, ew) = _want(x, W, get(r.z), dy, "tanh")
        close(r.dx, dx, "bf16", "dx", extra=ex)
        close(r.dW, dW, "bf16", "dW", extra=ew)
    # an infinite gradient stays one, and in its row
    dy[5, 7], dy[9, 3] = np.inf, np.nan
    Wp = np.abs(W) + 0.1
    r = hd.LinearRun.of(up(x, "bf16"), up(Wp, "bf16"), act="relu", dy=up(dy, "bf16"), wide_dz=True)
    r.forward()
    r.z.fill_(1.0)
    r.backward()
    dx = get(r.dx)
    assert (dx[5] == np.inf).all() and np.isnan(dx[9]).all()
    other = np.ones(M, bool)
    other[[5, 9]] = False
    assert np.isfinite(dx[other]).all()
    # 32 bits, and no activation: the same bits with it and without
    for dtype, act in (("f32", "gelu"), ("bf16", "none")):
        runs = [hd.LinearRun.of(up(x, dtype), up(W, dtype), act=act, dy=up(dy, dtype), wide_dz=w) for w in (False, True)]
        for r in runs:
            r.forward(), r.backward()
        assert torch.equal(runs[0].dx.nan_to_num(), runs[1].dx.nan_to_num()) and torch.equal(runs[0].dW.nan_to_num(), runs[1].dW.nan_to_num())
    e = hd.LinearRun.of(torch.empty(0, K, dtype=torch.bfloat16, device="cuda"), up(W, "bf16"), act="silu", train=True, wide_dz=True)
    e.dy = torch.empty(0, N, dtype=torch.bfloat16, device="cuda")
    e.forward(), e.backward()
    assert not e.dW.any()


def test_refusals():
    hd = _hd()
    for act in (-1, 5, 0x105, 0x200, 0x1ff, -0x100):
        assert hd.stacklstm_linear_bwd_workspace_bytes(hd.make_linear_dims(4, 4, 4, hd.SLSTM_BF16, act)) == 0
    plain, wide = (hd.make_linear_dims(1000, 64, 64, hd.SLSTM_BF16, a) for a in (2, 0x102))
    assert hd.stacklstm_linear_fwd_workspace_bytes(plain) == hd.stacklstm_linear_fwd_workspace_bytes(wide)
    n = hd.stacklstm_linear_bwd_workspace_bytes(plain)
    assert hd.stacklstm_linear_bwd_workspace_bytes(wide) > n
    t = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    small = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert hd.stacklstm_linear_bwd(wide, t(1000, 64), t(64, 64), t(1000, 64), t(1000, 64), t(1000, 64), None, None, small, check=False) == 4
