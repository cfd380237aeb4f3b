"""Views of wider matrices through every way that the operators read their operands (GPU, against 64 bits): rows whole 16 bytes
apart, at odd places, and dense matrices that begin off a 16-byte boundary."""
import numpy as np
import pytest
import torch

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DEV, DT, close, get, rng_for, rounded, up

pytestmark = pytest.mark.gpu
# first column and columns behind the last of a view; None: dense, one element into its memory
LAYOUTS = {"granules": (8, 8), "odd": (3, 2), "shifted": None}


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


def _view(a, dtype, layout):
    """a as a view with NaN around it, and a function that tells whether what is around it is as it was."""
    R, C = a.shape
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype])
    if LAYOUTS[layout] is None:
        big = torch.full((R * C + 9,), float("nan"), dtype=DT[dtype], device=DEV)
        v = big[1:1 + R * C].view(R, C)
        v.copy_(t)
        return v, lambda: bool(big[:1].isnan().all() and big[1 + R * C:].isnan().all())
    lo, hi = LAYOUTS[layout]
    big = torch.full((R, lo + C + hi), float("nan"), dtype=DT[dtype], device=DEV)
    v = big[:, lo:lo + C]
    v.copy_(t)
    return v, lambda: bool(big[:, :lo].isnan().all() and big[:, lo + C:].isnan().all())


# one launch for a backward and several, matrices copied and read as they are, tiles of 64 and more
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("M,K,N", [(1, 64, 72), (50, 72, 144), (50, 75, 141), (128, 200, 256), (100, 72, 640), (100, 131, 523), (200, 72, 144),
                                   (200, 75, 141), (700, 264, 520), (3000, 512, 768)])
def test_linear(M, K, N, layout, dtype):
    hd = _hd()
    rng = rng_for("layouts", M, K, N, layout, dtype)
    act = ["none", "tanh", "silu", "gelu"][(M + K) % 4]
    x, W, r0, dy = (rounded(rng.standard_normal(s), dtype) for s in ((M, K), (K, N), (M, N), (M, N)))
    W = rounded(W / np.sqrt(K), dtype)
    (X, _), (Wd, _), (R, _), (D, _), (Y, kept) = (_view(v, dtype, layout) for v in (x, W, r0, dy, r0))
    ld = lambda t: 0 if t.shape[0] < 2 or t.stride(0) == t.shape[1] else t.stride(0)
    d = hd.make_linear_dims(M, K, N, hd.TYPES[DT[dtype]], hd.ACTS[act], ld(X), ld(Wd), ld(R), ld(Y), ld(D))
    ws = torch.empty(max(hd.stacklstm_linear_fwd_workspace_bytes(d), hd.stacklstm_linear_bwd_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    z = torch.empty(M, N, dtype=DT[dtype], device=DEV)
    hd.stacklstm_linear_fwd(d, X, Wd, None, R, Y, z, ws)
    close(Y, ref.act(x @ W, act) + r0, dtype, "y")
    assert kept(), "written around y"
    dx, dW, db = (torch.full(s, 7.0, dtype=DT[dtype], device=DEV) for s in ((M, K), (K, N), (N,)))
    hd.stacklstm_linear_bwd(d, X, Wd, z if act != "none" else None, D, dx, dW, db, ws)
    dz = dy * ref.act_grad(get(z), act)
    # dz is rounded once for the products of 16-bit types
    e = 2.0 ** -8 if dtype == "bf16" else 1e-6
    close(dx, dz @ W.T, dtype, "dx", extra=e * (np.abs(dz) @ np.abs(W).T))
    close(dW, x.T @ dz, dtype, "dW", extra=e * (np.abs(x).T @ np.abs(dz)))
    close(db, dz.sum(0), dtype, "db", extra=1e-6 * np.abs(dz).sum(0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("rows,width", [(5, 16), (300, 40), (300, 77), (40, 512), (40, 1030), (600, 1024), (9, 8192)])
def test_norm(rows, width, layout, dtype):
    hd = _hd()
    rng = rng_for("norm layouts", rows, width, layout, dtype)
    x, res, dy = (rounded(rng.standard_normal((rows, width)), dtype) for _ in range(3))
    (X, _), (R, _), (D, _) = (_view(v, dtype, layout) for v in (x, res, dy))
    gamma, beta = 1 + 0.1 * rng.standard_normal(width), 0.1 * rng.standard_normal(width)
    f32 = lambda v: v.astype(np.float32).astype(np.float64)
    gamma, beta = f32(gamma), f32(beta)
    for with_res in (True, False):
        r = hd.NormRun.of(X, up(gamma, "f32"), up(beta, "f32"), res=R if with_res else None, dy=D)
        r.forward()
        s, y, mu, rstd = ref.norm_fwd(x, res if with_res else None, gamma, beta, 1e-5)
        close(r.y, y, dtype, "y")
        s = get(r.sum) if with_res else x
        r.backward()
        dx, dg, db = ref.norm_bwd(s, get(r.mean), get(r.rstd), gamma, dy, None)
        close(r.dx, dx, dtype, "dx", extra=1e-6 * 8 * np.abs(dy).max())
        close(r.dgamma, dg, "f32", "dgamma")
        close(r.dbeta, db, "f32", "dbeta")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("V", [64, 83, 4096, 40000, 65539])
def test_distill_and_beam(V, layout, dtype):
    """The bits of dense, aligned logits."""
    hd = _hd()
    rng = rng_for("softmax layouts", V, layout, dtype)
    R, K = 6, 5
    x = rounded(2 * rng.standard_normal((R, V)), dtype)
    index, value = up(rng.integers(0, V, (R, K)).astype(np.int32)), up(rng.standard_normal((R, K)).astype(np.float32))
    label, score = up(rng.integers(0, V, R).astype(np.int32)), up(-rng.random((2, 3)).astype(np.float32))
    dense = up(x, dtype)
    (X, _), (D, kept) = _view(x, dtype, layout), _view(x, dtype, layout)
    a = hd.DistillRun.of(dense, index, value, label, tau=2.0, alpha=0.5)
    b = hd.DistillRun.of(X, index, value, label, tau=2.0, alpha=0.5, dlogits=D)
    for run in (lambda r: r.step(), lambda r: (r.forward(), r.backward())):
        run(a), run(b)
        assert torch.equal(a.loss, b.loss) and torch.equal(a.dlogits, D) and kept()
    p, q = hd.BeamRun.of(dense, score), hd.BeamRun.of(X, score)
    p.select(), q.select()
    assert all(torch.equal(getattr(p, n), getattr(q, n)) for n in ("score_next", "parent", "token", "done_next"))
