"""Dropout on the GPU against the generator's definition."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import get, rng_for, rounded, strided, up

pytestmark = pytest.mark.gpu
KEY, STEP = 0x1234567890ABCDE, (3 << 32) + 77


def _ly():
    need_gpu()
    from paper_1904_03409_amd import layers
    return layers


def _seed(key=KEY, step=STEP):
    return torch.tensor([key, step], dtype=torch.int64, device="cuda")


def _within(got, want, terms, dtype, what):
    """A factor, a product and a sum in 32 bits (each half a step of what it comes to), and the output's rounding."""
    err = np.abs(get(got) - want)
    off = 3 * 2.0 ** -24 * terms + ref.HALF[dtype] * np.abs(want)
    assert (err <= off).all(), f"{what}: {(err - off).max()}"


SIZES = [(1, 1), (3, 7), (5, 8), (4, 9), (17, 16), (33, 100), (2, 2051), (300, 1), (70, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,W", SIZES)
def test_forward_and_backward(R, W, dtype):
    ly = _ly()
    rng = rng_for("dropout", R, W, dtype)
    p, period = [(0.1, 0), (0.5, 0), (0.3, 4), (0.9, 1)][(R + W) % 4]
    x, res, dy = (rounded(rng.standard_normal((R, W)), dtype) for _ in range(3))
    keep, scale = ref.keep(R, W, p, KEY, STEP, period)
    r = ly.DropoutRun.of(up(x, dtype), p, _seed(), up(res, dtype), period, up(dy, dtype))
    r.y.fill_(7), r.dx.fill_(7)
    r.forward(), r.backward()
    want = np.where(keep, x * scale, 0)
    _within(r.y, want + res, np.abs(want) + np.abs(want + res), dtype, "y")
    want = np.where(keep, dy * scale, 0)
    _within(r.dx, want, np.abs(want), dtype, "dx")
    assert np.array_equal(get(r.dx) != 0, keep & (dy != 0))
    # without a residual; in place of x, of the residual and of dy
    plain = ly.DropoutRun.of(up(x, dtype), p, _seed(), period=period)
    plain.forward()
    want = np.where(keep, x * scale, 0)
    _within(plain.y, want, np.abs(want), dtype, "y")
    for n in ("x", "res"):
        z = ly.DropoutRun.of(up(x, dtype), p, _seed(), up(res, dtype), period)
        z.y = getattr(z, n)
        z.forward()
        assert torch.equal(z.y, r.y)
    g = up(dy, dtype)
    ly.stacklstm_dropout_bwd(r.bwd_dims, g, _seed(), g)
    assert torch.equal(g, r.dx)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    ly = _ly()
    rng = rng_for("dstrides", dtype)
    R, W = 21, 45
    x, res, dy = (rounded(rng.standard_normal((R, W)), dtype) for _ in range(3))
    keep, scale = ref.keep(R, W, 0.4, KEY, STEP)
    Y = strided(x, dtype, 2)
    r = ly.DropoutRun.of(strided(x, dtype, 5), 0.4, _seed(), strided(res, dtype, 1), dy=strided(dy, dtype, 3), y=Y)
    r.forward(), r.backward()
    want = np.where(keep, x * scale, 0)
    _within(r.y, want + res, np.abs(want) + np.abs(want + res), dtype, "y")
    want = np.where(keep, dy * scale, 0)
    _within(r.dx, want, np.abs(want), dtype, "dx")
    around = torch.ones_like(Y._base, dtype=torch.bool)
    around[:, 2:2 + W] = False
    assert Y._base[around].isnan().all()


def test_none_all_and_what_is_dropped():
    """p 0 and 1; NaN and infinities that are dropped are gone, forward and backward."""
    ly = _ly()
    x = torch.randn(50, 33, device="cuda")
    assert torch.equal(ly.DropoutRun.of(x, 0.0, _seed()).forward(), x)
    res = torch.randn(50, 33, device="cuda")
    assert not ly.DropoutRun.of(x, 1.0, _seed()).forward().any()
    assert torch.equal(ly.DropoutRun.of(x.fill_(float("nan")), 1.0, _seed(), res).forward(), res)
    keep, _ = ref.keep(50, 33, 0.5, KEY, STEP)
    r = ly.DropoutRun.of(x, 0.5, _seed(), dy=x.clone().fill_(float("inf")))
    assert np.array_equal(np.isnan(get(r.forward())), keep)
    assert np.array_equal(np.isinf(get(r.backward())), keep) and not get(r.dx)[~keep].any()


def test_masks_differ_and_have_their_rate():
    ly = _ly()
    x = torch.ones(2000, 512, device="cuda")
    a, b, c = (ly.DropoutRun.of(x, 0.3, _seed(*s)).forward() for s in ((1, 1), (1, 2), (2, 1)))
    n = x.numel()
    for t in (a, b, c):
        rate = float((t == 0).float().mean())
        assert abs(rate - 0.3) < 5 * (0.21 / n) ** 0.5       # five standard deviations
    # two independent masks agree in 0.58 of their places
    for s, t in ((a, b), (a, c), (b, c)):
        assert abs(float(((s == 0) == (t == 0)).float().mean()) - 0.58) < 5 * (0.25 / n) ** 0.5
    # one mask for all steps
    t = ly.DropoutRun.of(x, 0.3, _seed(1, 1), period=50).forward().view(40, 50, 512)
    assert torch.equal(t, t[:1].expand_as(t)) and torch.equal(t[0], a[:50])


def test_types_share_a_mask():
    """The mask depends on place, key and step alone: 32-bit and 16-bit rows, whole or with others around them, drop the same."""
    ly = _ly()
    one = torch.ones(300, 203, device="cuda")
    a = ly.DropoutRun.of(one, 0.2, _seed()).forward()
    b = ly.DropoutRun.of(one.bfloat16(), 0.2, _seed()).forward()
    few = ly.DropoutRun.of(one[:100, :77], 0.2, _seed()).forward()
    assert torch.equal(a == 0, b == 0) and torch.equal(few, a[:100, :77])


def test_many_rows():
    """More groups than one launch has threads: the last rows are those of the mask's definition."""
    ly = _ly()
    R = (1 << 29) + 70
    x = torch.ones(R, 1, dtype=torch.bfloat16, device="cuda")
    y = ly.DropoutRun.of(x, 0.5, _seed(), y=x).forward()
    assert abs(float((y[:1 << 28] == 0).float().mean()) - 0.5) < 1e-3
    cut = lambda lo, n: np.array([_one(r) for r in range(lo, lo + n)])

    def _one(r):
        c, k, low = [0, r, STEP & 0xFFFFFFFF, STEP >> 32], [KEY & 0xFFFFFFFF, KEY >> 32], 0xFFFFFFFF
        for _ in range(10):
            a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [b >> 32 ^ c[1] ^ k[0], b & low, a >> 32 ^ c[3] ^ k[1], a & low]
            k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
        return (c[0] & 0xFFFF) >= 32768
    for lo in (0, (1 << 29) - 5, R - 50):
        assert np.array_equal(get(y[lo:lo + 50, 0])[:R - lo] != 0, cut(lo, 50)), lo
    del x, y
    torch.cuda.empty_cache()


def test_refusals():
    ly = _ly()
    x = torch.randn(4, 9, device="cuda")
    d = ly.make_dropout_dims(4, 9)
    for args in ((x.half(), None, _seed(), x), (x, x[:2], _seed(), x), (x, None, _seed().int(), x), (x, None, _seed()[:1], x), (x, None, None, x),
                 (x, None, _seed(), None), (x, None, _seed().cpu(), x)):
        with pytest.raises(ValueError):
            ly.stacklstm_dropout_fwd(d, *args)
