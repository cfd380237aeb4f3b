"""Attention to an encoder's states on the GPU against 64 bits."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT, get, rng_for, rounded, up

pytestmark = pytest.mark.gpu


def _ly():
    need_gpu()
    from paper_1904_03409_amd import layers
    return layers


def within(got, want, off, what):
    got = get(got)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    err = np.abs(got - want) - off
    worst = np.unravel_index(np.argmax(err), err.shape) if err.size else None
    assert err.size == 0 or err[worst] <= 1e-30, f"{what} {worst}: {got[worst]} for {want[worst]}, off by more than {off[worst]}"


def heads(a, dtype, steps_first=False, pad=0):
    """a on the GPU; steps_first: as a view of [T, B, H, D]; pad: heads apart in a wider buffer of NaN, at an odd place."""
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype])
    if steps_first:
        t = t.transpose(0, 1).contiguous()
    if pad:
        big = torch.full((*t.shape[:3], t.shape[3] + 2 * pad), float("nan"), dtype=t.dtype, device="cuda")
        big[..., pad:pad + t.shape[3]] = t.cuda()
        t = big[..., pad:pad + t.shape[3]]
    else:
        t = t.cuda()
    return t.transpose(0, 1) if steps_first else t


def inputs(rng, B, Tq, Tk, Hq, Hk, D, dtype, lens=False, mask=False):
    s = {n: rounded(rng.standard_normal(shape), dtype) for n, shape in
         (("q", (B, Tq, Hq, D)), ("k", (B, Tk, Hk, D)), ("v", (B, Tk, Hk, D)), ("dy", (B, Tq, Hq, D)))}
    q_len = rng.integers(0, Tq + 1, B).astype(np.int32) if lens else None
    k_len = rng.integers(0, Tk + 1, B).astype(np.int32) if lens else None
    if lens:
        q_len[-1], k_len[-1] = Tq + 3, Tk + 9            # past the end: all
        if B > 1:
            k_len[0] = min(1, Tk)
        if B > 2:
            k_len[1] = -4                                # below 0: none
    m = (rng.random((B, Tk)) < 0.6).astype(np.uint8) * rng.integers(1, 256, (B, Tk)).astype(np.uint8) if mask else None
    if mask and B > 3:
        m[2] = 0                                         # no key at all
    return s, q_len, k_len, m


def dev(a):
    return None if a is None else up(a)


def check(ly, s, q_len, k_len, m, dtype, scale=None, train=True, **layout):
    B, Tq, Hq, D = s["q"].shape
    Tk = s["k"].shape[1]
    ok = ref.seen(B, Tq, Tk, q_len, k_len, m)
    want, off = ref.attend(s["q"], s["k"], s["v"], ok, D ** -0.5 if scale is None else float(np.float32(scale)),
                           s["dy"] if train else None, dtype, bounds=True)
    t = {n: heads(a, dtype, **layout) for n, a in s.items()}
    r = ly.AttendRun.of(t["q"], t["k"], t["v"], dev(q_len), dev(k_len), dev(m), scale, t["dy"] if train else None)
    r.y.fill_(7)
    r.forward()
    within(r.y, want["y"], off["y"], "y")
    if train:
        for x in (r.dq, r.dk, r.dv):
            x.fill_(7)
        r.workspace.fill_(255)
        r.backward()
        for n in ("dq", "dk", "dv"):
            within(getattr(r, n), want[n], off[n], n)
    return r


# one of everything; both sides of the row tiles (16, 64, 128), key tiles (16, 32, 64, 128) and widths (32, 64, 128, 256); odd widths
SIZES = [(1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 1, 5), (3, 1, 17, 4, 4, 16), (2, 16, 33, 3, 3, 31), (1, 17, 64, 2, 1, 32), (4, 15, 65, 4, 1, 33),
         (5, 63, 60, 2, 2, 50), (2, 65, 128, 4, 2, 64), (3, 40, 129, 6, 3, 65), (2, 129, 31, 2, 2, 100), (1, 70, 200, 8, 2, 128),
         (2, 33, 90, 2, 1, 129), (1, 130, 70, 1, 1, 200), (2, 20, 47, 3, 1, 256), (1, 5, 300, 8, 1, 255), (2, 200, 260, 2, 1, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_backward(size, dtype):
    ly = _ly()
    rng = rng_for("attend", *size, dtype)
    check(ly, *inputs(rng, *size, dtype), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 40, 2, 2, 2, 200), (2, 150, 4, 4, 2, 128), (2, 30, 16, 2, 1, 256), (2, 70, 3, 1, 1, 64), (3, 21, 11, 3, 1, 72)])
def test_few_keys(size, dtype):
    """p (dp - delta) is small beside its terms: delta has to be as exact as they are."""
    ly = _ly()
    rng = rng_for("few", *size, dtype)
    check(ly, *inputs(rng, *size, dtype), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 64, 100, 128, 256])
def test_one_key(D, dtype):
    """Of one key (alone, or the only one that is there) y is its value, and moves with neither queries nor keys."""
    ly = _ly()
    rng = rng_for("one key", D, dtype)
    for Tk in (1, 12):
        s, _, _, _ = inputs(rng, 3, 33, Tk, 4, 2, D, dtype)
        m = np.zeros((3, Tk), np.uint8)
        m[:, Tk // 2] = 1
        r = check(ly, s, None, None, m, dtype)
        assert not r.dq.any() and not r.dk.any()
        assert np.array_equal(get(r.y), np.repeat(s["v"][:, Tk // 2:Tk // 2 + 1], 33, 1).repeat(2, 2))


def test_one_key_outweighs_the_others():
    """Many keys, of which one has nearly all of the weight: what its gradient is made of is far smaller than its terms."""
    ly = _ly()
    rng = rng_for("peak")
    s, _, _, _ = inputs(rng, 2, 40, 300, 2, 2, 128, "bf16")
    at = rng.integers(0, 300, (2, 40))
    for b in range(2):
        for t in range(40):
            s["q"][b, t] = rounded(s["k"][b, at[b, t]] * 0.55, "bf16")   # a score 6 above the others' spread
    ok = ref.seen(2, 40, 300)
    want = ref.attend(s["q"], s["k"], s["v"], ok, 128 ** -0.5, s["dy"])
    r = ly.AttendRun.of(*(heads(s[n], "bf16") for n in "qkv"), dy=heads(s["dy"], "bf16"))
    r.forward(), r.backward()
    for n in ("dq", "dk"):
        g, w = get(getattr(r, n)), want[n]
        # roundings of p, s and the output (each 2^-9 of the value in the mean square at most, sqrt(3) together) and as much again
        assert np.linalg.norm(g - w) <= 2 * 3 ** 0.5 * 2.0 ** -9 * np.linalg.norm(w), (n, np.linalg.norm(g - w) / np.linalg.norm(w))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(6, 9, 40, 2, 2, 24), (5, 70, 150, 4, 2, 64), (4, 140, 90, 2, 1, 120), (4, 1, 700, 4, 2, 40), (5, 33, 20, 2, 2, 256)])
def test_lengths_and_masks(size, dtype):
    """Ragged queries and keys, masked keys, sequences without any key; what is not there holds NaN and infinities."""
    ly = _ly()
    rng = rng_for("lens", *size, dtype)
    s, q_len, k_len, m = inputs(rng, *size, dtype, lens=True, mask=True)
    ok = ref.seen(size[0], size[1], size[2], q_len, k_len, m)
    clean = {n: a.copy() for n, a in s.items()}
    no_key = ~ref.seen(size[0], 1, size[2], None, k_len, m)[:, 0]
    no_query = ~ok.any(2)
    for n in ("k", "v"):
        s[n][no_key] = rng.choice([np.nan, np.inf, -np.inf], s[n][no_key].shape)
    for n in ("q", "dy"):
        s[n][no_query] = rng.choice([np.nan, np.inf, -np.inf], s[n][no_query].shape)
    want, off = ref.attend(clean["q"], clean["k"], clean["v"], ok, size[5] ** -0.5, clean["dy"], dtype, bounds=True)
    t = {n: heads(a, dtype) for n, a in s.items()}
    r = ly.AttendRun.of(t["q"], t["k"], t["v"], dev(q_len), dev(k_len), dev(m), dy=t["dy"])
    r.forward(), r.backward()
    for n, x in (("y", r.y), ("dq", r.dq), ("dk", r.dk), ("dv", r.dv)):
        within(x, want[n], off[n], n)
    assert not get(r.y)[no_query].any() and not get(r.dq)[no_query].any()
    assert not get(r.dk)[no_key].any() and not get(r.dv)[no_key].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [dict(steps_first=True), dict(pad=3), dict(steps_first=True, pad=1), dict(pad=8)])
def test_strides(layout, dtype):
    ly = _ly()
    for size in ((3, 50, 70, 4, 2, 64), (2, 20, 33, 2, 2, 37)):
        rng = rng_for("astride", *size, dtype)
        r = check(ly, *inputs(rng, *size, dtype, lens=True), dtype, **layout)
        assert (r.y.stride(0) < r.y.stride(1)) == layout.get("steps_first", False)


def test_outputs_in_a_wider_buffer():
    """y as a view between columns that keep what they hold; broadcast keys of one encoder for all sequences."""
    ly = _ly()
    rng = rng_for("wider")
    s, _, _, _ = inputs(rng, 4, 30, 45, 2, 2, 40, "f32")
    s["k"][:], s["v"][:] = s["k"][:1], s["v"][:1]
    q = heads(s["q"], "f32")
    k, v = (heads(s[n][:1], "f32").expand(4, -1, -1, -1) for n in ("k", "v"))
    # (one key for all places, too: a stride of 0 along them)
    one = heads(s["v"][:1, :1], "f32").expand(4, 45, -1, -1)
    assert torch.equal(ly.AttendRun.of(q, one, one).forward(), ly.AttendRun.of(q, one.contiguous(), one.contiguous()).forward())
    big = torch.full((4, 30, 2, 47), 5.0, device="cuda")
    r = ly.AttendRun.of(q, k, v, y=big[..., 3:43])
    r.forward()
    want, off = ref.attend(s["q"], s["k"], s["v"], ref.seen(4, 30, 45), 40 ** -0.5, None, "f32", bounds=True)
    within(r.y, want["y"], off["y"], "y")
    assert (big[..., :3] == 5).all() and (big[..., 43:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 5000, 2, 2, 64), (2, 8, 3000, 8, 2, 128), (1, 40, 2049, 1, 1, 256), (1, 200, 1500, 1, 1, 32), (3, 3, 999, 2, 1, 50)])
def test_long_keys_are_split(size, dtype):
    ly = _ly()
    rng = rng_for("split", *size, dtype)
    s, q_len, k_len, m = inputs(rng, *size, dtype, lens=size[0] > 1, mask=True)
    r = check(ly, s, q_len, k_len, m, dtype)
    assert ly.stacklstm_attend_fwd_workspace_bytes(r.dims) > 64
    y = r.y.clone()
    r.workspace.fill_(255)
    r.forward()
    assert torch.equal(r.y, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_from_zero(dtype):
    """Rows whose scores rise tile after tile, are very large, or very negative; scales of either sign, 0, and large."""
    ly = _ly()
    B, Tq, Tk, D = 1, 20, 300, 16
    rng = rng_for("far", dtype)
    s, _, _, _ = inputs(rng, B, Tq, Tk, 1, 1, D, dtype)
    s["q"][..., 0], s["k"][..., 0] = 8.0, rounded(np.linspace(-30, 30, Tk), dtype)[None, :, None]
    for scale in (0.25, -0.25, 0.0, 2.0):
        check(ly, s, None, None, None, dtype, scale)
    # a constant added to every score of a row changes nothing: 2^12 and 2^40 with a row's other terms exact in 32 bits
    for big in (4096.0, 2.0 ** 40):
        z = {n: a.copy() for n, a in s.items()}
        z["q"][..., 0], z["k"][..., 0] = big, 1.0
        z["q"][..., 1:], z["k"][..., 1:] = 0, 0
        r = check(ly, z, None, None, None, dtype, 1.0)
        assert np.abs(get(r.y) - z["v"].mean(1, keepdims=True)).max() < 2e-2
    # the largest score alone counts where the others are far below it
    z = {n: a.copy() for n, a in s.items()}
    z["q"][:], z["k"][:] = 0, 0
    z["q"][..., 0] = 2.0 ** 50
    z["k"][:, :, 0, 0] = -1
    z["k"][:, 77, 0, 0] = 1
    r = ly.AttendRun.of(*(heads(z[n], dtype) for n in "qkv"), scale=1.0, dy=heads(z["dy"], dtype))
    r.forward(), r.backward()
    assert np.array_equal(get(r.y)[0, :, 0], np.tile(z["v"][0, 77, 0], (Tq, 1)))
    assert np.isfinite(get(r.dq)).all() and np.isfinite(get(r.dk)).all() and not get(r.dv)[0, :77].any()


def test_nan_and_infinities_stay_in_their_rows():
    ly = _ly()
    rng = rng_for("nonfinite")
    s, _, _, _ = inputs(rng, 3, 40, 50, 2, 2, 24, "f32")
    s["q"][0, 5, 1, 3] = np.nan
    s["k"][1, 7, 0, 2] = -np.inf                         # a key whose scores are -inf or +inf
    s["q"][1, :, 0, 2] = 1.0
    r = ly.AttendRun.of(*(heads(s[n], "f32") for n in "qkv"))
    r.forward()
    y = get(r.y)
    assert np.isnan(y[0, 5, 1]).all() and np.isfinite(np.delete(y[0, :, 1], 5, 0)).all() and np.isfinite(y[0, :, 0]).all()
    k = np.delete(s["k"][1:2], 7, 1), np.delete(s["v"][1:2], 7, 1)
    want, off = ref.attend(s["q"][1:2], *k, ref.seen(1, 40, 49), 24 ** -0.5, None, "f32", bounds=True)
    within(r.y[1:2, :, 0], want["y"][:, :, 0], off["y"][:, :, 0], "y without the key at -inf")
    s["k"][2, :, 1, 0], s["q"][2, :, 1, 0] = -np.inf, 1.0            # all of a row's scores -inf: no key
    r = ly.AttendRun.of(*(heads(s[n], "f32") for n in "qkv"), dy=heads(np.nan_to_num(s["dy"]), "f32"))
    r.forward(), r.backward()
    assert not get(r.y)[2, :, 1].any() and not get(r.dq)[2, :, 1].any()


def test_no_keys_and_no_queries():
    ly = _ly()
    e = lambda *s: torch.randn(*s, device="cuda")
    r = ly.AttendRun.of(e(2, 3, 2, 8), e(2, 0, 2, 8), e(2, 0, 2, 8), dy=e(2, 3, 2, 8))
    r.y.fill_(7), r.dq.fill_(7)
    r.forward(), r.backward()
    assert not r.y.any() and not r.dq.any()
    r = ly.AttendRun.of(e(2, 0, 2, 8), e(2, 5, 2, 8), e(2, 5, 2, 8), dy=e(2, 0, 2, 8))
    r.dk.fill_(7), r.dv.fill_(7)
    r.forward(), r.backward()
    assert not r.dk.any() and not r.dv.any()
    r = ly.AttendRun.of(e(0, 4, 2, 8), e(0, 5, 2, 8), e(0, 5, 2, 8), dy=e(0, 4, 2, 8))
    r.forward(), r.backward()


def test_differences():
    ly = _ly()
    rng = rng_for("adiff")
    s, q_len, k_len, m = inputs(rng, 4, 9, 21, 4, 2, 12, "f32", lens=True, mask=True)
    lens = dev(q_len), dev(k_len), dev(m)
    f = lambda z: (get(ly.AttendRun.of(heads(z["q"], "f32"), heads(z["k"], "f32"), heads(z["v"], "f32"), *lens).forward()) * z["dy"]).sum()
    r = ly.AttendRun.of(heads(s["q"], "f32"), heads(s["k"], "f32"), heads(s["v"], "f32"), *lens, dy=heads(s["dy"], "f32"))
    r.forward(), r.backward()
    h = 2.0 ** -6
    for n in "qkv":
        u = rng.standard_normal(s[n].shape)
        move = lambda c: {**s, n: s[n] + c * u}
        num, g = (f(move(h)) - f(move(-h))) / (2 * h), get(getattr(r, "d" + n)) * u
        # third derivatives: h^2 of a term's size; fp32's rounding of the sums over h
        assert abs(num - g.sum()) <= 10 * h * h * np.abs(g).sum() + 1e-6 / h * np.abs(get(r.y) * s["dy"]).sum()


def test_offsets_past_32_bits():
    """Keys and queries whose places in their buffers lie past 2^31 elements and 2^32 bytes."""
    ly = _ly()
    rng = rng_for("far offsets")
    s, _, _, _ = inputs(rng, 2, 20, 40, 1, 1, 32, "bf16")
    apart = (1 << 31) + 40 * 32 + 7
    big = torch.empty(apart + (1 << 16), dtype=torch.bfloat16, device="cuda")

    def view(a, at):
        v = big.as_strided(a.shape, (apart, a.shape[3], a.shape[3], 1), at)
        v.copy_(torch.from_numpy(a))
        return v
    q, k, v, dy = (view(s[n], i << 12) for i, n in enumerate(("q", "k", "v", "dy")))
    ok = ref.seen(2, 20, 40)
    want, off = ref.attend(s["q"], s["k"], s["v"], ok, 32 ** -0.5, s["dy"], "bf16", bounds=True)
    r = ly.AttendRun.of(q, k, v, dy=dy, y=big.as_strided(q.shape, q.stride(), 4 << 12))
    r.dq, r.dk, r.dv = (big.as_strided(t.shape, t.stride(), i << 12) for t, i in ((q, 5), (k, 6), (v, 7)))
    r.dims.dq, r.dims.dk, r.dims.dv = ly.strides_of(r.dq), ly.strides_of(r.dk), ly.strides_of(r.dv)
    r.forward(), r.backward()
    for n, x in (("y", r.y), ("dq", r.dq), ("dk", r.dk), ("dv", r.dv)):
        within(x, want[n], off[n], n)


def test_many_workgroups():
    """More row tiles than one launch has workgroups (2^21): a query and a key to a sequence; y is v."""
    ly = _ly()
    B = (1 << 21) + 300
    e = lambda: torch.randn(B, 1, 1, 4, device="cuda")
    r = ly.AttendRun.of(e(), e(), e(), dy=e())
    r.y.fill_(7)
    r.forward(), r.backward()
    assert float((r.y - r.v).abs().max()) < 1e-6 and float((r.dv - r.dy).abs().max()) < 1e-6
    assert float(r.dq.abs().max()) < 1e-5 and float(r.dk.abs().max()) < 1e-5


def test_refusals():
    ly = _ly()
    q, k = torch.randn(2, 3, 2, 8, device="cuda"), torch.randn(2, 5, 2, 8, device="cuda")
    d = ly.make_attend_dims(2, 3, 5, 2, 2, 8)
    ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    y = torch.empty_like(q)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    for args in ((q.half(), k, k, None, None, None, y), (q, k.bfloat16(), k, None, None, None, y), (q, k[:, :4], k, None, None, None, y),
                 (q, k, k, i32(3), None, None, y), (q, k, k, None, i32(2).long(), None, y), (q, k, k, None, None, torch.ones(2, 4, device="cuda"), y),
                 (q, k, k, None, None, None, y.transpose(0, 1).contiguous().transpose(0, 1)), (q, k, None, None, None, None, y), (q.cpu(), k, k, None, None, None, y)):
        with pytest.raises((ValueError, AssertionError)):
            ly.stacklstm_attend_fwd(d, *args, None, ws)
    with pytest.raises(ValueError):
        ly.AttendRun.of(q.transpose(2, 3), k, k)
    with pytest.raises(Exception):
        ly.AttendRun.of(torch.randn(2, 3, 3, 8, device="cuda"), k, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 7, 3000, 2, 1, 48), (2, 65, 1100, 2, 2, 128), (1, 300, 700, 1, 1, 100), (1, 1500, 300, 2, 1, 200)])
def test_gradients_are_split(size, dtype):
    """Few row or key tiles: dq's keys, dk's and dv's queries over several workgroups; ragged, strided, with equal bits each time."""
    ly = _ly()
    rng = rng_for("gsplit", *size, dtype)
    s, q_len, k_len, m = inputs(rng, *size, dtype, lens=size[0] > 1, mask=True)
    r = check(ly, s, q_len, k_len, m, dtype, steps_first=True)
    got = [t.clone() for t in (r.dq, r.dk, r.dv)]
    r.workspace.fill_(255)
    r.backward()
    assert all(torch.equal(a, b) for a, b in zip(got, (r.dq, r.dk, r.dv)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(40, 2, 600, 8, 8, 24), (70, 3, 400, 8, 4, 50), (40, 1, 700, 7, 7, 136)])
def test_keys_are_split_for_few_rows_of_many_heads(size, dtype):
    """More row tiles than compute units, of which one wave has all the rows: dq's keys are split for these too."""
    ly = _ly()
    rng = rng_for("few rows", *size, dtype)
    s, q_len, k_len, m = inputs(rng, *size, dtype, lens=True, mask=True)
    check(ly, s, q_len, k_len, m, dtype)
