"""Forms of the layers' kernels that only certain sizes reach, and calls at the ends of what is allowed."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT, get, rng_for, up
from tests.test_gpu_layers_attend import check, dev, heads, inputs, within
from tests.test_gpu_layers_logprob import _check, _inputs

pytestmark = pytest.mark.gpu


def _ly():
    need_gpu()
    from paper_1904_03409_amd import layers
    return layers


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_up_to_31_bits(dtype):
    """2^31 - 2 queries of heads that share one key, a row tile short of 2^31; of one key y is its value."""
    ly = _ly()
    Tq, Hq = ((1 << 31) - 2) // 151, 151
    assert Tq * Hq == (1 << 31) - 2
    print(f"[gpu] {dtype} {Tq} queries, {Hq} heads", flush=True)
    q = torch.randn(1, 1, Hq, 1, device="cuda").to(DT[dtype]).expand(1, Tq, Hq, 1)
    k, v = (torch.randn(1, 1, 1, 1, device="cuda").to(DT[dtype]) for _ in range(2))
    y = torch.full((1, Tq, Hq, 1), 7.0, dtype=DT[dtype], device="cuda")
    ly.AttendRun.of(q, k, v, y=y).forward()
    low, high = y.aminmax()
    assert low == v.squeeze() and high == v.squeeze()
    del y
    torch.cuda.empty_cache()


# up to 16 rows (queries times the heads that share a key), whose waves share the keys, in every width by DMA and by way of registers; two row tiles to a
# wave by way of registers; dq and dk and dv of every width both ways, with keys in several tiles
SIZES = [(2, 1, 300, 8, 2, 128), (1, 4, 500, 2, 1, 100), (1, 3, 200, 2, 2, 131), (2, 2, 300, 2, 1, 256), (3, 2, 150, 8, 1, 27), (2, 5, 400, 3, 3, 32), (1, 16, 170, 1, 1, 61),
         (2, 3, 290, 4, 1, 64), (2, 70, 90, 2, 2, 50), (2, 90, 70, 2, 1, 30), (1, 50, 150, 2, 1, 63), (2, 40, 140, 2, 2, 29), (1, 80, 300, 2, 1, 121), (1, 60, 150, 1, 1, 250), (2, 34, 135, 1, 1, 32),
         (2, 100, 140, 2, 2, 64), (1, 65, 129, 1, 1, 24), (1, 20, 130, 4, 1, 160), (2, 3, 180, 2, 1, 101),
         (1, 20, 100, 2, 1, 121), (2, 24, 100, 2, 2, 40), (3, 300, 300, 90, 90, 132), (3, 290, 310, 90, 90, 131)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_forms(size, dtype):
    ly = _ly()
    rng = rng_for("forms", *size, dtype)
    check(ly, *inputs(rng, *size, dtype, lens=size[0] > 1, mask=size[5] % 2 == 0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(400, 130, 100, 4, 4, 40), (400, 130, 100, 4, 4, 37), (200, 300, 128, 4, 2, 24), (200, 300, 65, 4, 2, 21), (820, 70, 64, 2, 1, 64), (820, 70, 33, 2, 1, 17)])
def test_several_row_tiles_over_keys_that_stay(size, dtype):
    """A workgroup's later row tiles behind the last query, keys that end in the first tile or the second, masks, sequences without keys; NaN and
    infinities in what is not there."""
    ly = _ly()
    rng = rng_for("stay", *size, dtype)
    B, Tq, Tk, Hq, Hk, D = size
    s, q_len, k_len, m = inputs(rng, *size, dtype, lens=True, mask=True)
    m[4:B // 2] |= 1                                     # (all keys of these are there)
    q_len[5:9] = Tq, 0, 65, 64
    k_len[5:9] = Tk, Tk, 1, Tk // 2
    ok = ref.seen(B, Tq, Tk, q_len, k_len, m)
    clean = {n: a.copy() for n, a in s.items()}
    no_key, no_query = ~ref.seen(B, 1, Tk, None, k_len, m)[:, 0], ~ok.any(2)
    for n, none in (("k", no_key), ("v", no_key), ("q", no_query), ("dy", no_query)):
        s[n][none] = rng.choice([np.nan, np.inf, -np.inf], s[n][none].shape)
    t = {n: heads(a, dtype) for n, a in s.items()}
    r = ly.AttendRun.of(t["q"], t["k"], t["v"], dev(q_len), dev(k_len), dev(m), dy=t["dy"])
    for x in (r.y, r.dq, r.dk, r.dv):
        x.fill_(7)
    r.forward(), r.backward()
    assert not get(r.y)[no_query].any() and not get(r.dq)[no_query].any()
    some = np.unique(np.r_[0:10, B - 2, B - 1, rng.integers(0, B, 20)])
    want, off = ref.attend(*(clean[n][some] for n in "qkv"), ok[some], D ** -0.5, clean["dy"][some], dtype, bounds=True)
    for n, x in (("y", r.y), ("dq", r.dq), ("dk", r.dk), ("dv", r.dv)):
        within(x[torch.from_numpy(some).cuda()], want[n], off[n], n)
    # without a mask and lengths (whole tiles), against every sequence alone
    y = ly.AttendRun.of(*(heads(clean[n], dtype) for n in "qkv")).forward()
    for b in (0, B // 3, B - 1):
        one = ly.AttendRun.of(*(heads(clean[n][b:b + 1], dtype) for n in "qkv")).forward()
        want, off = ref.attend(*(clean[n][b:b + 1] for n in "qkv"), ref.seen(1, Tq, Tk), D ** -0.5, None, dtype, bounds=True)
        within(y[b:b + 1], want["y"], off["y"], "y")
        within(one, want["y"], off["y"], "y alone")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,G,N", [(30, 700, 2, 3), (513, 20001, 1, 5)])
def test_best_tokens(R, V, G, N, dtype):
    """Two and four vectors in a lane of a wave, a workgroup of 512 threads to a row."""
    ly = _ly()
    rng = rng_for("forms", R, V, G, N, dtype)
    x, token, legal, a, h = _inputs(rng, R, V, G, dtype)
    few = np.unique(np.r_[0:4, R - 1, rng.integers(0, R, 8)])
    want = ref.logprob(x[few], token[few], legal[few], N, a[few].astype(np.float64), h[few].astype(np.float64))
    r = ly.LogProbRun.of(up(x, dtype), up(token), up(legal), N, up(a), up(h))
    r.step()
    _check(r, few, want, dtype, a[few], h[few])
    r.forward(), r.backward()
    _check(r, few, want, dtype, a[few], h[few])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 50, 70, 4, 2, 64), (2, 9, 300, 4, 1, 48), (2, 33, 90, 2, 2, 160)])
def test_mixed_layouts(size, dtype):
    """Every matrix in a layout of its own: queries and dy in wider buffers, keys steps first, values heads first, gradients in other orders."""
    ly = _ly()
    rng = rng_for("mixed", *size, dtype)
    B, Tq, Tk, Hq, Hk, D = size
    s, q_len, k_len, m = inputs(rng, *size, dtype, lens=True, mask=True)
    v = heads(s["v"], dtype).permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    big = torch.full((Tq, B, Hq, D + 5), 5.0, dtype=DT[dtype], device="cuda")
    y = big[..., 2:2 + D].transpose(0, 1)
    r = ly.AttendRun.of(heads(s["q"], dtype, pad=3), heads(s["k"], dtype, steps_first=True), v, dev(q_len), dev(k_len), dev(m), None,
                        heads(s["dy"], dtype, pad=1, steps_first=True), y)
    r.dk = torch.full((Hk, Tk, B, D), 7.0, dtype=DT[dtype], device="cuda").permute(2, 1, 0, 3)
    r.dims.dk = ly.strides_of(r.dk)
    r.forward(), r.backward()
    want, off = ref.attend(s["q"], s["k"], s["v"], ref.seen(B, Tq, Tk, q_len, k_len, m), D ** -0.5, s["dy"], dtype, bounds=True)
    for n, x in (("y", r.y), ("dq", r.dq), ("dk", r.dk), ("dv", r.dv)):
        within(x, want[n], off[n], n)
    assert (big[..., :2] == 5).all() and (big[..., 2 + D:] == 5).all()


def test_graphs_of_split_calls():
    """Calls that go through a work space, and of more than 64 KB of LDS, captured together and replayed with other inputs and lengths."""
    ly = _ly()
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    runs = []
    for D, dtype in ((256, "f32"), (128, "bf16"), (50, "f32")):
        e = lambda T, H: rand(2, T, H, D).to(DT[dtype])
        k_len = torch.tensor([700, 333], dtype=torch.int32, device="cuda")
        runs.append(ly.AttendRun.of(e(40, 4), e(700, 2), e(700, 2), k_len=k_len, dy=e(40, 4)))
    lp = ly.LogProbRun.of(rand(3, 70000), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), top=4, dlogp=rand(3, 1))

    def step():
        for r in runs:
            r.forward(), r.backward()
        lp.step()
    outputs = lambda: [t for r in runs for t in (r.y, r.dq, r.dk, r.dv)] + [lp.logp, lp.entropy, lp.index, lp.value, lp.dlogits]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for r in runs:
            r.q.copy_(rand(*r.q.shape))
            r.k_len.copy_(torch.randint(0, 701, (2,), generator=g, device="cuda"))
        lp.logits.copy_(rand(3, 70000))
        step()
        want = [t.clone() for t in outputs()]
        for t in outputs() + [r.workspace for r in runs] + [lp.workspace]:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outputs())), i
