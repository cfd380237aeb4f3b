"""Beam search on the GPU: the selection exact (against a list of all continuations), the copies byte for byte."""
import numpy as np
import pytest
import torch

from tests import head_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import close, get, rng_for, rounded, strided, up

pytestmark = pytest.mark.gpu


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


def _select(hd, x, score, done=None, legal=None, eos=-1, dtype="f32"):
    r = hd.BeamRun.of(x if isinstance(x, torch.Tensor) else up(x, dtype), up(score, "f32"),
                      None if done is None else up(done), None if legal is None else up(legal), eos)
    r.select()
    return [t.cpu().numpy() for t in (r.score_next, r.parent, r.token, r.done_next)]


def _check(got, x, score, done, legal, eos, exact=False):
    """exact: the softmax sums are exact in 32 bits (up to the log), so places and ties are compared whole; otherwise every
    place is compared but where two totals of the reference are within rounding of each other."""
    want = ref.beam(x.astype(np.float32), legal, score.astype(np.float32), done, eos)
    close(got[0].astype(np.float64), want[0].astype(np.float64), "f32", "score_next")
    near = np.zeros(want[0].shape, bool)
    if not exact:
        with np.errstate(all="ignore"):
            gap = np.abs(np.diff(want[0].astype(np.float64), axis=1))
            tight = gap <= 4e-6 * np.maximum(1, np.abs(want[0][:, 1:]))
        near[:, 1:] |= tight
        near[:, :-1] |= tight
        near[:, -1] = True                             # (the next one past the end is not known)
    for g, w, name in zip(got[1:], want[1:], ("parent", "token", "done_next")):
        assert np.array_equal(g[~near], w[~near]), name


SIZES = [(1, 1, 1), (2, 1, 7), (3, 4, 2), (5, 8, 83), (2, 64, 3), (1, 64, 128), (2, 16, 512), (1, 3, 2731), (4, 2, 4096), (3, 5, 4097),
         (2, 16, 8193), (1, 2, 16390), (40, 7, 5003), (300, 1, 9000), (1, 4, 40001), (130, 2, 33000), (1, 64, 70001), (66, 4, 65600),
         (1, 1, 131072)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V", SIZES)
def test_select(B, K, V, dtype):
    hd = _hd()
    rng = rng_for("beam", B, K, V, dtype)
    x = rounded(2.5 * rng.standard_normal((B * K, V)), dtype)
    score = (-20 * rng.random((B, K)) - 1).astype(np.float32)
    done = (rng.random((B, K)) < 0.2).astype(np.uint8) if (B + K) % 2 else None
    legal = (rng.random((B * K, V)) < 0.6).astype(np.uint8) if V % 2 else None
    if B * K > 4:
        score[0, 0] = -np.inf                           # a beam that is not there
        if legal is not None:
            legal[1] = 0                                # one without a legal token
    got = _select(hd, x, score, done, legal, 1, dtype)
    few = np.arange(min(B, 3))
    rows = (few[:, None] * K + np.arange(K)).reshape(-1)
    _check([g[few] for g in got], x[rows], score[few], None if done is None else done[few], None if legal is None else legal[rows], 1)
    again = _select(hd, x, score, done, legal, 1, dtype)
    assert all(np.array_equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("V", [64, 2048, 4096, 16384, 40960, 131072])
@pytest.mark.parametrize("K", [1, 16, 64])
def test_ties_go_to_the_lower_place(V, K):
    """Logits of few values, powers of two of each: equal totals everywhere, also more of them than a list holds."""
    hd = _hd()
    rng = rng_for("ties", V, K)
    for kind in ("equal", "two", "few", "period"):
        x = np.zeros((K, V))
        if kind == "two":
            x[:, V // 2:] = 1.0
        elif kind == "few":
            x = np.round(2 * rng.standard_normal((K, V)))
        elif kind == "period":                          # all large ones with a few threads
            x[:, np.arange(V) % 1024 < 8] = 3.0
        score = np.where(np.arange(K) % 2, -1.0, -2.0).astype(np.float32)[None]
        got = _select(hd, x, score)
        # with the GPU's own log sums: read off the best continuation of each beam alone
        lse = []
        for k in range(K):
            one = _select(hd, x[k:k + 1], np.zeros((1, 1), np.float32))
            lse.append(np.float64(x[k].max()) - np.float64(one[0][0, 0]))
            w = x[k]
            assert abs(lse[-1] - (w.max() + np.log(np.exp(w - w.max()).sum()))) < 1e-5
        want = ref.beam(x.astype(np.float32), None, score, None, -1, lse=np.array(lse, np.float32))
        if len(set(np.float32(v) for v in lse)) == 1 or kind != "few":
            assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2]), kind
        assert (np.diff(got[0][0]) <= 0).all()
        # ties in falling order of totals, rising order of places
        place = got[1][0].astype(np.int64) * V + got[2][0]
        same = np.diff(got[0][0]) == 0
        assert (np.diff(place)[same] > 0).all(), kind


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", [(64, 83), (64, 1500), (64, 9000), (64, 33000), (64, 64001), (2, 64001), (3, 131072)])
def test_one_beam_ranks_its_logits(B, V, dtype):
    """Where one beam is alive, the continuations are its logits in order, equal ones by their place and with equal totals:
    a row has one log sum, whichever threads look at its tokens."""
    hd = _hd()
    rng = rng_for("beam one", B, V, dtype)
    K = 16
    x = rounded(2.5 * rng.standard_normal((B * K, V)), "bf16")
    score = np.full((B, K), -np.inf, np.float32)
    alive = rng.integers(0, K, B)
    score[np.arange(B), alive] = -20 * rng.random(B) - 1
    got = _select(hd, x, score, dtype=dtype)
    row = x[np.arange(B) * K + alive]
    order = np.argsort(-row, axis=1, kind="stable")[:, :K]
    assert np.array_equal(got[1], np.repeat(alive[:, None], K, 1))
    assert np.array_equal(got[2], order)
    top = np.take_along_axis(row, order, 1)
    assert np.array_equal(np.diff(got[0], axis=1) == 0, np.diff(top, axis=1) == 0)


@pytest.mark.parametrize("V", [90, 5000, 50000])
def test_nonfinite_and_masked(V):
    hd = _hd()
    rng = rng_for("bnan", V)
    B, K = 1, 8
    x = rng.standard_normal((B * K, V))
    x[0, 5] = np.nan
    x[1, 6] = np.inf
    x[2] = -np.inf
    x[3] = np.finfo(np.float32).min
    x[4, 3:] = -np.inf
    x[5, :V // 2] = np.finfo(np.float32).min
    score = np.full((B, K), -1.0, np.float32)
    score[0, 6], score[0, 7] = np.nan, -np.inf
    got = _select(hd, x, score)
    _check(got, x, score, None, None, -1, exact=False)
    assert not np.isin(got[1][got[0] > -np.inf], [0, 1, 2, 6, 7]).any()
    # nothing at all: every place its own parent
    got = _select(hd, np.full((B * K, V), -np.inf), score)
    assert np.all(got[0] == -np.inf) and np.array_equal(got[1][0], np.arange(K)) and (got[2] == -1).all() and got[3].all()
    # fewer continuations than beams
    legal = np.zeros((B * K, V), np.uint8)
    legal[4, 1] = legal[5, V - 1] = 1
    got = _select(hd, x, score, legal=legal)
    assert (got[0][0] > -np.inf).sum() == 2 and set(got[2][0][:2]) == {1, V - 1} and np.array_equal(got[1][0][2:], np.arange(2, K))
    assert abs(got[0][0][:2] + 1).max() < 1e-6          # a token alone has probability 1


def test_finished_beams():
    hd = _hd()
    for V in (50, 6000):
        x = np.zeros((3, V))
        score = np.array([[-1.0, -2.0, np.log(1 / V) - 1.0]], np.float32)
        done = np.array([[0, 1, 1]], np.uint8)
        s, parent, token, dn = _select(hd, x, score, done, None, 0)
        assert parent[0, 0] == 1 and token[0, 0] == -1 and s[0, 0] == -2 and dn[0, 0] == 1
        assert token[0, 1] == 0 and parent[0, 1] == 0 and dn[0, 1] == 1
        assert token[0, 2] == 1 and dn[0, 2] == 0       # the tie with the third beam's score goes to the lower place


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_logits(dtype):
    hd = _hd()
    rng = rng_for("bstride", dtype)
    for V in (77, 4111, 40005):
        x = rounded(rng.standard_normal((6, V)), dtype)
        score = -rng.random((2, 3)).astype(np.float32)
        a = _select(hd, x, score, dtype=dtype)
        b = _select(hd, strided(x, dtype, 3), score, dtype=dtype)
        assert all(np.array_equal(p, q) for p, q in zip(a, b))


def test_reorder():
    hd = _hd()
    rng = rng_for("reorder")
    B, K = 5, 6
    n = B * K
    d = hd.make_beam_dims(B, K, 1)
    shapes = [((n, 9, 16), torch.float32), ((n, 9, 7), torch.bfloat16), ((n,), torch.int32), ((n, 3), torch.uint8), ((n, 40, 257), torch.float32),
              ((n, 1, 8192), torch.bfloat16), ((n, 5, 3, 11), torch.uint8)]
    live9 = torch.from_numpy(rng.integers(-1, 12, n).astype(np.int32)).cuda()        # below 0 and past the end too
    live40 = torch.from_numpy(rng.integers(0, 41, n).astype(np.int32)).cuda()
    lives = [live9, live9, None, None, live40, None, live9.clamp(max=5)]
    parent = torch.from_numpy(rng.integers(0, K, (B, K)).astype(np.int32)).cuda()
    parent[1, 2], parent[2, 3] = -1, K                  # no such beam: nothing is copied
    src = [torch.from_numpy(rng.integers(0, 100, s)).to(t).cuda() for s, t in shapes]
    dst = [torch.full(s, 101, dtype=t, device="cuda") for s, t in shapes]
    hd.stacklstm_beam_reorder(d, parent, list(zip(src, dst, lives)))
    p = parent.cpu().numpy().reshape(-1)
    for s, o, lv in zip(src, dst, lives):
        want = torch.full_like(s, 101).cpu()
        for r in range(n):
            if 0 <= p[r] < K:
                q = r // K * K + p[r]
                if s.dim() == 1:
                    want[r] = s[q].cpu()
                else:
                    u = s.shape[1] if lv is None else int(lv[q].clamp(0, s.shape[1]))
                    want[r, :u] = s[q, :u].cpu()
        assert torch.equal(o.cpu(), want)


def test_refusals():
    hd = _hd()
    mk = hd.make_beam_dims
    for bad in (mk(-1, 2, 8), mk(1, 0, 8), mk(1, 65, 8), mk(1, 2, 0), mk(1, 2, (1 << 22) + 1), mk(1, 2, 8, 2), mk(1, 2, 8, 0, -2),
                mk(1, 2, 8, ld_logits=7)):
        assert hd.stacklstm_beam_workspace_bytes(bad) == 0
    x, s = torch.randn(4, 9000, device="cuda"), torch.zeros(2, 2, device="cuda")
    r = hd.BeamRun.of(x, s)
    r.workspace = torch.empty(8, dtype=torch.uint8, device="cuda")
    with pytest.raises(hd.StackLSTMError):
        r.select()
    with pytest.raises(ValueError):
        hd.BeamRun.of(x, torch.zeros(2, 3, device="cuda")).select()
    with pytest.raises(ValueError):
        hd.BeamRun.of(x, s, done=torch.zeros(2, 2, device="cuda")).select()
    d, parent = mk(2, 2, 8), torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    a, b = torch.zeros(4, 3, device="cuda"), torch.zeros(4, 3, device="cuda")
    with pytest.raises(hd.StackLSTMError):
        hd.stacklstm_beam_reorder(d, parent, [(a, a, None)])
    with pytest.raises(hd.StackLSTMError):
        hd.stacklstm_beam_reorder(d, parent, [(a, b, None), (b, torch.zeros_like(a), None)])
    big = torch.zeros(7, 3, device="cuda")
    with pytest.raises(hd.StackLSTMError):
        hd.stacklstm_beam_reorder(d, parent, [(big[:4], big[3:], None)])
    with pytest.raises(hd.StackLSTMError):
        hd.stacklstm_beam_reorder(d, parent, [(a, b, parent.reshape(-1)), (parent.reshape(-1).clone(), parent.reshape(-1), None)])
    with pytest.raises(hd.StackLSTMError):
        hd.stacklstm_beam_reorder(d, parent, [(a, torch.zeros_like(a), None)] * 9)
    with pytest.raises(ValueError):
        hd.stacklstm_beam_reorder(d, parent, [(a[:3], b[:3], None)])
    hd.stacklstm_beam_reorder(d, parent, [])
    e = hd.BeamRun.of(torch.empty(0, 8, device="cuda"), torch.empty(0, 2, device="cuda"))
    e.select()
