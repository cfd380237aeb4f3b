"""Beam selection on the GPU, every search of a batch: parents and tokens wherever 32-bit rounding cannot order two continuations
either way, and all of them where they can."""
import numpy as np
import pytest

from tests.gpu_helpers import need_gpu
from tests.head_gpu import TOL32, rng_for, rounded, up

pytestmark = pytest.mark.gpu


def _ordered(x, legal, score, done):
    """Continuations of one search in order, as far as some past the K-th: totals, parents, tokens (-1: a finished beam's)."""
    K, V = x.shape
    total = np.full((K, V), -np.inf, np.float32)
    with np.errstate(all="ignore"):
        for k in range(K):
            if done is not None and done[k]:
                total[k, 0] = score[k]
                continue
            v = x[k].astype(np.float32) if legal is None else np.where(legal[k] != 0, x[k], -np.inf).astype(np.float32)
            w = v.astype(np.float64)
            lse = np.float32(w.max() + np.log(np.exp(w - w.max()).sum()))
            total[k] = (v - lse) + score[k]
    flat = np.where(total > -np.inf, total, -np.inf).reshape(-1)
    n = min(K, int((flat > -np.inf).sum()))
    if n == 0:
        return np.zeros(0, np.float32), np.zeros(0, int), np.zeros(0, int)
    kth = np.partition(flat, flat.size - n)[flat.size - n]
    at = np.nonzero((flat >= kth - 1e-4 * max(1, abs(kth))) & (flat > -np.inf))[0]
    at = at[np.lexsort((at, -flat[at].astype(np.float64)))]
    parent = at // V
    token = np.where(done[parent] != 0, -1, at % V) if done is not None else at % V
    return flat[at], parent, token


# greedy decoding and single tokens; more searches than a few; a workgroup, whole rows, chunks
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (2, 1, 7), (70, 1, 2000), (40, 3, 17), (300, 1, 9000), (1, 1, 131072), (40, 7, 5003), (130, 2, 33000),
                                   (9, 4, 65600), (3, 64, 3000)])
def test_every_search(B, K, V, dtype):
    need_gpu()
    from paper_1904_03409_amd import head as hd
    rng = rng_for("every", B, K, V, dtype)
    x = rounded(2.5 * rng.standard_normal((B * K, V)), dtype)
    score = (-20 * rng.random((B, K)) - 1).astype(np.float32)
    done = (rng.random((B, K)) < 0.15).astype(np.uint8) if (B + V) % 2 else None
    legal = (rng.random((B * K, V)) < 0.6).astype(np.uint8) if V % 3 else None
    run = hd.BeamRun.of(up(x, dtype), up(score), None if done is None else up(done), None if legal is None else up(legal), 1)
    run.select()
    got = [t.cpu().numpy() for t in (run.score_next, run.parent, run.token, run.done_next)]
    seen = 0
    for b in range(B):
        rows = slice(b * K, b * K + K)
        total, parent, token = _ordered(x[rows], None if legal is None else legal[rows], score[b], None if done is None else done[b])
        n = min(K, len(total))
        assert (np.abs(got[0][b, :n] - total[:n]) <= TOL32 * np.maximum(1, np.abs(total[:n]))).all()
        # runs of totals that rounding cannot tell apart; one is in order where it is one beam's equal logits
        cut = np.nonzero(np.abs(np.diff(total)) > 4e-6 * np.maximum(1, np.abs(total[1:])))[0] + 1
        for g in np.split(np.arange(len(total)), cut):
            if len(g) > 1 and (len(set(parent[g])) > 1 or len(set(total[g])) > 1):
                continue
            g = g[g < n]
            seen += len(g)
            assert np.array_equal(got[1][b, g], parent[g]) and np.array_equal(got[2][b, g], token[g])
            assert np.array_equal(got[3][b, g], (token[g] == -1) | (token[g] == 1))
        assert (got[0][b, n:] == -np.inf).all() and np.array_equal(got[1][b, n:], np.arange(n, K)) and (got[2][b, n:] == -1).all()
        assert got[3][b, n:].all()
    assert seen >= 0.9 * min(K, 8) * B * (V > 1)
