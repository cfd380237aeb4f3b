"""The references of the layers around the states, pinned by differences and by published values (no GPU needed)."""
import numpy as np

from tests import layers_ref as ref


def test_attention_gradients_are_differences():
    rng = np.random.default_rng(1)
    B, Tq, Tk, Hq, Hk, D = 2, 3, 5, 4, 2, 6
    t = {"q": rng.standard_normal((B, Tq, Hq, D)), "k": rng.standard_normal((B, Tk, Hk, D)), "v": rng.standard_normal((B, Tk, Hk, D))}
    dy = rng.standard_normal((B, Tq, Hq, D))
    ok = ref.seen(B, Tq, Tk, [3, 2], [5, 3], rng.random((B, Tk)) < 0.7)
    out = ref.attend(**t, ok=ok, scale=0.7, dy=dy)
    for n in t:
        dirn = rng.standard_normal(t[n].shape)
        f = lambda s: (ref.attend(**{**t, n: t[n] + s * dirn}, ok=ok, scale=0.7)["y"] * dy).sum()
        num = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(num - (out["d" + n] * dirn).sum()) < 1e-7 * (1 + abs(num))


def test_logprob_gradient_is_differences():
    rng = np.random.default_rng(2)
    R, V, G = 6, 9, 3
    x = rng.standard_normal((R, V))
    token = rng.integers(-1, V + 1, (R, G))
    token[0] = 4
    legal = rng.random((R, V)) < 0.7
    legal[:, 4] = True
    a, h = rng.standard_normal((R, G)), rng.standard_normal(R)
    logp, ent, _, _, d = ref.logprob(x, token, legal, 2, a, h)
    dirn = rng.standard_normal(x.shape)
    barred = logp == -np.inf
    f = lambda s: sum((np.where(barred, 0, w) * o).sum() for o, w in
                      zip((np.where(barred, 0, v) for v in ref.logprob(x + s * dirn, token, legal)[:1]), (a,))) + \
        (ref.logprob(x + s * dirn, token, legal)[1] * h).sum()
    num = (f(1e-5) - f(-1e-5)) / 2e-5
    assert abs(num - (d * dirn).sum()) < 1e-7 * (1 + abs(num))
    assert np.abs(np.exp(ref.logprob(x, np.tile(np.arange(V), (R, 1)))[0]).sum(1) - 1).max() < 1e-12


def test_generator():
    """Known answers published with Philox4x32-10: of counter and key 0, and of all bits set."""
    def words(c, k):
        low = 0xFFFFFFFF
        for _ in range(10):
            a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [b >> 32 ^ c[1] ^ k[0], b & low, a >> 32 ^ c[3] ^ k[1], a & low]
            k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
        return c
    assert words([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert words([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    k, _ = ref.keep(1, 8, 0.5, 0, 0)
    bits = [h for w in (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8) for h in (w & 0xFFFF, w >> 16)]
    assert k[0].tolist() == [b >= 32768 for b in bits]
    k, s = ref.keep(40, 100, 0.25, 7, 9, 10)
    assert (k[:10] == k[10:20]).all() and abs(k[:10].mean() - 0.75) < 0.07 and abs(s - 4 / 3) < 1e-12
