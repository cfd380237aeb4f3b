"""64-bit references of the operators behind the recurrence, written from their formulas with numpy; shared by
the GPU tests and pinned by differences on the CPU (tests/test_head_ref.py)."""
import numpy as np


def norm_fwd(x, res, gamma, beta, eps):
    s = x if res is None else x + res
    mu = s.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((s - mu) ** 2).mean(1, keepdims=True) + eps)
    y = (s - mu) * rstd
    y = y * (1 if gamma is None else gamma) + (0 if beta is None else beta)
    return s, y, mu[:, 0], rstd[:, 0]


def norm_bwd(s, mu, rstd, gamma, dy, dsum):
    xh = (s - mu[:, None]) * rstd[:, None]
    g = dy * (1 if gamma is None else gamma)
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx + (0 if dsum is None else dsum), (dy * xh).sum(0), dy.sum(0)


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0)
    if name == "tanh":
        return np.tanh(z)
    if name == "silu":
        return z / (1 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).astype(z.dtype)
    if name == "tanh":
        return 1 - np.tanh(z) ** 2
    if name == "silu":
        q = 1 / (1 + np.exp(-z))
        return q + z * q * (1 - q)
    if name == "gelu":
        k = np.sqrt(2 / np.pi)
        a = np.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + a) + 0.5 * z * (1 - a * a) * k * (1 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def distill(x, index, value, label, grad, tau, alpha):
    """Loss and gradient, row by row as the definition reads."""
    R, V = x.shape
    loss, d = np.zeros(R), np.zeros((R, V))
    with np.errstate(all="ignore"):
        for r in range(R):
            def softmax(v):
                e = np.exp(v - v.max())
                return e / e.sum()
            there = [j for j in range(index.shape[1]) if 0 <= index[r, j] < V]
            if there and not all(value[r, j] == -np.inf for j in there):
                v = value[r, there] / tau
                p, q = softmax(v), softmax(x[r] / tau)
                lq = x[r] / tau - (x[r].max() / tau + np.log(np.exp((x[r] - x[r].max()) / tau).sum()))
                t = np.zeros(V)
                for pj, j in zip(p, there):
                    if pj != 0:
                        loss[r] += alpha * tau ** 2 * pj * (np.log(pj) - lq[index[r, j]])
                    t[index[r, j]] += pj
                if grad[r] != 0 and alpha != 0:
                    d[r] += grad[r] * alpha * tau * (q - t)
            if label is not None and 0 <= label[r] < V and alpha < 1:
                lse = x[r].max() + np.log(np.exp(x[r] - x[r].max()).sum())
                loss[r] += (1 - alpha) * (lse - x[r, label[r]])
                if grad[r] != 0:
                    t = np.zeros(V)
                    t[label[r]] = 1
                    d[r] += grad[r] * (1 - alpha) * (softmax(x[r]) - t)
    return loss, d


def beam(x, legal, score, done, eos, lse=None):
    """score_next, parent, token, done_next of one step, from the list of all continuations. x [B K, V] and
    score in the type the totals are added in; lse: per row, by default from x in 64 bits."""
    B, K = score.shape
    V = x.shape[1]
    f = score.dtype.type
    out = [np.full((B, K), -np.inf, score.dtype), np.tile(np.arange(K, dtype=np.int32), (B, 1)),
           np.full((B, K), -1, np.int32), np.ones((B, K), np.uint8)]
    with np.errstate(all="ignore"):
        for b in range(B):
            found = []
            for k in range(K):
                r = b * K + k
                if done is not None and done[b, k]:
                    if score[b, k] > -np.inf:
                        found.append((-score[b, k], k * V, k, -1))
                    continue
                v = x[r] if legal is None else np.where(legal[r] != 0, x[r], f(-np.inf))
                if lse is None:
                    w = v.astype(np.float64)
                    one = f(w.max() + np.log(np.exp(w - w.max()).sum()))
                else:
                    one = f(lse[r])
                total = (v - one) + score[b, k]
                there = np.nonzero(total > -np.inf)[0]
                for t in there[np.argsort(-total[there], kind="stable")[:K]]:      # (no beam gives more than K)
                    found.append((-total[t], k * V + t, k, t))
            found.sort()
            for n, (neg, place, k, t) in enumerate(found[:K]):
                out[0][b, n], out[1][b, n], out[2][b, n] = -neg, k, t
                out[3][b, n] = t == -1 or t == eos
    return out
