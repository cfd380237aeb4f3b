"""64-bit references of the layers around the states, written from their formulas with numpy, and bounds of what 32-bit sums
and named roundings may change; shared by the GPU tests and pinned by differences on the CPU (tests/test_layers_ref.py)."""
import numpy as np

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}    # a rounding's half step, relative to the value


def seen(B, Tq, Tk, q_len=None, k_len=None, mask=None):
    """[B, Tq, Tk]: which key each query attends to."""
    ok = np.ones((B, Tq, Tk), bool)
    if k_len is not None:
        ok &= (np.arange(Tk) < np.asarray(k_len)[:, None])[:, None, :]
    if q_len is not None:
        ok &= (np.arange(Tq) < np.asarray(q_len)[:, None])[:, :, None]
    if mask is not None:
        ok &= (np.asarray(mask) != 0)[:, None, :]
    return ok


def attend(q, k, v, ok, scale, dy=None, dtype="f32", bounds=False):
    """y, or y, dq, dk, dv, of [B, T, H, D] arrays; with bounds a second dict of how far each element may be off.

    Bounds: a dot product of D terms in 32 bits is off by 6 sqrt(D) 2^-24 of the sum of its terms' sizes (six standard deviations
    of as many independent roundings), a p by that of its x and by 16 2^-24 (its exponential, the sum and the division), a
    sum over n rows by 6 sqrt(n) 2^-24 of its terms' sizes. bf16 outputs and weights of a product are rounded once more, by at
    most 2^-8 of themselves. A backward's dy . y is that of the forward's y before its rounding, to 2^-8 / 254 of its terms; with up
    to 16 keys it is the sum of p (dy . v), whose p are not rounded."""
    B, Tq, Hq, D = q.shape
    Tk, Hk = k.shape[1:3]
    G, u, w = Hq // Hk, 2.0 ** -24, HALF[dtype]
    w_in = 0.0 if dtype == "f32" else w
    out = {"y": np.zeros(q.shape)}
    off = {"y": np.zeros(q.shape)}
    if dy is not None:
        for n, t in (("dq", q), ("dk", k), ("dv", v)):
            out[n], off[n] = np.zeros(t.shape), np.zeros(t.shape)
    s32 = lambda n: 6 * np.sqrt(max(n, 1)) * u
    for b in range(B):
        for h in range(Hq):
            c = h // G
            rows = np.nonzero(ok[b].any(1))[0]
            keys = np.nonzero(ok[b].any(0))[0]
            if len(rows) == 0:
                continue
            there = ok[b][np.ix_(rows, keys)]
            Q, K, V = q[b, rows, h], k[b, keys, c], v[b, keys, c]
            x = np.where(there, scale * (Q @ K.T), -np.inf)
            m = x.max(1, keepdims=True)
            e = np.exp(x - m)
            p = e / e.sum(1, keepdims=True)
            y = p @ V
            out["y"][b, rows, h] = y
            if bounds:
                dx = abs(scale) * s32(D) * (np.abs(Q) @ np.abs(K).T) + u * (np.abs(np.where(there, x, 0)) + np.abs(m))
                # (a p moves by its own x and by the mean move of the others)
                ep = dx + (p * dx).sum(1, keepdims=True) + 16 * u
                off["y"][b, rows, h] = (p * (ep + w_in)) @ np.abs(V) + s32(len(keys)) * (p @ np.abs(V)) + w * np.abs(y)
            if dy is None:
                continue
            g = dy[b, rows, h]
            dp = g @ V.T
            delta = (p * dp).sum(1, keepdims=True)
            ds = p * (dp - delta)
            out["dq"][b, rows, h] = scale * (ds @ K)
            out["dk"][b, keys, c] += scale * (ds.T @ Q)
            out["dv"][b, keys, c] += p.T @ g
            if bounds:
                ddp = s32(D) * (np.abs(g) @ np.abs(V).T)
                yd = (np.abs(g) * np.abs(y)).sum(1, keepdims=True)
                if Tk <= 16:
                    ddelta = (p * ((ep + s32(Tk)) * np.abs(dp) + ddp)).sum(1, keepdims=True)
                else:
                    y_off = off["y"][b, rows, h] - w * np.abs(y)
                    ddelta = (s32(D) + (w / 254 if w_in else 0)) * yd + (np.abs(g) * y_off).sum(1, keepdims=True)
                eds = np.abs(ds) * (ep + w_in + 2 * u) + p * (ddp + ddelta)
                off["dq"][b, rows, h] = abs(scale) * ((eds + s32(len(keys)) * np.abs(ds)) @ np.abs(K))
                off["dk"][b, keys, c] += abs(scale) * ((eds + s32(G * len(rows)) * np.abs(ds)).T @ np.abs(Q))
                off["dv"][b, keys, c] += (p * (ep + w_in + s32(G * len(rows)))).T @ np.abs(g)
    if bounds and dy is not None:
        for n in ("dq", "dk", "dv"):
            off[n] += w * np.abs(out[n])
    return (out, off) if bounds else out


def logprob(x, token, legal=None, N=0, dlogp=None, dent=None):
    """logp, entropy, index, value and dlogits (None without its inputs), row by row as the definition reads."""
    R, V = x.shape
    G = token.shape[1]
    logp, ent = np.zeros((R, G)), np.zeros(R)
    index, value = np.full((R, N), -1, np.int32), np.full((R, N), -np.inf)
    d = np.zeros((R, V))
    with np.errstate(all="ignore"):
        for r in range(R):
            allowed = np.ones(V, bool) if legal is None else legal[r] != 0
            z = np.where(allowed, x[r], -np.inf)
            m = np.nanmax(np.append(z, -np.inf))
            lse = m + np.log(np.exp(z - m).sum()) if m > -np.inf or np.isnan(z).any() else -np.inf
            logq = z - lse if lse > -np.inf or np.isnan(lse) else np.full(V, -np.inf)
            qv = np.exp(logq)
            ent[r] = -np.where(logq == -np.inf, 0.0, qv * logq).sum()
            for g in range(G):
                t = token[r, g]
                if 0 <= t < V:
                    logp[r, g] = logq[t] if allowed[t] else -np.inf
            best = np.nonzero(z > -np.inf)[0]
            best = best[np.argsort(-z[best], kind="stable")[:N]]
            index[r, :len(best)] = best
            value[r, :len(best)] = logq[best]
            a = np.zeros(G) if dlogp is None else dlogp[r]
            h = 0.0 if dent is None else dent[r]
            counts = [g for g in range(G) if 0 <= token[r, g] < V and allowed[token[r, g]]]
            if h == 0 and all(a[g] == 0 for g in counts):
                continue
            total = sum(a[g] for g in counts)
            d[r] = np.where(logq == -np.inf, 0.0, -qv * (total + h * (logq + ent[r])))
            for g in counts:
                d[r, token[r, g]] += a[g]
    return logp, ent, index, value, d


def keep(rows, width, p, key, step, period=0):
    """Which elements dropout keeps and their factor, word by word as Philox4x32-10 is defined, in Python's whole numbers."""
    cut = int(np.floor(np.float64(np.float32(p)) * 65536 + 0.5))
    out = np.zeros((rows, width), bool)
    low = 0xFFFFFFFF
    for r in range(min(rows, period) if period else rows):
        for g in range((width + 7) // 8):
            c, k = [g, r, step & low, step >> 32 & low], [key & low, key >> 32 & low]
            for _ in range(10):
                a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                c = [b >> 32 ^ c[1] ^ k[0], b & low, a >> 32 ^ c[3] ^ k[1], a & low]
                k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
            bits = [h for word in c for h in (word & 0xFFFF, word >> 16)]
            for i in range(min(8, width - 8 * g)):
                out[r, 8 * g + i] = bits[i] >= cut
    if period:
        out = out[np.arange(rows) % period]
    return out, (65536 / (65536 - cut) if cut < 65536 else 0.0)
