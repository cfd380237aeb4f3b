"""Performance cases of the layers around the states of a StackLSTM:

* ``attend``: states attend to an encoder's states of another length (heads, keys and values shared by several heads,
  lengths, masked keys); forward, or forward and backward.
* ``logprob``: log probabilities of given tokens, the entropy and the best tokens of rows of logits; or the same with the
  gradient of the logits, where the outputs' gradients are known beforehand.
* ``dropout``: x kept or dropped by a counter-based generator, scaled, added to a residual; forward, or forward and backward.

A case holds plain values only. ``own`` chooses between the library's operators and their
plain form in elementary torch operations in 32 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _attend(name, B, Tq, Tk, Hq, Hk, D, dtype, lens, mask, steps_first, train):
    return dict(name=name, op="attend", B=B, Tq=Tq, Tk=Tk, Hq=Hq, Hk=Hk, D=D, dtype=dtype, lens=lens, mask=mask,
                steps_first=steps_first, train=train)


def _logprob(name, rows, V, G, N, dtype, legal, train):
    return dict(name=name, op="logprob", rows=rows, V=V, G=G, N=N, dtype=dtype, legal=legal, train=train)


def _dropout(name, rows, width, dtype, p, res, period, train):
    return dict(name=name, op="dropout", rows=rows, width=width, dtype=dtype, p=p, res=res, period=period, train=train)


def listed():
    return [
        # one parser state looks at the words of its sentence between two steps: latency is everything
        _attend("attend_one_token", 1, 1, 60, 8, 8, 32, "f32", False, False, False, False),
        # eight beams of eight documents over long encoder states, four heads to a key: the keys' and values' bytes
        _attend("attend_beams_long", 8, 8, 16384, 16, 4, 128, "bf16", True, False, False, False),
        # training step of the paper's cell (hidden size 200) on 64 sentences of up to 60 words, 32 bits, widths that divide nothing
        _attend("attend_parser_train", 64, 119, 60, 4, 4, 50, "f32", True, True, True, True),
        # the large batch's states (hidden size 512) over its words, 16-bit
        _attend("attend_large_train", 256, 240, 120, 8, 8, 64, "bf16", True, False, True, True),
        # whole documents in training: thousands of states over thousands of words, matrix products
        _attend("attend_long_train", 2, 4096, 4000, 16, 4, 128, "bf16", True, False, False, True),
        # the transitions of 64 sentences' eight beams scored, the best eight kept
        _logprob("logprob_actions", 64 * 8, 83, 1, 8, "f32", True, False),
        # rewards with an entropy bonus over a vocabulary of words, with the logits' gradient
        _logprob("logprob_words_train", 4096, 32000, 1, 0, "bf16", False, True),
        # a teacher's 64 best words of every row, to be kept on disk
        _logprob("logprob_teacher", 1024, 64001, 1, 64, "bf16", False, False),
        # a handful of rows over the largest vocabulary: fewer rows than compute units
        _logprob("logprob_few_rows", 4, 131071, 3, 10, "f32", False, False),
        # the paper's cell (hidden size 200) over 64 sentences, between stacked layers
        _dropout("dropout_parser_train", 120 * 64, 200, "f32", 0.3, False, 0, True),
        # one mask for all steps of a sentence (recurrent layers), 32-bit
        _dropout("dropout_steps", 240 * 256, 512, "f32", 0.2, False, 256, False),
        # every returned state of the large batch before its residual sum, 16-bit activations
        _dropout("dropout_large_train", 240 * 256, 1024, "bf16", 0.1, True, 0, True),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng: random.Random):
    op = rng.choice(["attend", "attend", "logprob", "dropout"])
    dtype = rng.choice(["f32", "bf16"])
    train = rng.random() < 0.6
    if op == "attend":
        D = _log(rng, 16, 256)
        if rng.random() < 0.6:                   # whole multiples of 16 are more common than odd widths
            D = max(16, D // 16 * 16)
        Hk = rng.choice([1, 2, 3, 4, 8])
        Hq = Hk * rng.choice([1, 1, 2, 4])
        Tq = _log(rng, 1, 4096)
        Tk = _log(rng, 1, 16384)
        # no more pairs, and no more products, than the largest listed case (32-bit products cost sixteen times as much)
        pairs = min(2 * 16 * 4096 * 4000, 2 * 16 * 4096 * 4000 * 128 // (D * (16 if dtype == "f32" else 1)))
        Tk = max(1, min(Tk, pairs // (Tq * Hq)))
        # ... nor more bytes
        B = max(1, min(_log(rng, 1, 256), pairs // (Tq * Tk * Hq), (1 << 27) // (max(Tq * Hq, Tk * Hk) * D)))
        c = _attend("", B, Tq, Tk, Hq, Hk, D, dtype, rng.random() < 0.7, rng.random() < 0.3, rng.random() < 0.5, train)
    elif op == "logprob":
        V = _log(rng, 16, 131072)
        if rng.random() < 0.5:
            V = max(16, V // 16 * 16)
        rows = max(1, min(_log(rng, 1, 16384), 4096 * 32000 // (V * (2 if dtype == "f32" else 1))))
        c = _logprob("", rows, V, rng.randint(1, 4), rng.choice([0, min(V, _log(rng, 1, 64))]), dtype, rng.random() < 0.3, train)
    else:
        width = _log(rng, 16, 4096)
        if rng.random() < 0.5:
            width = max(16, width // 16 * 16)
        rows = min(_log(rng, 1, 61440), 61440 * 1024 // (width * (2 if dtype == "f32" else 1)))
        period = rng.choice([0, 0, _log(rng, 1, rows)])
        c = _dropout("", rows, width, dtype, rng.choice([0.1, 0.2, 0.3, 0.5]), rng.random() < 0.5, period, train)
    del c["name"]
    return c


# ----------------------------------------------------------------------------- inputs

def _lengths(n, longest, ragged):
    """Lengths of n sequences, between half of the longest and all of it."""
    return [longest - (i * (longest // 2)) // n if ragged else longest for i in range(n)]


def _inputs(case, seed):
    """Every input tensor of a case on the GPU."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(0x1A7E0000 + seed)
    t = DTYPE[case["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=g, device=dev)
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)
    s = {"case": case}
    if case["op"] == "attend":
        B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "D"))
        # a StackLSTM returns [steps, sentences, hidden]: its heads are a view of that
        def states(T, H):
            if case["steps_first"]:
                return normal(T, B, H, D).to(t).transpose(0, 1)
            return normal(B, T, H, D).to(t)
        s["q"], s["k"], s["v"] = states(Tq, Hq), states(Tk, Hk), states(Tk, Hk)
        s["dy"] = states(Tq, Hq) if case["train"] else None
        order = torch.randperm(B, generator=g, device=dev)
        lens = lambda longest: torch.tensor(_lengths(B, longest, True), dtype=torch.int32, device=dev)[order].contiguous()
        s["k_len"] = lens(Tk) if case["lens"] else None
        # a parser takes about two steps to a word
        s["q_len"] = lens(Tq) if case["lens"] and case["train"] else None
        # words that are not attended to (punctuation)
        s["mask"] = (rand(B, Tk) > 0.15).to(torch.uint8) if case["mask"] else None
    elif case["op"] == "logprob":
        R, V, G = case["rows"], case["V"], case["G"]
        s["logits"] = (2 * normal(R, V)).to(t)
        s["token"] = torch.randint(0, V, (R, G), generator=g, device=dev).int()
        s["token"] = torch.where(rand(R, G) < 0.1, -1, s["token"])           # padding
        s["legal"] = (rand(R, V) < 0.5).to(torch.uint8) if case["legal"] else None
        if case["legal"]:                        # what was chosen was allowed
            s["legal"].scatter_(1, s["token"].clamp(min=0).long(), 1)
        # advantages and the weight of the entropy's mean
        s["dlogp"] = normal(R, G) / R if case["train"] else None
        s["dentropy"] = torch.full((R,), 0.01 / R, device=dev) if case["train"] else None
    else:
        R, W = case["rows"], case["width"]
        s["x"] = normal(R, W).to(t)
        s["res"] = normal(R, W).to(t) if case["res"] else None
        s["dy"] = normal(R, W).to(t) if case["train"] else None
        # the generator's key and the step of training
        s["seed"] = torch.tensor([0x5DEECE66D * (seed + 1) & 0x7FFFFFFFFFFF, 1000 + seed], dtype=torch.int64, device=dev)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                      # output buffers and work space, kept by a program from step to step
        from paper_1904_03409_amd import layers
        if case["op"] == "attend":
            s["run"] = layers.AttendRun.of(s["q"], s["k"], s["v"], q_len=s["q_len"], k_len=s["k_len"], mask=s["mask"], dy=s["dy"])
        elif case["op"] == "logprob":
            s["run"] = layers.LogProbRun.of(s["logits"], s["token"], legal=s["legal"], top=case["N"], dlogp=s["dlogp"],
                                            dentropy=s["dentropy"])
        else:
            s["run"] = layers.DropoutRun.of(s["x"], case["p"], s["seed"], res=s["res"], period=case["period"], dy=s["dy"])
    return s


# ----------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"attend": _plain_attend, "logprob": _plain_logprob, "dropout": _plain_dropout}[op](s)
    r = s["run"]
    if op == "attend":
        r.forward()
        out = {"y": r.y}
        if case["train"]:
            r.backward()
            out.update(dq=r.dq, dk=r.dk, dv=r.dv)
    elif op == "logprob":
        if case["train"]:
            r.step()
        else:
            r.forward()
        out = {"logp": r.logp, "entropy": r.entropy}
        if case["N"]:
            out.update(index=r.index, value=r.value)
        if case["train"]:
            out["dlogits"] = r.dlogits
    else:
        r.forward()
        out = {"y": r.y}
        if case["train"]:
            r.backward()
            out["dx"] = r.dx
    return out


def _seen(s, dev):
    """Which key each query attends to: [B, Tq, Tk]."""
    case = s["case"]
    ok = torch.ones(case["B"], case["Tq"], case["Tk"], dtype=torch.bool, device=dev)
    if s["k_len"] is not None:
        ok &= (torch.arange(case["Tk"], device=dev) < s["k_len"][:, None])[:, None, :]
    if s["q_len"] is not None:
        ok &= (torch.arange(case["Tq"], device=dev) < s["q_len"][:, None])[:, :, None]
    if s["mask"] is not None:
        ok &= (s["mask"] != 0)[:, None, :]
    return ok


def _plain_attend(s):
    case = s["case"]
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "D"))
    t, G, scale = s["q"].dtype, Hq // Hk, 1 / math.sqrt(D)
    # [B Hk, G Tq, D] and [B Hk, Tk, D]: the queries that share a key's head side by side
    queries = lambda x: x.float().reshape(B, Tq, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(B * Hk, G * Tq, D)
    keys = lambda x: x.float().permute(0, 2, 1, 3).reshape(B * Hk, Tk, D)
    q, k, v = queries(s["q"]), keys(s["k"]), keys(s["v"])
    ok = _seen(s, q.device)[:, None, None].expand(B, Hk, G, Tq, Tk).reshape(B * Hk, G * Tq, Tk)
    x = torch.where(ok, torch.bmm(q, k.transpose(1, 2)) * scale, -math.inf)
    m = x.max(2, keepdim=True).values
    x = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = x.sum(2, keepdim=True)
    p = x / torch.where(total == 0, 1.0, total)
    del x
    back = lambda x: x.reshape(B, Hk, G, Tq, D).permute(0, 3, 1, 2, 4).reshape(B, Tq, Hq, D).to(t)
    back_keys = lambda x: x.reshape(B, Hk, Tk, D).permute(0, 2, 1, 3).to(t)
    out = {"y": back(torch.bmm(p, v))}
    if case["train"]:
        dy = queries(s["dy"])
        out["dv"] = back_keys(torch.bmm(p.transpose(1, 2), dy))
        dp = torch.bmm(dy, v.transpose(1, 2))
        ds = p * (dp - (p * dp).sum(2, keepdim=True)) * scale
        del dp, p
        out["dq"] = back(torch.bmm(ds, k))
        out["dk"] = back_keys(torch.bmm(ds.transpose(1, 2), q))
    return out


def _plain_logprob(s):
    case = s["case"]
    R, V, N = case["rows"], case["V"], case["N"]
    x = s["logits"].float()
    if s["legal"] is not None:
        x = torch.where(s["legal"] != 0, x, -math.inf)
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    logs = torch.log(total)
    there = s["token"] >= 0
    at = s["token"].clamp(min=0).long()
    out = {"logp": torch.where(there, (x.gather(1, at) - m) - logs, 0.0)}
    far = torch.where(e > 0, x - m, 0.0)
    ent = logs - (e * far).sum(1, keepdim=True) / total
    out["entropy"] = ent[:, 0]
    if N:
        # whole numbers in the order (logit, lower place first), all different
        bits = (x + 0.0).view(torch.int32).long()
        place = torch.arange(V, device=x.device)
        key = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF) * (1 << 32) + (0xFFFFFFFF - place)
        best = key.topk(N, dim=1).values
        at_best = 0xFFFFFFFF - (best & 0xFFFFFFFF)
        value = (x.gather(1, at_best) - m) - logs
        none = value == -math.inf                # fewer tokens than places
        out["index"] = torch.where(none, -1, at_best).int()
        out["value"] = value
    if case["train"]:
        q = e / total
        a = torch.where(there, s["dlogp"], 0.0)
        d = -q * (a.sum(1, keepdim=True) + s["dentropy"][:, None] * ((far - logs) + ent))
        d.scatter_add_(1, at, a)
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _philox(counter, key, rounds=10):
    """The counter-based generator Philox4x32 (Salmon et al., 2011): four words of 32 bits from four of a counter and two of a
    key, all in 64-bit tensors."""
    low = 0xFFFFFFFF

    def multiply(a, b):                          # the halves of a 64-bit product, from pieces that 63 bits hold
        p0, p1 = a * (b & 0xFFFF), a * (b >> 16)
        return (p1 + (p0 >> 16)) >> 16, (p0 + ((p1 & 0xFFFF) << 16)) & low

    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(rounds):
        h0, l0 = multiply(0xD2511F53, c0)
        h1, l1 = multiply(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _plain_dropout(s):
    case = s["case"]
    R, W, period = case["rows"], case["width"], case["period"]
    t, dev = s["x"].dtype, s["x"].device
    cut = int(math.floor(case["p"] * 65536 + 0.5))
    scale = 65536 / max(1, 65536 - cut)
    # eight elements of a row to a counter (group of eight, row, step), 16 bits to an element
    n = (W + 7) // 8
    row = torch.arange(min(R, period) if period else R, device=dev)[:, None]
    group = torch.arange(n, device=dev)[None, :]
    low = 0xFFFFFFFF
    zero = torch.zeros_like(row * group)
    key, step = s["seed"][0], s["seed"][1]
    words = _philox((zero + group, zero + row, zero + (step & low), zero + ((step >> 32) & low)), (key & low, (key >> 32) & low))
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=2)
    keep = (halves.reshape(-1, 8 * n)[:, :W] >= cut)
    if period:
        keep = keep[torch.arange(R, device=dev) % period]
    y = torch.where(keep, s["x"].float() * scale, 0.0)
    out = {"y": (y if s["res"] is None else y + s["res"].float()).to(t)}
    if case["train"]:
        out["dx"] = torch.where(keep, s["dy"].float() * scale, 0.0).to(t)
    return out


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "attend":
        B, Hq, Hk, D = case["B"], case["Hq"], case["Hk"], case["D"]
        lk = _lengths(B, case["Tk"], case["lens"])
        lq = _lengths(B, case["Tq"], case["lens"] and case["train"])
        # (both in one order: the longest parses are those of the longest sentences)
        pairs = sum(a * b for a, b in zip(lq, lk)) * Hq
        rows_q, rows_k = sum(lq) * Hq * D * e, sum(lk) * Hk * D * e
        every = (B * case["Tq"] * Hq * D * e, B * case["Tk"] * Hk * D * e)   # outputs are written whole
        nbytes = rows_q + 2 * rows_k + every[0] + (B * case["Tk"] if case["mask"] else 0)
        flops = 4 * D * pairs
        if case["train"]:
            nbytes += rows_q + every[0] + 2 * every[1]                       # dy; dq, dk, dv
            flops += 10 * D * pairs
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "logprob":
        n = case["rows"] * case["V"]
        nbytes = n * e * (2 if case["train"] else 1) + (n if case["legal"] else 0)
        nbytes += case["rows"] * (8 * case["G"] + 4 + 8 * case["N"] + (4 * case["G"] + 4 if case["train"] else 0))
        return {"bytes": nbytes, "flops": n * (12 if case["train"] else 6)}
    n = case["rows"] * case["width"]
    return {"bytes": n * e * (2 + (1 if case["res"] else 0) + (2 if case["train"] else 0)), "flops": n * (3 if case["train"] else 2)}


# ----------------------------------------------------------------------------- 64-bit reference

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    if case["op"] == "logprob":
        return _exact_logprob(s)
    return _exact_dropout(s)


def _exact_attend(s):
    """Sentence by sentence on the keys and queries that are there, gradients by differentiation."""
    case = s["case"]
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "D"))
    dev, G = s["q"].device, Hq // Hk
    zeros = lambda T, H: torch.zeros(B, T, H, D, dtype=torch.float64, device=dev)
    out = {"y": zeros(Tq, Hq)}
    if case["train"]:
        out.update(dq=zeros(Tq, Hq), dk=zeros(Tk, Hk), dv=zeros(Tk, Hk))
    k_len = [Tk] * B if s["k_len"] is None else s["k_len"].tolist()
    q_len = [Tq] * B if s["q_len"] is None else s["q_len"].tolist()
    for b in range(B):
        n = q_len[b]
        at = torch.arange(k_len[b], device=dev)
        if s["mask"] is not None:
            at = at[s["mask"][b, :k_len[b]].bool()]
        if at.numel() == 0:
            continue
        for h in range(Hk):
            heads = slice(h * G, (h + 1) * G)
            leaf = lambda x: x.double().detach().requires_grad_(case["train"])
            q, k, v = leaf(s["q"][b, :n, heads]), leaf(s["k"][b, at, h]), leaf(s["v"][b, at, h])
            rows = q.reshape(n * G, D)
            y = torch.mm(torch.softmax(torch.mm(rows, k.t()) / D ** 0.5, 1), v).reshape(n, G, D)
            out["y"][b, :n, heads] = y.detach()
            if case["train"]:
                dq, dk, dv = torch.autograd.grad(y, (q, k, v), s["dy"][b, :n, heads].double())
                out["dq"][b, :n, heads] = dq
                out["dk"][b, at, h], out["dv"][b, at, h] = dk, dv
    return out


def _exact_logprob(s):
    case = s["case"]
    x = s["logits"].double().requires_grad_(case["train"])
    masked = x if s["legal"] is None else x.masked_fill(s["legal"] == 0, -math.inf)
    lse = torch.logsumexp(masked, 1, keepdim=True)
    there = s["token"] >= 0
    at = s["token"].clamp(min=0).long()
    logp = (masked.gather(1, at) - lse).masked_fill(~there, 0.0)
    q = torch.exp(masked - lse)
    entropy = -(q * (x - lse)).sum(1)            # (x itself: a token that is not allowed has q = 0)
    out = {"logp": logp.detach(), "entropy": entropy.detach()}
    if case["N"]:
        top = (masked - lse).detach().topk(case["N"], dim=1).values
        out.update(index=None, value=top)
    if case["train"]:
        out["dlogits"], = torch.autograd.grad([logp, entropy], x, [s["dlogp"].double(), s["dentropy"].double()])
    return out


def _exact_dropout(s):
    case = s["case"]
    R, W, period = case["rows"], case["width"], case["period"]
    key, step = (int(v) for v in s["seed"].tolist())
    u64 = np.uint64
    rows, n, low = min(R, period) if period else R, -(-W // 8), u64(0xFFFFFFFF)
    ctr = np.empty((4, rows * n), u64)
    ctr[0], ctr[1] = np.tile(np.arange(n, dtype=u64), rows), np.repeat(np.arange(rows, dtype=u64), n)
    ctr[2], ctr[3] = step & 0xFFFFFFFF, step >> 32 & 0xFFFFFFFF
    k = [key & 0xFFFFFFFF, key >> 32 & 0xFFFFFFFF]
    for i in range(10):
        a, b = ctr[0] * u64(0xD2511F53), ctr[2] * u64(0xCD9E8D57)            # (64 bits hold the products)
        k0, k1 = u64((k[0] + i * 0x9E3779B9) & 0xFFFFFFFF), u64((k[1] + i * 0xBB67AE85) & 0xFFFFFFFF)
        ctr = np.stack([(b >> u64(32)) ^ ctr[1] ^ k0, b & low, (a >> u64(32)) ^ ctr[3] ^ k1, a & low])
    half = np.ascontiguousarray(ctr.astype(np.uint32).T).view(np.uint16).reshape(rows, 8 * n)[:, :W]
    dropped = round(case["p"] * 65536)
    factor = torch.from_numpy(np.where(half < dropped, 0.0, 1 / (1 - dropped / 65536))).to(s["x"].device)
    if period:
        factor = factor.repeat((R + period - 1) // period, 1)[:R]
    out = {"y": s["x"].double() * factor}
    if case["res"]:
        out["y"] += s["res"].double()
    if case["train"]:
        out["dx"] = s["dy"].double() * factor
    return out
