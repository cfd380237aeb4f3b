"""Performance cases of the operators between the states of a StackLSTM and its answers:

* ``norm``: layer norm of state rows, after an optional residual sum; forward, or forward and
  backward with the sums over rows that are the gradients of the weight and the bias.
* ``linear``: act(x W + b) + residual; forward, or forward and backward (dx, dW, db).
* ``distill``: the loss of a student's logits against a teacher's top logits and labels, with
  the gradient of the logits in the same pass.
* ``beam``: one step of a beam search: the best continuations over beams and vocabulary, then
  the stacks of states copied to the beams that continue them.

A case holds plain values only. ``own`` chooses between the library's operators and their
plain form in elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5


def _norm(name, rows, width, dtype, res, train):
    return dict(name=name, op="norm", rows=rows, width=width, dtype=dtype, res=res, train=train)


def _linear(name, M, K, N, dtype, act, res, train):
    return dict(name=name, op="linear", M=M, K=K, N=N, dtype=dtype, act=act, res=res, train=train)


def _distill(name, rows, V, K, dtype, tau, alpha):
    return dict(name=name, op="distill", rows=rows, V=V, K=K, dtype=dtype, tau=tau, alpha=alpha)


def _beam(name, B, K, V, dtype, legal, slots, H):
    return dict(name=name, op="beam", B=B, K=K, V=V, dtype=dtype, legal=legal, slots=slots, H=H)


def listed():
    return [
        # the states on top of one sentence's eight beams, normalised between two parser steps:
        # latency is everything
        _norm("norm_beams", 8, 512, "f32", True, False),
        # training step of the paper's cell (hidden size 200) on 64 sentences, stack and buffer
        _norm("norm_paper_train", 179 * 128, 200, "f32", False, True),
        # residual sum and norm of every returned state of the large batch, 16-bit activations
        _norm("norm_large_train", 240 * 256, 1024, "bf16", True, True),
        # logits of one decoding step over a vocabulary of words: 64 beams in all, the weight is
        # read for a few rows
        _linear("linear_vocab_step", 64, 1024, 32000, "bf16", "none", False, False),
        # a parser's hidden layer in training, 32-bit, sizes that divide nothing
        _linear("linear_parser_train", 120 * 64, 500, 333, "f32", "tanh", False, True),
        # feed-forward layer over the large batch's states in 16 bits
        _linear("linear_large_train", 240 * 256, 1024, 4096, "bf16", "gelu", True, True),
        # a small parser taught by a larger one: transitions with labels
        _distill("distill_actions", 120 * 64, 83, 8, "f32", 1.0, 0.7),
        # next-word logits of a training batch against a stored teacher's 64 best
        _distill("distill_words", 4096, 32000, 64, "bf16", 2.0, 0.5),
        # a handful of rows over the largest vocabulary: fewer rows than compute units
        _distill("distill_few_rows", 16, 131071, 32, "f32", 1.5, 1.0),
        # beam parsing of 64 sentences: masked transitions, stacks of 121 slots
        _beam("beam_actions", 64, 8, 83, "f32", True, 121, 256),
        # one sentence's words searched alone: four rows over the largest vocabulary
        _beam("beam_alone", 1, 4, 131072, "f32", False, 33, 512),
        # batched search over words in 16 bits with a wide beam, recurrent states only
        _beam("beam_words", 64, 16, 64001, "bf16", False, 1, 1024),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng: random.Random):
    op = rng.choice(["norm", "linear", "distill", "beam"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "norm":
        width = _log(rng, 16, 4096)
        if rng.random() < 0.5:                   # whole multiples of 16 are as common as odd widths
            width = max(16, width // 16 * 16)
        rows = min(_log(rng, 1, 61440), 61440 * 1024 // (width * (2 if dtype == "f32" else 1)))
        c = _norm("", rows, width, dtype, rng.random() < 0.5, rng.random() < 0.6)
    elif op == "linear":
        train = rng.random() < 0.6
        K, N = _log(rng, 16, 1024), _log(rng, 16, 32000)
        if rng.random() < 0.5:
            K, N = max(16, K // 16 * 16), max(16, N // 16 * 16)
        # no more work than the largest listed case (32-bit products cost eight times as much)
        cap = 240 * 256 * 1024 * 4096 // (8 if dtype == "f32" else 1)
        M = max(1, min(_log(rng, 1, 61440), cap // (K * N)))
        act = rng.choice(["none", "relu", "tanh", "silu", "gelu"])
        if act == "relu" and train and dtype == "f32":
            act = "silu"                         # (one z rounded to the other side of 0 is a whole gradient off in 32 bits)
        c = _linear("", M, K, N, dtype, act, rng.random() < 0.5, train)
    elif op == "distill":
        V = _log(rng, 16, 131072)
        if rng.random() < 0.5:
            V = max(16, V // 16 * 16)
        rows = max(1, min(_log(rng, 1, 16384), 4096 * 32000 // (V * (2 if dtype == "f32" else 1))))
        c = _distill("", rows, V, min(V, _log(rng, 1, 64)), dtype, rng.choice([1.0, 1.5, 2.0, 4.0]),
                     rng.choice([0.3, 0.5, 0.9, 1.0]))
    else:
        V = _log(rng, 16, 131072)
        if rng.random() < 0.5:
            V = max(16, V // 16 * 16)
        K = _log(rng, 1, 16)
        B = max(1, min(_log(rng, 1, 64), 64 * 16 * 64001 // (K * V * (2 if dtype == "f32" else 1))))
        H, slots = _log(rng, 16, 1024), _log(rng, 1, 121)
        slots = max(1, min(slots, (64 * 8 * 121 * 256) // (B * K * H)))
        c = _beam("", B, K, V, dtype, rng.random() < 0.5, slots, H)
    del c["name"]
    return c


# ----------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    """Every input tensor of a case on the GPU."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(0x0E4A0000 + seed)
    t = DTYPE[case["dtype"]]
    normal = lambda *s: torch.randn(*s, generator=g, device=dev)
    rand = lambda *s: torch.rand(*s, generator=g, device=dev)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device=dev)
    s = {"case": case}
    if case["op"] == "norm":
        R, W = case["rows"], case["width"]
        # states of unit size around a row's own mean, as a stack of layers hands on
        s["x"] = (normal(R, W) + 0.5 * normal(R, 1)).to(t)
        s["res"] = normal(R, W).to(t) if case["res"] else None
        s["gamma"], s["beta"] = 1 + 0.1 * normal(W), 0.1 * normal(W)
        s["dy"] = normal(R, W).to(t) if case["train"] else None
        s["dsum"] = normal(R, W).to(t) if case["train"] and case["res"] else None
    elif case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = normal(M, K).to(t)
        s["W"] = (normal(K, N) / math.sqrt(K)).to(t)
        s["b"] = (0.1 * normal(N)).to(t)
        s["res"] = normal(M, N).to(t) if case["res"] else None
        s["dy"] = normal(M, N).to(t) if case["train"] else None
    elif case["op"] == "distill":
        R, V, K = case["rows"], case["V"], case["K"]
        s["logits"] = (2 * normal(R, V)).to(t)
        # K places of a row, all different; the teacher's values in falling order, a tail of some
        # rows not stored, one row in twenty without a teacher, one in ten without a label
        step = 1 + (rand(R, 1) * (V // K)).long().clamp(max=max(0, V // K - 1))
        s["index"] = ((ints(0, V, R, 1) + step * torch.arange(K, device=dev)) % V).int()
        s["value"] = (3 * normal(R, K)).sort(dim=1, descending=True).values
        keep = torch.arange(K, device=dev) < (1 + (1.5 * K * rand(R, 1)).long())
        keep &= rand(R, 1) > 0.05
        s["index"] = torch.where(keep, s["index"], -1)
        s["label"] = torch.where(rand(R) > 0.1, ints(0, V, R), -1).int()
        # the mean over rows; one in ten is padding
        s["grad"] = torch.where(rand(R) > 0.1, 1.0 / R, 0.0)
    else:
        B, K, V, S, H = case["B"], case["K"], case["V"], case["slots"], case["H"]
        s["logits"] = (2.5 * normal(B * K, V)).to(t)
        s["legal"] = (rand(B * K, V) < 0.5).to(torch.uint8) if case["legal"] else None
        s["score"] = -20 * rand(B, K) - 1
        s["done"] = (rand(B, K) < 0.1).to(torch.uint8)
        s["live"] = ints(1, S + 1, B * K).int()          # slots in use: the pointer and what is below it
        s["h"], s["c"] = normal(B * K, S, H), normal(B * K, S, H)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "beam":                     # the other half of a search's two sets of states
        s["h_next"], s["c_next"] = torch.zeros_like(s["h"]), torch.zeros_like(s["c"])
        s["live_next"] = torch.zeros_like(s["live"])
    if own:                                      # output buffers and work space, kept by a program from step to step
        from paper_1904_03409_amd import head
        if case["op"] == "norm":
            s["run"] = head.NormRun.of(s["x"], s["gamma"], s["beta"], res=s["res"], dy=s["dy"], dsum=s["dsum"], eps=EPS)
        elif case["op"] == "linear":
            s["run"] = head.LinearRun.of(s["x"], s["W"], s["b"], res=s["res"], act=case["act"], dy=s["dy"])
        elif case["op"] == "distill":
            s["run"] = head.DistillRun.of(s["logits"], s["index"], s["value"], label=s["label"], grad=s["grad"],
                                          tau=case["tau"], alpha=case["alpha"])
        else:
            states = [(s["h"], s["h_next"], s["live"]), (s["c"], s["c_next"], s["live"]), (s["live"], s["live_next"], None)]
            s["run"] = head.BeamRun.of(s["logits"], s["score"], s["done"], legal=s["legal"], eos=0, states=states)
    return s


# ----------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"norm": _plain_norm, "linear": _plain_linear, "distill": _plain_distill, "beam": _plain_beam}[op](s)
    r = s["run"]
    if op == "norm":
        r.forward()
        out = {"y": r.y}
        if case["res"]:
            out["sum"] = r.sum
        if case["train"]:
            r.backward()
            out.update(dx=r.dx, dgamma=r.dgamma, dbeta=r.dbeta)
    elif op == "linear":
        r.forward()
        out = {"y": r.y}
        if case["train"]:
            r.backward()
            out.update(z=r.z, dx=r.dx, dW=r.dW, db=r.db)
            if case["act"] == "none":
                del out["z"]
    elif op == "distill":
        r.step()
        out = {"loss": r.loss, "dlogits": r.dlogits}
    else:
        r.select()
        r.reorder()
        out = {"score": r.score_next, "parent": r.parent, "token": r.token, "done": r.done_next, "h": s["h_next"],
               "c": s["c_next"], "live": s["live_next"]}
    return out


def _plain_norm(s):
    case = s["case"]
    t = s["x"].dtype
    x = s["x"].float()
    if case["res"]:
        x = x + s["res"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    out = {"y": (d * rstd * s["gamma"] + s["beta"]).to(t)}
    if case["res"]:
        out["sum"] = x.to(t)
    if case["train"]:
        # the backward reads the sum as the forward wrote it
        xh = ((out["sum"].float() if case["res"] else x) - mean) * rstd
        dy = s["dy"].float()
        gy = dy * s["gamma"]
        dx = rstd * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
        if case["res"]:
            dx = dx + s["dsum"].float()
        out.update(dx=dx.to(t), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
    return out


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "tanh":
        return torch.tanh(z)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "tanh":
        a = torch.tanh(z)
        return 1 - a * a
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if act == "gelu":
        k = math.sqrt(2 / math.pi)
        a = torch.tanh(k * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + a) + 0.5 * z * (1 - a * a) * k * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain_linear(s):
    case = s["case"]
    t = s["x"].dtype
    x, W = s["x"].float(), s["W"].float()
    z = x @ W + s["b"].float()
    y = _act(z, case["act"])
    if case["res"]:
        y = y + s["res"].float()
    out = {"y": y.to(t)}
    if case["train"]:
        dz = s["dy"].float()
        if case["act"] != "none":
            out["z"] = z.to(t)                   # kept for the backward in the tensors' type
            dz = dz * _act_grad(out["z"].float(), case["act"])
        out.update(dx=(dz @ W.t()).to(t), dW=(x.t() @ dz).to(t), db=dz.sum(0).to(t))
    return out


def _distill_terms(s, f):
    """Loss and gradient of every row in the type f."""
    case = s["case"]
    tau, alpha, V = case["tau"], case["alpha"], case["V"]
    x, idx, label = s["logits"].to(f), s["index"].long(), s["label"].long()
    held = (idx >= 0) & (idx < V)
    v = torch.where(held, s["value"].to(f) / tau, -math.inf)
    some = held.any(1, keepdim=True)
    top = torch.where(some, v.max(1, keepdim=True).values, 0.0)
    e = torch.exp(v - top)
    total = torch.where(some, e.sum(1, keepdim=True), 1.0)
    p = e / total
    logp = v - top - torch.log(total)
    big = x.max(1, keepdim=True).values
    et, e1 = torch.exp((x - big) / tau), torch.exp(x - big)
    st, s1 = et.sum(1, keepdim=True), e1.sum(1, keepdim=True)
    at = idx.clamp(0, V - 1)
    logq = (x.gather(1, at) - big) / tau - torch.log(st)
    kl = torch.where(p > 0, p * (logp - logq), 0.0).sum(1)
    known = (label >= 0) & (label < V)
    lab = label.clamp(0, V - 1)[:, None]
    ce = torch.where(known, (torch.log(s1) - (x.gather(1, lab) - big))[:, 0], 0.0)
    loss = alpha * tau * tau * kl + (1 - alpha) * ce
    g = s["grad"].to(f)[:, None]
    a = torch.where(some, g * alpha * tau, 0.0)
    b = torch.where(known[:, None], g * (1 - alpha), 0.0)
    d = a / st * et + b / s1 * e1
    d.scatter_add_(1, at, -a * p)
    d.scatter_add_(1, lab, -b)
    return loss, d


def _plain_distill(s):
    loss, d = _distill_terms(s, torch.float32)
    return {"loss": loss, "dlogits": d.to(s["logits"].dtype)}


def _plain_beam(s):
    case = s["case"]
    B, K, V = case["B"], case["K"], case["V"]
    x = s["logits"].float()
    if s["legal"] is not None:
        x = torch.where(s["legal"] != 0, x, -math.inf)
    big = x.max(1, keepdim=True).values
    lse = big + torch.log(torch.exp(x - big).sum(1, keepdim=True))
    total = (x - lse) + s["score"].reshape(B * K, 1)
    # a finished beam goes on as it is, in its first place
    first = torch.arange(V, device=x.device) == 0
    kept = torch.where(first, s["score"].reshape(B * K, 1), -math.inf)
    total = torch.where(s["done"].reshape(B * K, 1) != 0, kept, total)
    total = torch.where(total.isnan(), -math.inf, total).reshape(B, K * V) + 0.0
    # whole numbers in the order (score, lower place first), all different
    bits = total.view(torch.int32).long()
    place = torch.arange(K * V, device=x.device)
    key = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF) * (1 << 32) + (0xFFFFFFFF - place)
    best = key.topk(K, dim=1).values
    at = 0xFFFFFFFF - (best & 0xFFFFFFFF)
    score = total.gather(1, at)
    none = score == -math.inf                    # fewer continuations than beams
    slot = torch.arange(K, device=x.device).expand(B, K)
    parent = torch.where(none, slot, at // V)
    was = s["done"].gather(1, parent) != 0
    token = torch.where(none | was, -1, at % V).int()
    done = (none | was | (token == 0)).to(torch.uint8)
    row = (parent + K * torch.arange(B, device=x.device)[:, None]).reshape(-1)
    live = s["live"][row]
    use = (torch.arange(case["slots"], device=x.device) < live[:, None])[:, :, None]
    return {"score": score, "parent": parent.int(), "token": token, "done": done,
            "h": torch.where(use, s["h"][row], s["h_next"]), "c": torch.where(use, s["c"][row], s["c_next"]), "live": live}


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "norm":
        n = case["rows"] * case["width"]
        nbytes = 2 * n * e + 8 * case["width"] + 8 * case["rows"]    # x, y; gamma, beta; mean, rstd
        nbytes += 2 * n * e if case["res"] else 0                    # residual, sum
        if case["train"]:
            nbytes += 2 * n * e + 8 * case["width"]                  # dy, dx; dgamma, dbeta
            nbytes += n * e if case["res"] else 0                    # dsum
        return {"bytes": nbytes, "flops": n * (18 if case["train"] else 8)}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        nbytes = (M * K + K * N + M * N + N) * e                     # x, W, y, b
        nbytes += M * N * e if case["res"] else 0
        flops = 2 * M * K * N
        if case["train"]:
            nbytes += (M * N + M * K + K * N + N) * e                # dy, dx, dW, db
            nbytes += M * N * e if case["act"] != "none" else 0      # z
            flops *= 3
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "distill":
        n = case["rows"] * case["V"]
        return {"bytes": 2 * n * e + case["rows"] * (8 * case["K"] + 12), "flops": n * 10}
    B, K, V = case["B"], case["K"], case["V"]
    nbytes = B * K * (V * e + (V if case["legal"] else 0) + 5 + 13 + 8)
    nbytes += 2 * 2 * 4 * B * K * case["H"] * (case["slots"] + 1) // 2    # h, c: the slots in use, read and written
    return {"bytes": nbytes, "flops": 4 * B * K * V}


# ----------------------------------------------------------------------------- 64-bit reference

def exact(case, seed):
    s = _inputs(case, seed)
    d = lambda k: None if s[k] is None else s[k].double()
    if case["op"] == "norm":
        x = d("x") if s["res"] is None else d("x") + d("res")
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        inv = (var + EPS).pow(-0.5)
        xh = (x - mean) * inv
        out = {"y": torch.addcmul(d("beta"), xh, d("gamma"))}
        if case["res"]:
            out["sum"] = x
        if case["train"]:
            dxh = d("dy") * d("gamma")
            n = case["width"]
            dx = (n * dxh - dxh.sum(1, keepdim=True) - xh * (dxh * xh).sum(1, keepdim=True)) * (inv / n)
            out.update(dx=dx if s["dsum"] is None else dx + d("dsum"), dgamma=torch.sum(d("dy") * xh, 0),
                       dbeta=torch.sum(d("dy"), 0))
        return out
    if case["op"] == "linear":
        x, W = d("x"), d("W")
        z = torch.addmm(d("b"), x, W).requires_grad_(case["train"])
        fn = {"none": lambda v: v * 1.0, "relu": torch.relu, "tanh": torch.tanh, "silu": torch.nn.functional.silu,
              "gelu": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[case["act"]]
        y = fn(z)
        if case["train"]:
            dz, = torch.autograd.grad(y, z, d("dy"))
        out = {"y": y.detach() if s["res"] is None else y.detach() + d("res")}
        if case["train"]:
            if case["act"] != "none":
                out["z"] = z.detach()
            out.update(dx=torch.mm(dz, W.t()), dW=torch.mm(x.t(), dz), db=dz.sum(0))
        return out
    if case["op"] == "distill":
        tau, alpha, R, V = case["tau"], case["alpha"], case["rows"], case["V"]
        x = d("logits").requires_grad_(True)
        loss = torch.zeros(R, dtype=torch.float64, device=x.device)
        idx, val = s["index"].long(), d("value")
        some = (idx >= 0).any(1).nonzero()[:, 0]
        if some.numel():
            val = val[some].masked_fill(idx[some] < 0, -math.inf)
            logp = torch.log_softmax(val / tau, 1)
            logq = torch.log_softmax(x[some] / tau, 1).gather(1, idx[some].clamp(min=0))
            term = torch.exp(logp) * (logp.masked_fill(idx[some] < 0, 0.0) - logq)
            loss = loss.index_add(0, some, alpha * tau ** 2 * term.sum(1))
        lab = s["label"].long()
        lab_rows = (lab >= 0).nonzero()[:, 0]
        if lab_rows.numel() and alpha < 1:
            ce = torch.nn.functional.cross_entropy(x[lab_rows], lab[lab_rows], reduction="none")
            loss = loss.index_add(0, lab_rows, (1 - alpha) * ce)
        if not loss.requires_grad:
            return {"loss": loss, "dlogits": torch.zeros_like(x)}
        g, = torch.autograd.grad(loss, x, d("grad"))
        return {"loss": loss.detach(), "dlogits": g}
    B, K, V = case["B"], case["K"], case["V"]
    x = d("logits")
    if s["legal"] is not None:
        x = x.masked_fill(s["legal"] == 0, -math.inf)
    total = torch.log_softmax(x, 1).reshape(B, K, V) + d("score")[:, :, None]
    done = s["done"].bool()
    total[done] = -math.inf
    total[:, :, 0] = torch.where(done, d("score"), total[:, :, 0])
    total = total.nan_to_num(nan=-math.inf, neginf=-math.inf).reshape(B, K * V)
    return {"score": total.topk(K, dim=1).values, "parent": None, "token": None, "done": None, "h": None, "c": None,
            "live": None}
