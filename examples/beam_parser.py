"""A small transition parser on the library's own operators: trained by distillation, run by beam search.

The states of a StackLSTM (the stack of an arc-standard parser) go through layer norm, a hidden layer with a residual and an
output layer to scores of the transitions: shift, or an arc with one of a few labels that pops the stack. A larger parser
with random weights stands for the teacher; only its best few scores of every state are kept. The student is trained
on them and on the transitions of the streams. Then sentences are parsed by beam search: every beam has its own stack of states,
copied when a beam is continued twice, and one cell step computes the pushed state of every beam.

    python examples/beam_parser.py [--steps 40] [--beams 4] [--dtype f32|bf16]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1904_03409_amd import head as hd  # noqa: E402
from paper_1904_03409_amd import stacklstm as sl  # noqa: E402
from paper_1904_03409_amd import workloads as wk  # noqa: E402

LABELS = 5
ACTIONS = 1 + 2 * LABELS                         # shift, left arcs, right arcs
SHIFT = 0


class Parser:
    """Parameters: the cell (fp32, as the library's StackLSTM has them) and what follows it in `dtype`."""

    def __init__(self, inputs, hidden, dtype, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.I, self.H, self.dtype = inputs, hidden, dtype
        self.W, self.U, self.b = 0.2 * rand(inputs, 4 * hidden), 0.1 * rand(hidden, 4 * hidden), torch.zeros(4 * hidden, device="cuda")
        self.gamma, self.beta = torch.ones(hidden, device="cuda"), torch.zeros(hidden, device="cuda")
        # 32-bit masters of the layers; the products take them in dtype
        self.W1, self.b1 = rand(hidden, hidden) / hidden ** 0.5, torch.zeros(hidden, device="cuda")
        self.W2, self.b2 = rand(hidden, ACTIONS) / hidden ** 0.5, torch.zeros(ACTIONS, device="cuda")

    def layers(self, states, train):
        """norm, hidden layer with residual, output layer over rows of states; their buffers are kept by the caller."""
        t = lambda p: p.to(self.dtype)
        norm = hd.NormRun.of(states.to(self.dtype), self.gamma, self.beta, train=train)
        hidden = hd.LinearRun.of(norm.y, t(self.W1), t(self.b1), res=norm.y, act="tanh", train=train)
        out = hd.LinearRun.of(hidden.y, t(self.W2), t(self.b2), train=train)
        return norm, hidden, out

    def scores(self, states):
        runs = self.layers(states, False)
        for r in runs:
            r.forward()
        return runs[-1].y


def streams(words, rng):
    """Arc-standard streams of sentences of `words` words: ops [T, B] (+1 shift, -1 arc, 0 behind the end) and actions."""
    ops = [wk.ops_arc_standard_stream(rng, int(n)) for n in words]
    T = max(len(o) for o in ops)
    op = np.zeros((T, len(ops)), np.int8)
    act = np.full((T, len(ops)), -1, np.int32)
    for j, o in enumerate(ops):
        op[: len(o), j] = o
        act[: len(o), j] = np.where(o == 1, SHIFT, rng.integers(1, ACTIONS, len(o)))
    return op, act


def cell_inputs(op, sentences):
    """x [T, B, I]: the word that a shift brings, zeros elsewhere."""
    x = torch.zeros(*op.shape, sentences.shape[2], device="cuda")
    for j in range(op.shape[1]):
        at = np.nonzero(op[:, j] == 1)[0]
        x[torch.from_numpy(at).cuda(), j] = sentences[j, : len(at)]
    return x


def run_cell(p, op, x):
    """The StackLSTM over whole streams, with the buffers of a training step."""
    T, B = op.shape
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")
    dims = sl.make_dims(T, B, p.I, p.H)
    z = torch.zeros(B, p.H, device="cuda")
    return sl.DeviceRun(dims=dims, x=x, ops=torch.from_numpy(op).cuda(), W=p.W, U=p.U, b=p.b, h0=z, c0=z.clone(), dh_top=None,
                        dc_top=None, h_cell=e(T, B, p.H), c_cell=e(T, B, p.H), h_top=e(T, B, p.H), c_top=e(T, B, p.H),
                        ptr=e(T + 1, B, dtype=torch.int32), top=e(T, B, dtype=torch.int32),
                        workspace=e(sl.stacklstm_workspace_bytes(dims), dtype=torch.uint8), dx=e(T, B, p.I),
                        dW=e(p.I, 4 * p.H), dU=e(p.H, 4 * p.H), db=e(4 * p.H), dh0=e(B, p.H), dc0=e(B, p.H))


def train(student, teacher, op, act, sentences, steps, top=6, rate=0.5):
    """Distillation steps on one batch of streams; returns the mean loss of every step."""
    T, B = op.shape
    x = cell_inputs(op, sentences)
    # the teacher's best scores of every state, kept as they would be in a file
    tr = run_cell(teacher, op, x)
    tr.forward()
    value, index = teacher.scores(tr.h_top.reshape(T * B, -1)).float().topk(top, dim=1)
    value, index = value.contiguous(), index.int().contiguous()
    # the state after step t answers for the action of step t + 1; behind a sentence's end nothing is asked
    label = torch.from_numpy(np.concatenate([act[1:], np.full((1, B), -1, np.int32)]).reshape(-1)).cuda()
    asked = label >= 0
    index[~asked] = -1
    grad = asked.float() / asked.sum()
    run = run_cell(student, op, x)
    losses = []
    for _ in range(steps):
        run.forward()
        norm, hidden, out = student.layers(run.h_top.reshape(T * B, -1), True)
        for r in (norm, hidden, out):
            r.forward()
        loss = hd.DistillRun.of(out.y, index, value, label, grad, tau=2.0, alpha=0.5)
        losses.append((loss.step() * grad).sum())
        out.dy = loss.dlogits
        out.backward()
        hidden.dy = out.dx
        hidden.backward()
        norm.dy = hidden.dx + out.dx             # through the hidden layer and past it
        norm.backward()
        run.dh_top = norm.dx.float().reshape(T, B, -1)
        run.backward()
        for w, d in ((student.W, run.dW), (student.U, run.dU), (student.b, run.db), (student.gamma, norm.dgamma),
                     (student.beta, norm.dbeta), (student.W1, hidden.dW), (student.b1, hidden.db), (student.W2, out.dW),
                     (student.b2, out.db)):
            w -= rate * d.float()
    return [float(v) for v in losses]


def legal_actions(shifted, depth, words):
    """uint8 [rows, ACTIONS]: shift while words are left, arcs on two stack items."""
    m = torch.zeros(len(words), ACTIONS, dtype=torch.uint8, device="cuda")
    m[:, SHIFT] = shifted < words
    m[:, 1:] = (depth >= 2)[:, None]
    return m


def search(p, sentences, words, K):
    """Beam search over the transitions: scores [B, K], actions [B, K, T] (-1 behind a sentence's end)."""
    B, most, I = sentences.shape
    rows, H = B * K, p.H
    words_r = torch.as_tensor(words, device="cuda").repeat_interleave(K)
    # slot 0 of a stack is the initial state; two sets of states, one read and one written by a step's copies
    zeros = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    i32 = torch.int32
    sets = [[zeros(rows, most + 1, H), zeros(rows, most + 1, H), zeros(rows, dtype=i32) + 1, zeros(rows, dtype=i32)] for _ in range(2)]
    score = torch.full((B, K), -float("inf"), device="cuda")
    score[:, 0] = 0                              # the other beams are not there yet
    done = torch.zeros(B, K, dtype=torch.uint8, device="cuda")
    dims = sl.make_dims(1, rows, I, H)
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")
    h_new, c_new, ptr, top = e(1, rows, H), e(1, rows, H), e(2, rows, dtype=torch.int32), e(1, rows, dtype=torch.int32)
    push = torch.ones(1, rows, dtype=torch.int8, device="cuda")
    at = torch.arange(rows, device="cuda")
    sentence = at // K
    T = 2 * max(words) - 1
    history = torch.full((rows, T), -1, dtype=torch.int32, device="cuda")
    for step in range(T):
        (h, c, live, shifted), nxt = sets
        depth = live - 1                         # live: slots in use, the initial state's among them
        logits = p.scores(h[at, depth.long()])
        legal = legal_actions(shifted, depth, words_r)
        states = [(h, nxt[0], live), (c, nxt[1], live), (live, nxt[2], None), (shifted, nxt[3], None)]
        old = history.clone()
        run = hd.BeamRun.of(logits, score, done, legal=legal, states=states + [(old, history, None)])
        run.select()
        run.reorder()
        sets.reverse()
        h, c, live, shifted = sets[0]
        score, token = run.score_next, run.token.reshape(-1)
        history[:, step] = token
        # every beam's pushed state in one cell step; beams that popped keep theirs
        top_at = (live - 1).long()
        x = sentences[sentence, shifted.long().clamp(max=most - 1)][None].contiguous()
        sl.stacklstm_fwd_static(dims, x, push, p.W, p.U, p.b, h[at, top_at], c[at, top_at], h_new, c_new, None, None, ptr, top)
        shift = token == SHIFT
        r, s = at[shift], live[shift].long()
        h[r, s], c[r, s] = h_new[0, r], c_new[0, r]
        live += torch.where(shift, 1, torch.where(token > 0, -1, 0)).int()
        shifted += shift.int()
        # a parse is complete with one item on the stack and no word left
        over = (live == 2) & (shifted == words_r) & (token >= 0)
        done = torch.where(over.reshape(B, K), 1, run.done_next).to(torch.uint8)
    return score, history.reshape(B, K, T)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    t = torch.float32 if a.dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(7)
    words = rng.integers(3, 13, 24)
    op, act = streams(words, rng)
    sentences = torch.randn(len(words), int(words.max()), 32, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    student, teacher = Parser(32, 64, t, 1), Parser(32, 128, t, 2)
    losses = train(student, teacher, op, act, sentences, a.steps)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} over {a.steps} steps")
    score, history = search(student, sentences, [int(w) for w in words], a.beams)
    for j in range(3):
        names = ["shift" if v == SHIFT else f"{'left' if v <= LABELS else 'right'}-{(v - 1) % LABELS}" for v in history[j, 0].tolist() if v >= 0]
        print(f"sentence {j} ({words[j]} words): log p {float(score[j, 0]):.3f}: {' '.join(names)}")


if __name__ == "__main__":
    main()
