"""The operators together: the example parser is trained, its searches' scores are those of its parses scored whole; graphs."""
import os
import sys

import numpy as np
import pytest
import torch

from tests.gpu_helpers import need_gpu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _setup(dtype, words):
    import beam_parser as bp
    sentences = torch.randn(len(words), max(words), 16, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    return bp, sentences, bp.Parser(16, 40, dtype, 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_lowers_the_loss(dtype):
    need_gpu()
    words = [3, 7, 5, 9]
    bp, sentences, student = _setup(dtype, words)
    rng = np.random.default_rng(4)
    op, act = bp.streams(words, rng)
    losses = bp.train(student, bp.Parser(16, 72, dtype, 6), op, act, sentences, 25)
    assert np.isfinite(losses).all() and losses[-1] < 0.8 * losses[0], losses


@pytest.mark.parametrize("K", [1, 3, 8])
def test_search_scores_are_those_of_its_parses(K):
    """Every beam's actions, run as one stream through the whole StackLSTM and scored in 64 bits from its states, give the
    score that the search carried along; beams are ordered and differ; one beam is the greedy parse."""
    need_gpu()
    words = [1, 2, 4, 8]
    bp, sentences, p = _setup(torch.float32, words)
    score, history = bp.search(p, sentences, words, K)
    B, T = len(words), history.shape[2]
    s = score.cpu().numpy()
    for j, n in enumerate(words):
        alive = [k for k in range(K) if s[j, k] > -np.inf]
        assert alive and (np.diff(s[j, alive]) <= 0).all()
        assert len({tuple(history[j, k].tolist()) for k in alive}) == len(alive)
        for k in alive:
            acts = [v for v in history[j, k].tolist() if v >= 0]
            assert len(acts) == 2 * n - 1 and acts.count(bp.SHIFT) == n
            op = np.array([1 if v == bp.SHIFT else -1 for v in acts], np.int8)[:, None]
            run = bp.run_cell(p, op, bp.cell_inputs(op, sentences[j:j + 1]))
            run.forward()
            states = torch.cat([torch.zeros(1, p.H, device="cuda"), run.h_top[:-1, 0]]).double()
            mean = states.mean(1, keepdim=True)
            y = (states - mean) / torch.sqrt(((states - mean) ** 2).mean(1, keepdim=True) + 1e-5) * p.gamma.double() + p.beta.double()
            y = torch.tanh(y @ p.W1.double() + p.b1.double()) + y
            logits = y @ p.W2.double() + p.b2.double()
            depth, shifted, total = 0, 0, 0.0
            for t, v in enumerate(acts):
                legal = torch.zeros(bp.ACTIONS, dtype=torch.bool, device="cuda")
                legal[bp.SHIFT] = shifted < n
                legal[1:] = depth >= 2
                assert legal[v]
                lp = torch.log_softmax(logits[t].masked_fill(~legal, -float("inf")), 0)
                if K == 1:
                    assert float(lp.max() - lp[v]) < 1e-4
                total += float(lp[v])
                depth += 1 if v == bp.SHIFT else -1
                shifted += v == bp.SHIFT
            # fp32 states and sums over at most 15 steps
            assert abs(total - s[j, k]) < 1e-4 * (1 + abs(total)), (j, k, total, s[j, k])


def test_command_line(monkeypatch, capsys):
    need_gpu()
    import beam_parser as bp
    monkeypatch.setattr(sys, "argv", ["beam_parser.py", "--steps", "5", "--dtype", "bf16"])
    bp.main()
    out = capsys.readouterr().out
    assert "loss" in out and "sentence 2" in out


def test_graph_replays():
    """A captured step of every operator, replayed between eager work, gives the eager bits each time."""
    need_gpu()
    from paper_1904_03409_amd import head as hd
    g = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, W, b = rand(700, 100), rand(100, 3000) / 10, rand(3000)
    norm = hd.NormRun.of(x, rand(100), rand(100), train=True)
    lin = hd.LinearRun.of(norm.y, W, b, act="silu", train=True)
    dis = hd.DistillRun.of(lin.y, torch.randint(0, 3000, (700, 9), generator=g, device="cuda").int(), rand(700, 9), tau=2.0)
    K = 4
    few = rand(K, 70000)
    src, dst = rand(K, 5, 33), torch.zeros(K, 5, 33, device="cuda")
    beam = hd.BeamRun.of(few, -torch.rand(1, K, generator=g, device="cuda"), states=[(src, dst, None)])

    def step():
        norm.forward()
        lin.forward()
        dis.step()
        lin.dy = dis.dlogits
        lin.backward()
        norm.dy = lin.dx
        norm.backward()
        beam.select()
        beam.reorder()

    outs = lambda: [t.clone() for t in (norm.y, lin.y, dis.loss, dis.dlogits, lin.dW, lin.db, norm.dx, norm.dgamma, beam.score_next,
                                        beam.parent, beam.token, dst)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(rand(700, 100))
        few.copy_(rand(K, 70000))
        step()
        want = outs()
        for t in (norm.y, lin.y, dis.loss, dis.dlogits, lin.dW, norm.dx, norm.dgamma, beam.score_next, dst):
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, outs())), i
