"""The layers around the states together with the operators behind them: a training step of a parser that looks at its sentence's
words, captured and replayed; its gradients against differences; streams."""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import need_gpu
from tests.head_gpu import get

pytestmark = pytest.mark.gpu


class Step:
    """states attend to words, dropout and a residual sum, norm, output layer, rewards with an entropy bonus; and backward."""

    def __init__(self, dtype, T=17, B=6, words=23, H=2, D=20, V=70, p=0.25, seed=1):
        from paper_1904_03409_amd import head as hd
        from paper_1904_03409_amd import layers as ly
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        W = H * D
        self.h_top, self.enc, self.val = rand(T, B, W).to(dtype), rand(words, B, W).to(dtype), rand(words, B, W).to(dtype)
        heads = lambda t: t.view(t.shape[0], B, H, D).transpose(0, 1)
        self.q_len = torch.randint(1, T + 1, (B,), generator=g, device="cuda").int()
        self.k_len = torch.randint(1, words + 1, (B,), generator=g, device="cuda").int()
        self.att = ly.AttendRun.of(heads(self.h_top), heads(self.enc), heads(self.val), self.q_len, self.k_len, train=True)
        self.seed = torch.tensor([seed, 5], dtype=torch.int64, device="cuda")
        rows = lambda t: t.transpose(0, 1).reshape(T * B, W)
        assert rows(self.att.y).data_ptr() == self.att.y.data_ptr()          # (steps first, as the states are)
        self.drop = ly.DropoutRun.of(rows(self.att.y), p, self.seed, self.h_top.view(T * B, W), period=B, train=True)
        self.norm = hd.NormRun.of(self.drop.y, 1 + 0.1 * rand(W), 0.1 * rand(W), train=True)
        self.Wo, self.bo = (rand(W, V) / W ** 0.5).to(dtype), (0.1 * rand(V)).to(dtype)
        self.out = hd.LinearRun.of(self.norm.y, self.Wo, self.bo, train=True)
        token = torch.randint(0, V, (T * B, 1), generator=g, device="cuda").int()
        asked = (torch.arange(T, device="cuda")[:, None] < self.q_len).reshape(-1)
        self.a = torch.where(asked, rand(T * B), 0.0)[:, None].contiguous() / T
        self.h = torch.where(asked, 0.1 / T, 0.0)
        self.lp = ly.LogProbRun.of(self.out.y, token, top=4, dlogp=self.a, dentropy=self.h)

    def forward(self):
        for r in (self.att, self.drop, self.norm, self.out):
            r.forward()
        self.lp.forward()

    def __call__(self):
        for r in (self.att, self.drop, self.norm, self.out):
            r.forward()
        self.lp.step()
        self.out.dy = self.lp.dlogits
        self.out.backward()
        self.norm.dy = self.out.dx
        self.norm.backward()
        self.drop.dy = self.norm.dx
        self.drop.backward()
        T, B, W = self.h_top.shape
        self.att.dy = self.drop.dx.view(T, B, *self.att.q.shape[2:]).transpose(0, 1)
        self.att.backward()
        self.dh_top = self.att.dq.transpose(0, 1).reshape(T, B, W) + self.norm.dx.view(T, B, W)

    def outputs(self):
        return [t.clone() for t in (self.att.y, self.drop.y, self.lp.logp, self.lp.entropy, self.lp.index, self.lp.value, self.lp.dlogits,
                                    self.att.dq, self.att.dk, self.att.dv, self.drop.dx, self.out.dW, self.norm.dgamma, self.dh_top)]

    def value(self):
        self.forward()
        return (get(self.lp.logp) * get(self.a)).sum() + (get(self.lp.entropy) * get(self.h)).sum()


def test_gradients_are_differences():
    """Of the states, the words and their values, through every layer."""
    need_gpu()
    s = Step(torch.float32)
    s()
    step, size = 2.0 ** -7, np.abs(get(s.lp.logp) * get(s.a)).sum() + np.abs(get(s.lp.entropy) * get(s.h)).sum()
    grads = {"h_top": get(s.dh_top), "enc": get(s.att.dk.transpose(0, 1)), "val": get(s.att.dv.transpose(0, 1))}
    rng = np.random.default_rng(3)
    for n, g in grads.items():
        t = getattr(s, n)
        u = rng.standard_normal(t.shape)
        move, was = torch.from_numpy(u).float().cuda(), t.clone()
        d = g.reshape(u.shape) * u
        t.copy_(was + step * move)
        hi = s.value()
        t.copy_(was - step * move)
        lo = s.value()
        t.copy_(was)
        # third derivatives: step^2 of a term's size (through a softmax, a norm and another softmax: 40); fp32's rounding over the step
        assert abs((hi - lo) / (2 * step) - d.sum()) <= 40 * step * step * np.abs(d).sum() + 2e-6 / step * size, n


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_graph_replays(dtype):
    """A captured step, replayed between eager work and with other inputs, lengths and seeds, gives the eager bits each time; an
    eager run of the same buffers lives beside it."""
    need_gpu()
    s = Step(dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s()
    replayed = s.dh_top
    for i in range(4):
        s.h_top.copy_(torch.randn(s.h_top.shape, device="cuda"))
        s.q_len.copy_(torch.randint(0, 18, (6,), device="cuda"))
        s.k_len.copy_(torch.randint(0, 24, (6,), device="cuda"))
        s.seed[1] += 1
        s()
        want = s.outputs()
        for t in (s.att.y, s.drop.y, s.lp.logp, s.lp.value, s.lp.dlogits, s.att.dq, s.att.dk, s.att.dv, s.drop.dx, s.out.dW):
            t.fill_(7)
        s.att.workspace.fill_(255)
        torch.cuda.synchronize()
        s.dh_top = replayed
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, s.outputs())), i


def test_streams():
    """Two steps at once on two streams, each with buffers of its own, give the bits of one alone."""
    need_gpu()
    steps = [Step(torch.bfloat16, T=60, B=20, words=300, seed=i) for i in (1, 2)]
    want = []
    for s in steps:
        s()
        want.append(s.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(3):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(p, q) for p, q in zip(w, s.outputs()))


def test_beams_of_a_sentence_share_its_words():
    """A decoding step: the beams of a sentence are the queries of one call; each beam alone gives the same within its rounding."""
    need_gpu()
    from paper_1904_03409_amd import layers as ly
    B, K, T, H, D = 3, 5, 900, 4, 32
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(B, n, H, D, generator=g, device="cuda") for n in (K, T, T))
    k_len = torch.tensor([900, 1, 333], dtype=torch.int32, device="cuda")
    y = ly.AttendRun.of(q, k, v, k_len=k_len).forward()
    for b in range(K):
        one = ly.AttendRun.of(q[:, b:b + 1], k, v, k_len=k_len).forward()
        assert float((one - y[:, b:b + 1]).abs().max()) < 1e-5
