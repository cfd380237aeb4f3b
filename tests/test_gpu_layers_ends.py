"""The widest rows of log probabilities and dropout."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT, get, rng_for, up
from tests.test_gpu_layers_logprob import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1 << 22, (1 << 22) - 3])
def test_widest_vocabulary(V, dtype):
    """2^22 tokens, 64 given and the 64 best; a row of equal logits, whose best are its first."""
    need_gpu()
    from paper_1904_03409_amd import layers as ly
    rng = rng_for("widest", V, dtype)
    x, token, legal, a, h = _inputs(rng, 3, V, 64, dtype)
    x[1] = 1.5
    h[:] = h / 4
    want = ref.logprob(x, token, legal, 64, a.astype(np.float64), h.astype(np.float64))
    r = ly.LogProbRun.of(up(x, dtype), up(token), up(legal), 64, up(a), up(h))
    r.step()
    _check(r, np.arange(3), want, dtype, a, h)
    r.forward(), r.backward()
    _check(r, np.arange(3), want, dtype, a, h)


def test_widest_dropout():
    """2^24 columns: a row's last groups have their own bits."""
    need_gpu()
    from paper_1904_03409_amd import layers as ly
    W, key, step = 1 << 24, 12345, 6
    seed = torch.tensor([key, step], dtype=torch.int64, device="cuda")
    for dtype in ("f32", "bf16"):
        x = torch.ones(3, W, dtype=DT[dtype], device="cuda")
        y = get(ly.DropoutRun.of(x, 0.25, seed).forward()[:, -64:] != 0)
        for r in range(3):
            for g in range(8):
                c, k, low = [W // 8 - 8 + g, r, step, 0], [key, 0], 0xFFFFFFFF
                for _ in range(10):
                    p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
                    c = [q >> 32 ^ c[1] ^ k[0], q & low, p >> 32 ^ c[3] ^ k[1], p & low]
                    k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
                bits = [b for w in c for b in (w & 0xFFFF, w >> 16)]
                assert [bool(v) for v in y[r, 8 * g:8 * g + 8]] == [b >= 16384 for b in bits], (dtype, r, g)
