"""Log probabilities of tokens at -inf in rows that hold NaN or +inf."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import close, up

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [70, 3000, 70001])
def test_tokens_at_minus_infinity(V):
    """NaN where the row has NaN or +inf (alone or among numbers), else -inf; a token that is not allowed is at -inf in any row."""
    need_gpu()
    from paper_1904_03409_amd import layers as ly
    rng = np.random.default_rng(V)
    x, legal = rng.standard_normal((6, V)), np.ones((6, V), np.uint8)
    x[:, 5] = -np.inf
    x[1, 11], x[2, 11] = np.nan, np.inf
    x[3], x[4] = -np.inf, -np.inf
    x[4, V - 1] = np.nan
    legal[:, 6], legal[5, 11], x[5, 11] = 0, 0, np.nan                       # (row 5: its NaN is not allowed)
    token = np.tile(np.array([5, 6, 7, -1], np.int32), (6, 1))
    want = ref.logprob(x, token, legal)
    assert np.isnan(want[0][[1, 2, 4], 0]).all() and (want[0][[0, 3, 5], 0] == -np.inf).all() and (want[0][:, 1] == -np.inf).all()
    r = ly.LogProbRun.of(up(x, "f32"), up(token), up(legal), dlogp=torch.zeros(6, 4, device="cuda"))
    r.forward()
    close(r.logp, want[0], "f32", "logp")
    r.logp.fill_(7)
    r.step()
    close(r.logp, want[0], "f32", "logp of a step")
