"""Calls of more threads than one launch may have (a grid of 2^32 threads and more is refused by HIP)."""
import pytest
import torch

from tests.gpu_helpers import need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _hd():
    need_gpu()
    from paper_1904_03409_amd import head
    return head


def test_norm_of_many_narrow_rows():
    hd = _hd()
    R = (1 << 29) + 70
    x = torch.arange(R, device="cuda", dtype=torch.int32).remainder_(8191).float()[:, None]
    y, mean, rstd = torch.full((R, 1), 7.0, device="cuda"), torch.full((R,), 7.0, device="cuda"), torch.full((R,), 7.0, device="cuda")
    hd.stacklstm_norm_fwd(hd.make_norm_dims(R, 1), x, None, None, None, None, y, mean, rstd)
    assert torch.equal(mean, x[:, 0]) and not y.any()
    assert rstd.min() == rstd.max()
