"""Forms of the attention kernels that only certain sizes reach, and calls at the ends of what is allowed."""
import pytest
import torch

from tests.gpu_helpers import need_gpu
from tests.head_gpu import DT

pytestmark = pytest.mark.gpu


def _ly():
    need_gpu()
    from paper_1904_03409_amd import layers
    return layers


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_up_to_31_bits(dtype):
    """2^31 - 2 queries of heads that share one key, a row tile short of 2^31; of one key y is its value."""
    ly = _ly()
    Tq, Hq = ((1 << 31) - 2) // 151, 151
    assert Tq * Hq == (1 << 31) - 2
    print(f"[gpu] {dtype} {Tq} queries, {Hq} heads", flush=True)
    q = torch.randn(1, 1, Hq, 1, device="cuda").to(DT[dtype]).expand(1, Tq, Hq, 1)
    k, v = (torch.randn(1, 1, 1, 1, device="cuda").to(DT[dtype]) for _ in range(2))
    y = torch.full((1, Tq, Hq, 1), 7.0, dtype=DT[dtype], device="cuda")
    ly.AttendRun.of(q, k, v, y=y).forward()
    low, high = y.aminmax()
    assert low == v.squeeze() and high == v.squeeze()
    del y
    torch.cuda.empty_cache()
