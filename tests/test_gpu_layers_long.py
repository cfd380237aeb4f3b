"""Attention in 32 bits over thousands of keys or queries: the error of its sums in the mean square."""
import numpy as np
import pytest
import torch

from tests import layers_ref as ref
from tests.gpu_helpers import need_gpu
from tests.head_gpu import get

pytestmark = pytest.mark.gpu

# The mean square error of a rounding in fp32, relative to the value: uniform in half a step (1 / sqrt 3), a step that is between 2^-24
# and 2^-25 of the value (sqrt(3 / 8 / ln 2) over mantissas that are spread evenly over their logarithm).
ROUND = 2.0 ** -24 * 3 ** -0.5 * (3 / 8 / np.log(2)) ** 0.5


def bound(n, D):
    """Of a sum over n rows of random signs, taken 16 at a time: two chains of roundings (each sqrt(length / 2) of one); three
    products over the width of a head in each term (score, dy . v, dy . y) likewise; a term's exponential of a score up to 8 from the reference
    (8 ln 2 roundings), its own two and those of the softmax's sum. Half as much again for what is not independent."""
    terms = 3 * D / 2 + (8 * np.log(2)) ** 2 + 8
    return 1.5 * ROUND * (n / 16 / 2 + 16 / 2 + terms) ** 0.5


# long keys for y and dq, long queries for dk and dv (up to 128 keys of heads up to 64 in a kernel of their own); every width of the kernels,
# whole vectors or not; as many heads as keep the work unsplit; one row tile, whose waves share the keys
SIZES = [(512, 16384, 64, 30), (512, 16384, 64, 48), (512, 16384, 64, 50), (512, 16384, 64, 128), (512, 16384, 64, 200), (512, 16384, 64, 250), (3, 16384, 256, 64),
         (2, 16384, 256, 132), (16384, 512, 64, 32), (16384, 512, 64, 50), (16384, 512, 64, 100), (16384, 512, 64, 101), (16384, 512, 64, 256), (16384, 512, 64, 201), (16384, 100, 256, 48),
         (16384, 60, 256, 50), (16384, 128, 256, 32)]


@pytest.mark.parametrize("Tq,Tk,H,D", SIZES)
def test_long_sums_in_32_bits(Tq, Tk, H, D):
    need_gpu()
    from paper_1904_03409_amd import layers as ly
    g = torch.Generator(device="cuda").manual_seed(Tq + Tk + D)
    rand = lambda T: torch.randn(1, T, H, D, generator=g, device="cuda")
    q, k, v, dy = rand(Tq), rand(Tk), rand(Tk), rand(Tq)
    r = ly.AttendRun.of(q, k, v, dy=dy)
    assert H * max(1, Tq // 128) >= 256 or H * max(1, Tk // 128) >= 256
    r.forward(), r.backward()
    for h in (0, H - 1):
        one = lambda t: get(t[:, :, h:h + 1].contiguous())
        want = ref.attend(*map(one, (q, k, v)), ref.seen(1, Tq, Tk), D ** -0.5, one(dy))
        for n in ("y", "dq", "dk", "dv"):
            got, w = one(getattr(r, n)), want[n]
            off = np.linalg.norm(got - w) / np.linalg.norm(w)
            print(f"[gpu] {Tq} x {Tk} x {D} head {h} {n}: {off:.3g}", flush=True)
            assert off <= bound(Tk if n in ("y", "dq") else Tq, D), n
    torch.cuda.empty_cache()
