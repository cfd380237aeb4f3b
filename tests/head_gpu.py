"""Helpers of the GPU tests of the operators behind the recurrence."""
import numpy as np
import torch

DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# Error of a 32-bit result, against the largest of its tensor: the framework's bar for fp32 outputs.
TOL32 = 1e-5
# One rounding to 8 significant bits, of the value itself.
ULP16 = 2.0 ** -8


def rng_for(*key):
    """A generator of a test's own, the same in every run."""
    return np.random.default_rng(sum((i + 1) * ord(c) for i, c in enumerate("/".join(str(k) for k in key))))


def rounded(a, dtype):
    """a as it is after rounding to the type, in 64 bits."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]).double().numpy()


def up(a, dtype=None):
    """a on the GPU in the type."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t.to(DT[dtype]) if dtype else t).to(DEV)


def strided(a, dtype, pad):
    """The same as a view of a wider matrix whose rows start `pad` columns in (NaN around it)."""
    big = torch.full((a.shape[0], a.shape[1] + pad + 3), float("nan"), dtype=DT[dtype], device=DEV)
    v = big[:, pad:pad + a.shape[1]]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]))
    return v


def get(t):
    return t.detach().double().cpu().numpy()


def close(got, want, dtype, what, extra=0.0):
    """Errors within the type's bound, plus `extra` where a named rounding adds to it; infinities and NaN alike."""
    got, want = get(got) if isinstance(got, torch.Tensor) else got, np.asarray(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN elsewhere"
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf]), f"{what}: infinities elsewhere"
    fine = np.isfinite(want)
    if not fine.any():
        return
    bound = TOL32 * np.abs(want[fine]).max() + np.broadcast_to(extra, want.shape)[fine]
    if dtype == "bf16":
        bound = bound + ULP16 * np.abs(want[fine])
    err = np.abs(got[fine] - want[fine])
    worst = np.argmax(err - bound)
    assert (err <= bound).all(), f"{what}: {err[worst]} at value {want[fine][worst]} (bound {np.broadcast_to(bound, err.shape)[worst]})"
