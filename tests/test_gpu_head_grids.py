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


def test_distill_of_many_narrow_rows():
    hd = _hd()
    R, V = (1 << 29) + 70, 2
    x = torch.arange(R * V, device="cuda", dtype=torch.int32).remainder_(61).to(torch.bfloat16).view(R, V)
    index = torch.full((R, 1), -1, dtype=torch.int32, device="cuda")
    value, label = torch.zeros(R, 1, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    loss = torch.full((R,), 7e9, device="cuda")
    d = torch.full((R, V), 7.0, dtype=torch.bfloat16, device="cuda")
    dims = hd.make_distill_dims(R, V, 1, hd.SLSTM_BF16, 1.0, 0.0)
    ws = torch.empty(hd.stacklstm_distill_workspace_bytes(dims), dtype=torch.uint8, device="cuda")
    hd.stacklstm_distill_step(dims, x, index, value, label, None, loss, d, ws)
    worst, off = 0.0, 0.0
    for lo in range(0, R, 1 << 26):                      # log(1 + exp(x1 - x0)) and its derivative, a piece at a time
        p = x[lo:lo + (1 << 26)].float()
        gap = p[:, 1] - p[:, 0]
        worst = max(worst, float((loss[lo:lo + (1 << 26)] - torch.logaddexp(gap, torch.zeros_like(gap))).abs().max()))
        off = max(off, float((d[lo:lo + (1 << 26), 1].float() - torch.sigmoid(gap)).abs().max()))
    assert worst < 60 * 1e-5 and off < 2.0 ** -8


def test_distill_of_many_long_rows():
    """Rows in chunks, in place: every row is one base row, shifted."""
    hd = _hd()
    R, V = 233100, 32772
    base = torch.randn(V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    x = base + torch.arange(R, device="cuda").remainder_(4).float()[:, None]
    label = torch.arange(R, device="cuda", dtype=torch.int32).remainder_(V)
    index, value = torch.full((R, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(R, 1, device="cuda")
    loss = torch.full((R,), 7e9, device="cuda")
    dims = hd.make_distill_dims(R, V, 1, hd.SLSTM_F32, 1.0, 0.0)
    ws = torch.empty(hd.stacklstm_distill_workspace_bytes(dims), dtype=torch.uint8, device="cuda")
    hd.stacklstm_distill_step(dims, x, index, value, label, None, loss, x, ws)
    want = torch.logsumexp(base.double(), 0) - base.double()
    assert float((loss - want[label.long()]).abs().max()) < 1e-5 * float(want.max())
    q = torch.softmax(base.double(), 0)
    for lo in (0, 116500, 232950, R - 90):
        d = q.repeat(90, 1)
        d[torch.arange(90, device="cuda"), label[lo:lo + 90].long()] -= 1
        assert float((x[lo:lo + 90] - d).abs().max()) < 1e-5


def test_beam_of_many_searches():
    hd = _hd()
    B, V = (1 << 23) + 9, 3
    x = torch.arange(B * V, device="cuda", dtype=torch.int32).remainder_(1009).float().view(B, V)
    r = hd.BeamRun.of(x, torch.zeros(B, 1, device="cuda"))
    r.parent.fill_(7), r.token.fill_(7), r.score_next.fill_(7)
    r.select()
    assert torch.equal(r.token[:, 0], x.argmax(1).int()) and not r.parent.any()
    for lo in (0, 1 << 21, (1 << 22) - 500, B - 1000):  # searches need nothing of each other: fewer of them give the same bits
        few = hd.BeamRun.of(x[lo:lo + 1000], torch.zeros(1000, 1, device="cuda"))
        few.select()
        assert torch.equal(r.score_next[lo:lo + 1000], few.score_next)


def test_beam_of_many_rows():
    hd = _hd()
    K, V = 64, 129
    B = (1 << 18) + 3
    # beams further down score less, and a row's best token is its own number: search b goes on with beam 0's best tokens
    row = torch.arange(B * K, device="cuda", dtype=torch.int32)
    x = torch.zeros(B * K, V, dtype=torch.bfloat16, device="cuda")
    at = (row % V).long()
    for lo in range(0, B * K, 1 << 22):
        x[torch.arange(lo, min(B * K, lo + (1 << 22)), device="cuda"), at[lo:lo + (1 << 22)]] = 50.0
    score = (-100.0 * torch.arange(K, device="cuda", dtype=torch.float32)).repeat(B, 1)
    r = hd.BeamRun.of(x, score)
    r.parent.fill_(7), r.token.fill_(7), r.score_next.fill_(7)
    r.select()
    best = at.view(B, K)[:, 0].int()
    assert not r.parent.any() and torch.equal(r.token[:, 0], best)
    # then the lowest tokens but that one
    lowest = torch.arange(K - 1, device="cuda", dtype=torch.int32).repeat(B, 1)
    assert torch.equal(r.token[:, 1:], lowest + (lowest >= best[:, None]).int())
    assert float(r.score_next[:, 0].abs().max()) < 1e-5


@pytest.mark.parametrize("width", [1, 300])
def test_reorder_of_many_rows(width):
    hd = _hd()
    K = 64
    B = ((1 << 28) + (1 << 8)) // K if width == 1 else ((1 << 24) + (1 << 8)) // K
    n = B * K
    src = torch.arange(n, device="cuda", dtype=torch.int32).remainder_(251).to(torch.uint8)[:, None]
    src = src + torch.arange(width, device="cuda").to(torch.uint8)
    dst = torch.full_like(src, 255)
    parent = torch.arange(n, device="cuda", dtype=torch.int32).mul_(7).add_(5).remainder_(K).view(B, K)
    other, copy = torch.arange(n, device="cuda", dtype=torch.int32), torch.full((n,), -1, dtype=torch.int32, device="cuda")
    hd.stacklstm_beam_reorder(hd.make_beam_dims(B, K, 1), parent, [(src, dst, None), (other, copy, None)])
    frm = parent.view(-1) + torch.arange(B, device="cuda", dtype=torch.int32).mul_(K).repeat_interleave(K)
    assert torch.equal(copy, frm)
    for lo in range(0, n, 1 << 24):
        assert torch.equal(dst[lo:lo + (1 << 24)], src[frm[lo:lo + (1 << 24)].long()])


@pytest.mark.parametrize("N", [1, 2])
def test_linear_of_many_rows(N):
    """2^24 tiles of one column, odd rows (copied) and whole ones."""
    hd = _hd()
    M, K = 1 << 30, 1 if N == 1 else 8
    x = torch.arange(M, device="cuda", dtype=torch.int32).remainder_(253).to(torch.bfloat16)[:, None]
    if K > 1:
        x = x.repeat(1, K)
    W = torch.zeros(K, N, dtype=torch.bfloat16, device="cuda")
    W[0] = 1.0
    y = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    d = hd.make_linear_dims(M, K, N, hd.SLSTM_BF16)
    ws = torch.empty(hd.stacklstm_linear_fwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    hd.stacklstm_linear_fwd(d, x, W, None, None, y, None, ws)
    assert all(torch.equal(y[:, n], x[:, 0]) for n in range(N))
    if N == 1:
        dx = torch.full((M, K), 7.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(hd.stacklstm_linear_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        hd.stacklstm_linear_bwd(d, x, W, None, x, dx, None, None, ws)
        assert torch.equal(dx, x)


@pytest.mark.parametrize("M,N", [(130, 520), (130, 513), (3, 515)])
def test_linear_weight_gradient_of_many_inputs(M, N):
    """More tiles of dW than a launch has, sums of db beside them; one row of x and dy is not zero."""
    hd = _hd()
    K, r = 1 << 24, M // 2
    x, dy = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    x[r] = torch.arange(K, device="cuda", dtype=torch.int32).remainder_(13).to(torch.bfloat16)
    dy[r] = torch.arange(N, device="cuda").remainder_(11).to(torch.bfloat16)
    d = hd.make_linear_dims(M, K, N, hd.SLSTM_BF16)
    ws = torch.empty(hd.stacklstm_linear_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    dW, db = torch.full((K, N), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((N,), 7.0, dtype=torch.bfloat16, device="cuda")
    hd.stacklstm_linear_bwd(d, x, None, None, dy, None, dW, db, ws)
    assert torch.equal(db, dy[r])
    assert torch.equal(dW, x[r][:, None] * dy[r])        # whole numbers up to 120
