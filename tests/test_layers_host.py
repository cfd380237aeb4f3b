"""C-ABI of the layers around the states (no GPU needed): the library exports what the header declares, work-space sizes, and
refusals that launch nothing (the addresses are never followed)."""
import ctypes
import os
import re

import pytest

from paper_1904_03409_amd import layers as ly

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "stacklstm_layers.h")
P, NUL, SIZE = ctypes.c_void_p, ctypes.c_void_p(0), ctypes.c_size_t


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_library_exports_every_declared_function():
    names = sorted(set(re.findall(r"\b(stacklstm_\w+)\s*\(", _text())))
    assert set(names) == set(ly.EXPORTS) and len(names) == 11
    lib = ly.load_library()
    assert not [n for n in names if not hasattr(lib, n)]


@pytest.mark.parametrize("struct", ["slstm_strides", "slstm_attend_dims", "slstm_logprob_dims", "slstm_dropout_dims"])
def test_structures_have_the_headers_fields(struct):
    body = [b for b, n in re.findall(r"typedef struct \{([^}]*)\} (\w+);", _text()) if n == struct][0]
    want = []
    for line in body.split(";"):
        words = line.split()
        if words:
            want += [(n.strip(" ,"), words[0]) for n in " ".join(words[1:]).split(",")]
    kinds = {ctypes.c_int64: "int64_t", ctypes.c_int32: "int32_t", ctypes.c_float: "float", ly.slstm_strides: "slstm_strides"}
    assert [(n, kinds[t]) for n, t in getattr(ly, struct)._fields_] == want


def test_work_spaces():
    mk = ly.make_attend_dims
    # row tiles that fill the chip need none for splits
    assert ly.stacklstm_attend_fwd_workspace_bytes(mk(2, 4096, 4000, 16, 4, 128, 1)) <= 64
    # one query over a long sequence is split; its parts are bounded by a float row for every 128 keys
    n = ly.stacklstm_attend_fwd_workspace_bytes(mk(1, 1, 1 << 20, 8, 8, 64))
    assert 64 < n <= (1 << 20) // 128 * 8 * (64 + 2) * 4 + 256
    assert ly.stacklstm_attend_bwd_workspace_bytes(mk(3, 5, 7, 4, 2, 16)) >= 3 * 5 * 4 * 4
    # a byte to an element of a 16-bit y beside a row's two statistics, but where the backward needs no y
    width = ly.stacklstm_attend_stats_width
    assert [width(mk(3, 5, 700, 4, 2, 50, t)) for t in (0, 1)] == [2, 2 + 13] and width(mk(3, 5, 128, 4, 2, 64, 1)) == 2
    assert width(mk(3, 5, 128, 4, 2, 65, 1)) == 2 + 17 and width(mk(-1, 5, 128, 4, 2, 65, 1)) == 0
    # rows that fit registers need none
    assert ly.stacklstm_logprob_workspace_bytes(ly.make_logprob_dims(4096, 32000, 1, 64, 1)) <= 64
    assert ly.stacklstm_logprob_workspace_bytes(ly.make_logprob_dims(4, 131071, 3, 10)) >= 4 * 32 * (12 + 80)


def test_refusals_launch_nothing():
    lib = ly.load_library()
    mk = ly.make_attend_dims
    inf, nan = float("inf"), float("nan")
    S = ly.slstm_strides
    bad = [mk(-1, 1, 1, 1, 1, 8), mk(1, -1, 1, 1, 1, 8), mk(1, 1, -1, 1, 1, 8), mk(1, 1, 1, 0, 1, 8), mk(1, 1, 1, 1, 0, 8),
           mk(1, 1, 1, 3, 2, 8), mk(1, 1, 1, 1, 2, 8), mk(1, 1, 1, 1, 1, 0), mk(1, 1, 1, 1, 1, 257), mk(1, 1, 1, 1, 1, 8, 2),
           mk(1, 1, 1, 1, 1, 8, 0, inf), mk(1, 1, 1, 1, 1, 8, 0, nan), mk(1, (1 << 24) + 1, 1, 1, 1, 8), mk(1, 1, (1 << 24) + 1, 1, 1, 8),
           mk(1 << 10, 1 << 20, 1, 2, 1, 8), mk(1 << 10, 1, 1 << 20, 2, 2, 8), mk(1, 1, 1, 1 << 17, 1, 8),
           mk(2, 3, 4, 2, 2, 8, q=S(-1, 8, 8)), mk(2, 3, 4, 2, 2, 8, k=S(1 << 41, 8, 8)),
           # outputs with two elements at one place: broadcast, overlapping heads, overlapping sequences
           mk(2, 3, 4, 2, 2, 8, y=S(0, 16, 8)), mk(2, 3, 4, 2, 2, 8, dq=S(48, 16, 7)), mk(2, 3, 4, 2, 2, 8, dk=S(63, 16, 8)),
           mk(2, 3, 4, 2, 2, 8, dv=S(8, 8, 32)),
           # ... and one whose end no 64-bit offset reaches
           mk(1 << 30, 1, 1, 1, 1, 8, y=S(1 << 39, 8, 8)), None]
    one = P(1 << 20)
    for d in bad:
        assert lib.stacklstm_attend_fwd_workspace_bytes(d) == 0 and lib.stacklstm_attend_bwd_workspace_bytes(d) == 0
        assert lib.stacklstm_attend_fwd(d, *[one] * 9, SIZE(1 << 30), NUL) == 1
        assert lib.stacklstm_attend_bwd(d, *[one] * 13, SIZE(1 << 30), NUL) == 1
    good = mk(2, 3, 4, 2, 2, 8, y=S(16, 32, 8), q=S(0, 16, 8))
    a = [P(i << 24) for i in range(1, 14)]
    assert lib.stacklstm_attend_fwd_workspace_bytes(good) > 0
    # missing arrays, an output that is an input, work spaces that are missing, too small or at an odd place
    assert lib.stacklstm_attend_fwd(good, *[NUL] * 9, SIZE(0), NUL) == 1
    for hole in (0, 1, 2, 6):
        assert lib.stacklstm_attend_fwd(good, *[NUL if i == hole else a[i] for i in range(9)], SIZE(1 << 30), NUL) == 1
    for same in (0, 1, 2):
        assert lib.stacklstm_attend_fwd(good, *[a[same] if i == 6 else a[i] for i in range(9)], SIZE(1 << 30), NUL) == 1
    for hole in (0, 1, 2, 6, 7, 8, 9, 10, 11, 12):
        assert lib.stacklstm_attend_bwd(good, *[NUL if i == hole else a[i] for i in range(13)], SIZE(1 << 30), NUL) == 1
    for out in (9, 10, 11):
        for other in (0, 1, 2, 6, 8, 9 + (out - 8) % 3):
            assert lib.stacklstm_attend_bwd(good, *[a[other] if i == out else a[i] for i in range(13)], SIZE(1 << 30), NUL) == 1
    assert lib.stacklstm_attend_bwd(good, *a, SIZE(8), NUL) == 4
    assert lib.stacklstm_attend_bwd(good, *a[:12], P((13 << 24) + 8), SIZE(1 << 30), NUL) == 1
    long = mk(1, 1, 1 << 16, 1, 1, 8)
    assert lib.stacklstm_attend_fwd(long, *a[:9], SIZE(8), NUL) == 4 and lib.stacklstm_attend_fwd(long, *a[:8], NUL, SIZE(0), NUL) == 1

    ml = ly.make_logprob_dims
    for d in (ml(-1, 8), ml(4, 0), ml(4, 8, -1), ml(4, 8, 65), ml(4, 8, 1, -1), ml(4, 8, 1, 65), ml(4, 8, 1, 0, 2), ml(4, (1 << 22) + 1),
              ml(4, 8, ld_logits=7), ml(4, 8, ld_dlogits=7), ml(1 << 31, 8), None):
        assert lib.stacklstm_logprob_workspace_bytes(d) == 0
        assert lib.stacklstm_logprob_fwd(d, *a[:9], SIZE(1 << 30), NUL) == 1
        assert lib.stacklstm_logprob_bwd(d, *a[:7], NUL) == 1
        assert lib.stacklstm_logprob_step(d, *a[:11], SIZE(1 << 30), NUL) == 1
    d = ml(4, 131072, 2, 3)
    for hole in (0, 2, 3, 5, 6, 8):
        assert lib.stacklstm_logprob_fwd(d, *[NUL if i == hole else a[i] for i in range(9)], SIZE(1 << 30), NUL) == 1
    for hole in (0, 2, 3, 6):
        assert lib.stacklstm_logprob_bwd(d, *[NUL if i == hole else a[i] for i in range(7)], NUL) == 1
    for hole in (0, 2, 5, 7, 8, 9, 10):
        assert lib.stacklstm_logprob_step(d, *[NUL if i == hole else a[i] for i in range(11)], SIZE(1 << 30), NUL) == 1
    assert lib.stacklstm_logprob_fwd(d, *a[:9], SIZE(8), NUL) == 4
    # in place with other strides
    other = ml(4, 8, 1, ld_logits=8, ld_dlogits=9)
    assert lib.stacklstm_logprob_bwd(other, *a[:6], a[0], NUL) == 1

    md = ly.make_dropout_dims
    for d in (md(-1, 8), md(4, 0), md(4, 8, 2), md(4, 8, 0, -0.1), md(4, 8, 0, 1.1), md(4, 8, 0, nan), md(4, 8, period=-1),
              md(4, 8, ld_x=7), md(4, 8, ld_res=7), md(4, 8, ld_y=7), md(1 << 31, 8), md(4, (1 << 24) + 1), md(4, 8, period=1 << 31), None):
        assert lib.stacklstm_dropout_fwd(d, *a[:4], NUL) == 1 and lib.stacklstm_dropout_bwd(d, *a[:3], NUL) == 1
    d = md(4, 8)
    for hole in (0, 2, 3):
        assert lib.stacklstm_dropout_fwd(d, *[NUL if i == hole else a[i] for i in range(4)], NUL) == 1
    assert lib.stacklstm_dropout_fwd(md(4, 8, ld_x=9), a[0], NUL, a[2], a[0], NUL) == 1
    assert lib.stacklstm_dropout_fwd(md(4, 8, ld_res=9), a[0], a[1], a[2], a[1], NUL) == 1


def test_nothing_to_do_is_done():
    lib = ly.load_library()
    assert lib.stacklstm_attend_fwd(ly.make_attend_dims(0, 3, 4, 1, 1, 8), *[NUL] * 9, SIZE(0), NUL) == 0
    assert lib.stacklstm_attend_fwd(ly.make_attend_dims(2, 0, 4, 1, 1, 8), *[NUL] * 9, SIZE(0), NUL) == 0
    assert lib.stacklstm_attend_bwd(ly.make_attend_dims(2, 0, 0, 1, 1, 8), *[NUL] * 13, SIZE(0), NUL) == 0
    assert lib.stacklstm_logprob_fwd(ly.make_logprob_dims(0, 8, 1, 2), *[NUL] * 9, SIZE(0), NUL) == 0
    assert lib.stacklstm_logprob_step(ly.make_logprob_dims(0, 8), *[NUL] * 11, SIZE(0), NUL) == 0
    assert lib.stacklstm_logprob_bwd(ly.make_logprob_dims(0, 8), *[NUL] * 7, NUL) == 0
    assert lib.stacklstm_dropout_fwd(ly.make_dropout_dims(0, 8), *[NUL] * 4, NUL) == 0
    assert lib.stacklstm_dropout_bwd(ly.make_dropout_dims(0, 8), *[NUL] * 3, NUL) == 0


def test_strides_of_views():
    import torch
    t = torch.zeros(5, 3, 2, 8)
    s = ly.strides_of(t.transpose(0, 1))
    assert (s.b, s.t, s.h) == (16, 48, 8)
    s = ly.strides_of(t)
    assert (s.b, s.t, s.h) == (48, 16, 8)
    # one sequence: its stride is any
    s = ly.strides_of(t[:1, :, :, :4])
    assert (s.t, s.h) == (16, 8)
    with pytest.raises(ValueError):
        ly.strides_of(t.transpose(2, 3))
    like = ly._like(t.transpose(0, 1))
    assert like.shape == (3, 5, 2, 8) and like.stride() == (16, 48, 8, 1)
