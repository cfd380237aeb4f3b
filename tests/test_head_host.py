"""C-ABI of the operators behind the recurrence (no GPU needed): the library exports what the header declares, and the
host-only answers: work-space sizes, refusals that launch nothing."""
import ctypes
import os
import re

import pytest

from paper_1904_03409_amd import head as hd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "stacklstm_head.h")


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_library_exports_every_declared_function():
    names = sorted(set(re.findall(r"\b(stacklstm_\w+)\s*\(", _text())))
    assert set(names) == set(hd.EXPORTS) and len(names) == 14
    lib = ctypes.CDLL(hd._sl.LIB_PATH)
    assert not [n for n in names if not hasattr(lib, n)]
    hd.load_library()


@pytest.mark.parametrize("struct", ["slstm_norm_dims", "slstm_linear_dims", "slstm_distill_dims", "slstm_beam_dims",
                                    "slstm_beam_state"])
def test_structures_have_the_headers_fields(struct):
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct, _text()).group(1)
    want = []
    for line in body.split(";"):
        words = line.replace("*", " * ").split()
        if words:
            typ = "pointer" if "*" in words else words[0]
            want += [(n.strip(" ,"), typ) for n in " ".join(words[words.index("*") + 1:] if "*" in words else words[1:]).split(",")]
    kinds = {ctypes.c_int64: "int64_t", ctypes.c_int32: "int32_t", ctypes.c_float: "float", ctypes.c_void_p: "pointer"}
    assert [(n, kinds[t]) for n, t in getattr(hd, struct)._fields_] == want


def test_work_spaces():
    # sums of a backward's columns: a few blocks of rows at most
    assert 0 < hd.stacklstm_norm_workspace_bytes(hd.make_norm_dims(1, 8)) <= 64
    assert hd.stacklstm_norm_workspace_bytes(hd.make_norm_dims(1 << 30, 1024)) <= 1024 * 2 * 1024 * 4
    # a product that fills the chip needs none for its parts, a backward dz
    d = hd.make_linear_dims(61440, 1024, 4096, hd.SLSTM_BF16, hd.ACTS["gelu"])
    assert hd.stacklstm_linear_fwd_workspace_bytes(d) <= 64
    n = hd.stacklstm_linear_bwd_workspace_bytes(d)
    assert 61440 * 4096 * 2 <= n <= 61440 * 4096 * 2 + (64 + 8) * 1024 * 4096 * 4
    # parts of a split sum are bounded by the output
    for M, K, N in ((1, 1 << 20, 64), (64, 1 << 24, 64), (1, 1, 1)):
        assert 0 < hd.stacklstm_linear_fwd_workspace_bytes(hd.make_linear_dims(M, K, N)) <= max(64, 64 * M * N * 4 + 256)
    # rows that fit registers need none
    assert hd.stacklstm_distill_workspace_bytes(hd.make_distill_dims(4096, 32000, 64, hd.SLSTM_BF16)) <= 64
    assert hd.stacklstm_distill_workspace_bytes(hd.make_distill_dims(16, 131071, 32)) > 16 * 33 * 4
    assert hd.stacklstm_beam_workspace_bytes(hd.make_beam_dims(64, 8, 83)) <= 64
    assert hd.stacklstm_beam_workspace_bytes(hd.make_beam_dims(64, 16, 64001, hd.SLSTM_BF16)) == 64 * 16 * 16 * 8


def test_refusals_launch_nothing():
    """Argument errors come back before any device is looked for (this process has none)."""
    lib = hd.load_library()
    nul, size = ctypes.c_void_p(0), ctypes.c_size_t(0)
    n, l, d, b = hd.make_norm_dims(4, 8), hd.make_linear_dims(4, 8, 8), hd.make_distill_dims(4, 8, 2), hd.make_beam_dims(2, 2, 8)
    for dims in (n, None):
        assert lib.stacklstm_norm_fwd(dims, *[nul] * 9) == 1
        assert lib.stacklstm_norm_bwd(dims, *[nul] * 10, size, nul) == 1
    for dims in (l, None):
        assert lib.stacklstm_linear_fwd(dims, *[nul] * 7, size, nul) == 1
        assert lib.stacklstm_linear_bwd(dims, *[nul] * 8, size, nul) == 1
    for dims in (d, None):
        assert lib.stacklstm_distill_fwd(dims, *[nul] * 7, size, nul) == 1
        assert lib.stacklstm_distill_bwd(dims, *[nul] * 8) == 1
        assert lib.stacklstm_distill_step(dims, *[nul] * 8, size, nul) == 1
    for dims in (b, None):
        assert lib.stacklstm_beam_select(dims, *[nul] * 9, size, nul) == 1
        assert lib.stacklstm_beam_reorder(dims, nul, None, 1, nul) == 1
    assert lib.stacklstm_beam_reorder(b, nul, None, 9, nul) == 1 and lib.stacklstm_beam_reorder(b, nul, None, -1, nul) == 1
    # nothing to do is done
    assert lib.stacklstm_norm_fwd(hd.make_norm_dims(0, 8), *[nul] * 9) == 0
    assert lib.stacklstm_distill_step(hd.make_distill_dims(0, 8, 2), *[nul] * 8, size, nul) == 0
    assert lib.stacklstm_beam_select(hd.make_beam_dims(0, 2, 8), *[nul] * 9, size, nul) == 0
    assert lib.stacklstm_beam_reorder(b, nul, None, 0, nul) == 0
    for f in (lib.stacklstm_norm_workspace_bytes, lib.stacklstm_linear_fwd_workspace_bytes, lib.stacklstm_distill_workspace_bytes,
              lib.stacklstm_beam_workspace_bytes):
        assert f(None) == 0
