"""Ends of the layers' ranges (no GPU needed)."""
import pytest
import torch

from paper_1904_03409_amd import layers as ly


def test_scales():
    """Scores are taken in base 2: scale log2 e has to be a number too."""
    n = lambda scale: ly.stacklstm_attend_fwd_workspace_bytes(ly.make_attend_dims(1, 2, 3, 1, 1, 8, 0, scale))
    assert n(2.0 ** 127) and n(-2.0 ** 127) and n(2.0 ** -149) and n(0.0)
    assert n(2.0 ** 127 * (1 + 2.0 ** -23)) == 0 and n(-3.4e38) == 0
    assert ly.stacklstm_attend_bwd_workspace_bytes(ly.make_attend_dims(1, 2, 3, 1, 1, 8, 0, 3e38)) == 0


def test_strides_of_one_head_for_all():
    """Strides of 0 stand for dense ones: a head that all sequences, places and heads share is refused, of two axes it is taken."""
    one = torch.zeros(1, 1, 1, 8)
    with pytest.raises(ValueError, match="one head for all"):
        ly.strides_of(one.expand(2, 3, 4, 8))
    s = ly.strides_of(torch.zeros(1, 1, 4, 8).expand(2, 3, 4, 8))
    assert (s.b, s.t, s.h) == (0, 0, 8)
    s = ly.strides_of(one.expand(2, 3, 1, 8))
    assert (s.b, s.t, s.h) == (0, 0, 8)
    assert ly.strides_of(one.expand(0, 3, 4, 8)) is not None
