"""Calls that the operators behind the recurrence refuse before anything is launched (no GPU needed; the addresses are never
followed)."""
import ctypes

from paper_1904_03409_amd import head as hd

P = ctypes.c_void_p


def _reorder(states, B=2, K=2):
    """The call's code for [(src, dst, slot_bytes, slots, live)]."""
    arr = (hd.slstm_beam_state * len(states))()
    for s, (src, dst, size, slots, live) in zip(arr, states):
        s.src, s.dst, s.slot_bytes, s.slots, s.live = src, dst, size, slots, live
    return hd.load_library().stacklstm_beam_reorder(hd.make_beam_dims(B, K, 1), P(1 << 20), arr, len(states), P(0))


def test_states_are_not_written_to_one_place():
    """Four rows of 48 bytes each: two states with one dst, or with dsts that share a byte, would leave either's bytes."""
    a, b, c, d = (i << 24 for i in (1, 2, 3, 4))
    assert _reorder([(a, c, 16, 3, None), (b, c, 16, 3, None)]) == 1
    assert _reorder([(a, c, 16, 3, None), (b, c + 4 * 48 - 1, 16, 3, None)]) == 1
    assert _reorder([(a, c + 4 * 48 - 1, 16, 3, None), (b, c, 16, 3, None)]) == 1
    assert _reorder([(a, c, 16, 3, None), (b, d, 16, 3, None), (b, c + 5, 1, 1, None)]) == 1
