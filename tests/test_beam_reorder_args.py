"""Which lists of tensors the reordering of beams' states takes, without a GPU:
the library's call is replaced by one that keeps its arguments, and tensors on
the CPU stand for those on the device."""
import ctypes

import pytest
import torch

B, W = 2, 3


@pytest.fixture
def reorder(monkeypatch):
    import paper_2406_02528_amd as mmf
    calls = []

    class Lib:
        @staticmethod
        def mmf_beam_reorder(src, dst, rows, n, *rest):
            at = lambda p: list((ctypes.c_uint64 * n).from_address(p if isinstance(p, int) else p.value)) if n else []  # noqa: E731
            calls.append((at(src), at(dst)))
            return 0

    monkeypatch.setattr(mmf, "_lib", Lib)
    monkeypatch.setattr(mmf, "_here", lambda: -1)
    monkeypatch.setattr(mmf, "_stream_here", lambda stream, here: 0)
    parents = torch.zeros(B, W, dtype=torch.int32)
    return lambda states, outs=None: mmf.mmf_beam_reorder(states, parents, B, W, outs), calls


def state(words=4):
    return torch.zeros(B * W, words)


def test_lists_that_are_taken(reorder):
    call, calls = reorder
    a, b, c, d = (state() for _ in range(4))
    empty = state(0)
    for states, outs in (([a, b], None), ([a, b], [c, d]), ([a, b], [a, b]), ([a, b], [a, c]), ([a, a], [b, c]),
                         ([a, b, empty], [c, d, empty]), ([empty, empty], [empty, empty]), ([empty, a], [a[:, :0], b]), ([], [])):
        call(states, outs)
        want = [[t.data_ptr() for t in x] for x in (states, states if outs is None else outs)]
        assert list(calls[-1]) == want
    assert len(calls) == 9


def test_a_tensor_that_is_written_and_read_in_other_places_is_refused(reorder):
    """The rows of all tensors move in one launch, in no order."""
    call, calls = reorder
    a, b, c, d = (state() for _ in range(4))
    for states, outs in (([a, b], [b, a]), ([a, b], [b, c]), ([a, b], [c, a]), ([a, b, c], [b, c, d]), ([a, a], [a, b]),
                         ([a, a], [b, a])):
        with pytest.raises(ValueError, match="reads"):
            call(states, outs)
    with pytest.raises(ValueError, match="twice"):
        call([a, a])
    with pytest.raises(ValueError, match="twice"):
        call([a, b], [c, c])
    assert not calls
