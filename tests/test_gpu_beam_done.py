"""Beams that are done, wherever the token that ends a sequence lies: a row is cut
into pieces of equal size, mostly smaller than what a workgroup's threads cover (1024
or 4096 tokens), so that a piece's last threads stand behind its end, on tokens of
the next piece.  A done beam has one token with a probability, counted once."""
import numpy as np
import pytest
import torch

from _parity import log
from test_gpu_beam import BF, F32, check, draw


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def ends(V, piece, covered):
    """Tokens around the borders of the first pieces, and the row's own."""
    near = [0, piece - 1, piece, piece + 7, (piece + covered) // 2, covered - 1, covered, 2 * piece - 1, 2 * piece,
            piece + covered - 1, V - 1]
    return sorted({e for e in near if 0 <= e < V})


# B, W, V, and the pieces that these are cut into: tokens of a piece, and those that its threads cover
CASES = [(4, 6, 6454, 922, 1024), (1, 4, 32000, 1000, 1024), (2, 3, 1025, 513, 1024), (3, 5, 1500, 750, 1024),
         (20, 8, 5000, 2500, 4096), (40, 4, 9001, 3001, 4096), (70, 8, 1300, 1300, 4096), (2, 2, 70001, 3889, 4096)]


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,W,V,piece,covered", CASES)
def test_the_end_token_in_every_place(mmf, B, W, V, piece, covered, t):
    z, s, g = draw(B, W, V, t, V + W)
    n = W
    for end in ends(V, piece, covered):
        log(f"[beam done] {B} {W} {V} {t} end={end}")
        done = (torch.rand(B, W, generator=g) < 0.6).to(torch.uint8)
        done[0] = 1                                           # a batch whose beams are all done
        got = check(mmf, z, s, done, end, n)
        # the beams of the first batch go on as they are
        order = np.argsort(-s[0].numpy(), kind="stable")
        assert (got["parents"][0] == order).all() and (got["tokens"][0] == end).all()
        assert (got["scores"][0] == s[0].numpy()[order]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,W,V,piece,covered", CASES)
def test_more_candidates_than_a_done_beam_has(mmf, B, W, V, piece, covered, t):
    """One beam, done: its candidates behind the first have no probability and come
    in the order of their tokens."""
    z, s, _ = draw(B, 1, V, t, V)
    done = torch.ones(B, 1, dtype=torch.uint8)
    for end in ends(V, piece, covered):
        for n in (2, 33, 64):
            got = check(mmf, z, s, done, end, n)
            others = [i for i in range(n) if i != end][:n - 1]
            assert (got["tokens"] == np.array([end] + others)).all()
