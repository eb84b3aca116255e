"""Distillation over rows with masked tokens (logits of -inf) and with NaN, at
the lengths on both sides of the border from which a row is read twice: 4096
vectors of 8 bf16 logits, 8192 of fp32.  A thread takes every 1024th vector of
such a row.  Error bounds as derived in test_gpu_distill.py: a masked token's
exponential is 0 exactly."""
import pytest
import torch

from _parity import log
from test_gpu_distill import check, inputs, run

BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")
LENGTHS = [32775, 32776, 33001, 65543, 65544, 70003, 140001]


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def masked(V):
    """Which tokens each of the rows is denied: runs that are a thread's first
    vector, its last, all of it, some of both, and nearly the whole row."""
    m = torch.zeros(9, V, dtype=torch.bool)
    m[0, :24] = True                       # the start
    m[1, 16:24] = True                     # one vector of a row that starts on one
    m[2, 8183:8215] = True                 # a thread's first and its second vectors
    m[3, -4099:] = True                    # the end
    m[4, ::3] = True                       # some of every vector
    m[5] = True
    m[5, V // 2:V // 2 + 3] = False        # all but three
    m[6] = True
    m[6, :1] = False                       # all but the first
    m[7, :V - 9] = True                    # all but the last
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", LENGTHS)
def test_masked_tokens(mmf, V, t):
    log(f"[distill masks] V={V} {t}")
    z, _, te, dl = inputs(9, V, 5, t, F32, V)
    off = masked(V)
    z[off] = -INF
    g = torch.Generator().manual_seed(V)
    idx = torch.empty(9, 5, dtype=torch.int32)
    for i, row in enumerate(off):          # the teacher's tokens are among the others, some of them twice
        free = (~row).nonzero()[:, 0]
        idx[i] = free[torch.randint(0, len(free), (5,), generator=g)].to(torch.int32)
    for inplace in (False, True):
        check(mmf, z, idx, te, 1.5, dl, t, inplace=inplace)
    check(mmf, z, idx, te, 1.0, -dl, BF if t == F32 else F32)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", LENGTHS)
def test_one_value_that_is_no_number(mmf, V, t):
    """Anywhere in a row, with -inf alone beside it for the thread that has it,
    before it or behind it: the row's loss and gradient are NaN, the others' not."""
    log(f"[distill masks] no number V={V} {t}")
    at = [0, 3, 8200, 8200 + 8192, V // 2, V - 1]
    n = len(at)
    for value in (float("nan"), INF):
        z, _, te, dl = inputs(2 * n, V, 3, t, F32, V)
        idx = torch.full((2 * n, 3), 100, dtype=torch.int32)
        z[n:] = -INF
        z[n:, 100:103] = 1.0
        for i, c in enumerate(at):
            z[2 * (i // 2), c] = value     # of the rows drawn every other one
            z[n + i, c] = value
        bad = torch.tensor([not z[i].isfinite().all() if i < n else True for i in range(2 * n)])
        loss, dz = run(mmf, z, idx, te, 2.0, dl, F32)
        assert loss[bad].isnan().all() and dz[bad].isnan().all()
        assert loss[~bad].isfinite().all() and dz[~bad].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", LENGTHS)
def test_no_token_possible(mmf, V, t):
    """A row of -inf alone gives NaN; where dloss is 0 or no entry is there, 0."""
    z, idx, te, dl = inputs(3, V, 3, t, F32, V)
    z[:] = -INF
    dl[1] = 0.0
    idx[2] = -1
    loss, dz = run(mmf, z, idx, te, 2.0, dl, t)
    assert loss[:2].isnan().all() and loss[2] == 0
    assert dz[0].isnan().all() and (dz[1:] == 0).all()
