"""Clipping where the norm or the limit is not finite."""
import pytest
import torch

from _parity import dev, log

BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def bits(t):
    return t.view(torch.int16 if t.dtype == BF else torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True], ids=["out", "in_place"])
@pytest.mark.parametrize("bad", [INF, -INF, 3.0e38, 1.0], ids=["inf", "-inf", "overflow", "finite"])
def test_no_limit(mmf, bad, in_place):
    """An infinite max_norm changes nothing, whatever the norm is, infinite
    among it (an infinite gradient, or a norm past fp32); a NaN in the norm
    still reaches every output."""
    log(f"[clip] max_norm=inf value={bad} in_place={in_place}")
    gen = torch.Generator(device="cuda").manual_seed(21)
    grads = [torch.randn(n, generator=gen, device=dev()).to(t) for n, t in ((40000, F32), (333, BF), (0, F32), (1, F32))]
    grads[0][17:39] = bad
    grads[1][5] = bad if abs(bad) == INF else 1.0
    before = [g.clone() for g in grads]
    outs = None if in_place else [torch.full_like(g, NAN) for g in grads]
    norm = torch.zeros(1, device=dev())
    mmf.mmf_grad_norm(grads, norm)
    assert bool(norm.isinf()) == (bad != 1.0)
    mmf.mmf_grad_clip(grads, norm, INF, outs)
    for b, g, o in zip(before, grads, grads if in_place else outs):
        assert torch.equal(bits(o), bits(b)) and torch.equal(bits(g), bits(b))
    norm.fill_(NAN)
    mmf.mmf_grad_clip(grads, norm, INF, outs)
    assert all(o.isnan().all() for o in (grads if in_place else outs))
