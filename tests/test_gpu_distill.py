"""Distillation from a teacher's best tokens against 64 bits (CPU).

With u = 2^-24: an exponential 2^(x log2(e) / tau) has its argument rounded
three times and its result once (1.5 |x| 3 u + 2 u relative, x <= 0 the
distance from the maximum in units of tau); where |x| > 30 it is below 2^-43
and held to an absolute bound of the largest.  Sums are fp64 after fp32 sums of
at most 8.  So q is within (140 + 10) u relative (x >= -30), ln of the sum
within 160 u, and
  loss: tau^2 sum p |d ln q| <= 160 u tau^2, rounded once: u |loss|
  dz: dloss tau 160 u q (at the teacher's tokens q - p is taken in fp64), rounded
    to fp32 and then to its type.
"""
import pytest
import torch

from _parity import dev, log

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U = 2.0 ** -24


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def inputs(M, V, K, zt, tt, seed=0, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(M, V, generator=g) * scale).to(zt)
    idx = torch.stack([torch.randperm(V, generator=g)[:K] if V >= K else torch.randint(0, V, (K,), generator=g)
                       for _ in range(M)]).to(torch.int32)
    t = (torch.randn(M, K, generator=g) * 3).to(tt)
    return z, idx, t, torch.rand(M, generator=g) + 0.1


def reference(z, idx, t, tau, dloss):
    """loss, dz and the q and p behind it, in 64 bits."""
    M, V = z.shape
    tau = float(torch.tensor(tau, dtype=F32))  # as the call takes it
    lq = torch.log_softmax(z.double() / tau, 1)
    ok = (idx >= 0) & (idx < V) & (t != -float("inf"))
    some = ok.any(1)
    tt = torch.where(ok, t.double() / tau, -float("inf"))
    tt[~some] = 0.0
    lp = torch.log_softmax(tt, 1)
    p = torch.where(ok, lp.exp(), 0.0)
    at = torch.where(ok, idx, 0).long()
    terms = torch.where(ok & (p > 0), p * (lp - lq.gather(1, at)), 0.0)
    loss = tau * tau * terms.sum(1)
    target = torch.zeros(M, V, dtype=F64).scatter_add_(1, at, p)
    dz = (lq.exp() - target) * (dloss.double() * tau)[:, None]
    loss[~some] = 0.0
    dz[~some | (dloss == 0)] = 0.0
    return loss, dz, lq.exp(), target


def run(mmf, z, idx, t, tau, dloss, dt, inplace=False):
    z, idx, t, dloss = (x.to(dev()) for x in (z, idx, t, dloss))
    M, V = z.shape
    loss, loss2 = (torch.full((M,), float("nan"), device=dev()) for _ in range(2))
    mmf.mmf_distill_fwd(z, idx, t, tau, loss)
    dz = z.clone() if inplace else torch.full((M, V), float("nan"), dtype=dt, device=dev())
    mmf.mmf_distill_bwd(dz if inplace else z, idx, t, tau, dloss, dz, loss2)
    alone = torch.full((M, V), float("nan"), dtype=dt, device=dev())
    mmf.mmf_distill_bwd(z, idx, t, tau, dloss, alone)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) or (loss.isnan() == loss2.isnan()).all()
    assert torch.equal(alone.nan_to_num(7.0), dz.nan_to_num(7.0))
    return loss.cpu(), dz.cpu()


def check(mmf, z, idx, t, tau, dloss, dt, inplace=False, rows=slice(None)):
    want, dwant, q, p = reference(z, idx, t, tau, dloss)
    loss, dz = run(mmf, z, idx, t, tau, dloss, dt, inplace)
    err = (loss.double() - want).abs()[rows]
    assert (err <= 160 * U * tau * tau + U * want[rows].abs()).all(), float(err.max())
    half = torch.finfo(dt).eps / 2
    top = q.amax(1, keepdim=True)
    bound = dloss.double()[:, None].abs() * tau * (160 * U * q + 2.0 ** -43 * top) * (1 + half)
    bound = bound + (half + U) * dwant.abs() + 1e-38
    bad = ~((dz.double() - dwant).abs() <= bound)[rows]
    assert not bad.any(), int(bad.sum())
    return loss, dz


SHAPES = [(1, 1, 1), (3, 2, 1), (2, 7, 3), (5, 33, 5), (4, 1000, 20), (3, 1023, 64), (2, 4099, 256), (2, 8192, 1), (3, 32000, 64),
          (2, 33001, 128), (2, 65543, 17), (1, 131072, 1024), (2, 140001, 33), (70, 515, 515)]


@pytest.mark.gpu
@pytest.mark.parametrize("zt", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("dt", [F32, BF], ids=["d_f32", "d_bf16"])
@pytest.mark.parametrize("M,V,K", SHAPES)
def test_loss_and_gradient(mmf, M, V, K, zt, dt):
    log(f"[distill] M={M} V={V} K={K} {zt} {dt}")
    z, idx, t, dl = inputs(M, V, K, zt, BF if V % 2 else F32, V + K)
    check(mmf, z, idx, t, 1.0 if K % 2 else 2.5, dl, dt)
    if zt == dt:
        check(mmf, z, idx, t, 0.7, -dl, dt, inplace=True)


@pytest.mark.gpu
@pytest.mark.parametrize("zt", [F32, BF], ids=["f32", "bf16"])
def test_entries_that_are_none(mmf, zt):
    z, idx, t, dl = inputs(9, 2000, 12, zt, F32, 4)
    inf = float("inf")
    idx[0, 3:] = -1
    idx[1] = -1                                   # a row of padding
    idx[2, 0], idx[2, 1] = 2000, 2 ** 31 - 1      # outside
    t[3, 2:] = -inf
    t[4] = -inf                                   # no entry either
    idx[5, 5:9] = idx[5, 0]                       # a token more than once
    z[6, :1900] = -inf                            # tokens that the student is denied
    idx[6] = torch.arange(1950, 1962)
    t[7, 0] = -inf
    z[7, idx[7, 0].long()] = -inf                 # and where p is 0
    z[1] = float("nan")                           # what padding holds
    z[4, 100] = inf
    z[8] = float("nan")
    dl[8] = 0.0
    keep = [0, 2, 3, 5, 6, 7]
    clean = z.clone()
    clean[[1, 4, 8]] = 0.0
    want, dwant, _, _ = reference(clean, idx, t, 2.0, dl)
    loss, dz = run(mmf, z, idx, t, 2.0, dl, F32)
    assert (loss[[1, 4]] == 0).all() and (dz[[1, 4, 8]] == 0).all() and loss[8].isnan()
    clean_loss, clean_dz = check(mmf, clean, idx, t, 2.0, dl, F32, rows=keep)
    assert torch.equal(clean_loss[keep], loss[keep]) and torch.equal(clean_dz[keep], dz[keep])


@pytest.mark.gpu
def test_infinite_and_missing_values(mmf):
    z, idx, t, dl = inputs(5, 700, 4, F32, F32, 5)
    inf = float("inf")
    z[0, 5], z[1, 5], z[2] = float("nan"), inf, -inf
    z[3, idx[3, 0].long()] = -inf                 # the teacher wants what the student denies
    loss, dz = run(mmf, z, idx, t, 1.0, dl, F32)
    assert loss[:3].isnan().all() and dz[:3].isnan().all() and loss[3] == inf
    want, dwant, _, _ = reference(z, idx, t, 1.0, dl)
    assert torch.allclose(dz[3:].double(), dwant[3:], rtol=1e-4, atol=1e-8) and loss[4] > 0


@pytest.mark.gpu
def test_the_gradient_is_the_slope_of_the_loss(mmf):
    z, idx, t, _ = inputs(3, 257, 9, F32, F32, 6)
    tau, eps = 1.7, 2.0 ** -6
    one = torch.ones(3)
    _, dz = run(mmf, z, idx, t, tau, one, F32)
    for i in [0, 100, 256, int(idx[0, 0])]:
        up, down = z.clone(), z.clone()
        up[:, i] += eps
        down[:, i] -= eps
        a, b = (reference(x, idx, t, tau, one)[0] for x in (up, down))
        slope = (a - b) / (2 * eps)
        # differences: third derivative of the loss <= 1 / tau times eps^2 / 6
        assert ((slope - dz[:, i].double()).abs() <= eps * eps / 6 + 200 * U * tau).all()
