"""Beam search and distillation at their limits: the largest sizes, rows past 32
bits of the inputs, what lies around the outputs, equal bits on repetition.
Error bounds as derived in test_gpu_beam.py and test_gpu_distill.py."""
import numpy as np
import pytest
import torch

from _parity import dev, log
from test_gpu_beam import check as check_beam, draw, reference as beam_reference, reorder_case, reordered
from test_gpu_distill import U, inputs as distill_inputs, reference as distill_reference

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("B,W,V,n", [(1, 1, 2 ** 18, 64), (1, 3, 2 ** 18, 1), (1, 64, 2 ** 15, 64), (200, 1, 300, 7),
                                     (40, 16, 1025, 16), (1, 2, 32, 64), (1, 48, 2000, 64), (2, 32, 3000, 64),
                                     (1, 64, 64, 64)], ids=str)
def test_largest_selections(mmf, B, W, V, n):
    log(f"[beam] {B} {W} {V} {n}")
    z, s, g = draw(B, W, V, F32, V + n)
    done = (torch.rand(B, W, generator=g) < 0.3).to(torch.uint8)
    check_beam(mmf, z, s, done, V - 1, n)
    check_beam(mmf, z, s, None, -1, n)


@pytest.mark.gpu
def test_selection_of_few_different_logits(mmf):
    """bf16 logits that repeat, the best of all beams in one place."""
    g = torch.Generator().manual_seed(9)
    z = (torch.randint(-2, 3, (3, 5, 9000), generator=g) * 2.0).to(BF)
    z[:, 2, 4000:4064] = 8.0
    check_beam(mmf, z, torch.zeros(3, 5), None, 7, 64)
    z = torch.full((2, 3, 20000), -3.0).to(BF)      # one value alone
    check_beam(mmf, z, torch.zeros(2, 3), None, -1, 50)


@pytest.mark.gpu
def test_logits_past_32_bits(mmf):
    B, W, V, n = 5400, 4, 50001, 4                  # 4.3 GB of fp32
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = torch.empty(B * W, V, device=dev())
    for i in range(0, B * W, 2048):
        z[i:i + 2048] = torch.randn(z[i:i + 2048].shape, generator=gen, device=dev()) * 3
    s = -20 * torch.rand(B, W, generator=gen, device=dev())
    out = [torch.empty(B, n, device=dev())] + [torch.full((B, n), -1, dtype=torch.int32, device=dev()) for _ in range(2)]
    mmf.mmf_beam_select(z, s, None, -1, B, W, n, *out, None)
    last = z[-2 * W:].reshape(2, W, V).double().cpu().numpy()
    want = beam_reference(last, s[-2:].cpu().numpy(), None, -1, n)
    assert np.array_equal(out[1][-2:].cpu().numpy(), want["tokens"])
    assert np.array_equal(out[2][-2:].cpu().numpy(), want["parents"])
    got = out[0][-2:].double().cpu().numpy()
    assert (np.abs(got - want["scores"]) <= 2.0 ** -17 + 2.0 ** -24 * np.abs(want["scores"])).all()


@pytest.mark.gpu
@pytest.mark.parametrize("W,words", [(4, 1 << 18), (16, 1 << 17), (20, 1 << 12)])
def test_large_rows_in_place(mmf, W, words):
    """Rows past the size from which the copies pass the caches, and past 32 bits
    of their array (the first case)."""
    B = max(2, (2 ** 30 + 2 ** 22) // (W * words)) if W == 4 else 3
    gen = torch.Generator(device="cuda").manual_seed(W)
    x = torch.randint(0, 2 ** 31 - 1, (B * W, words), generator=gen, dtype=torch.int32, device=dev())
    parents = torch.randint(0, W, (B, W), generator=gen, dtype=torch.int32, device=dev())
    src = (parents.long() + W * torch.arange(B, device=dev())[:, None]).reshape(-1)
    out = torch.empty_like(x)
    mmf.mmf_beam_reorder([x], parents, B, W, [out])
    assert all(torch.equal(out[i], x[src[i]]) for i in list(range(0, B * W, 37)) + [B * W - 1])
    mmf.mmf_beam_reorder([x], parents, B, W)
    assert torch.equal(x, out)


@pytest.mark.gpu
@pytest.mark.parametrize("W", [3, 11, 33])
def test_nothing_around_the_beams_is_written(mmf, W):
    B, V, n = 3, 777, 5
    z, s, g = draw(B, W, V, BF, W)
    pad = 64

    def guarded(count, dt):
        full = torch.full((count + 2 * pad,), 7, dtype=dt, device=dev())
        return full, full[pad:pad + count]

    fs = [guarded(B * n, dt) for dt in (F32, torch.int32, torch.int32, torch.uint8)]
    need = mmf.mmf_beam_select_workspace_bytes(B, W, V, n)
    ws = torch.full((need + 256,), 77, dtype=torch.uint8, device=dev())
    first = None
    for _ in range(3):
        mmf.mmf_beam_select(z.reshape(B * W, V).to(dev()), s.to(dev()), None, 5, B, W, n, *(v.reshape(B, n) for _, v in fs),
                            ws[:need])
        now = [v.clone() for _, v in fs]
        assert first is None or all(torch.equal(a, b) for a, b in zip(now, first))
        first = now
    assert (ws[need:] == 77).all() and all((f[:pad] == 7).all() and (f[-pad:] == 7).all() for f, _ in fs)
    states, parents = reorder_case(B, W, [(20,), (300,)], W)
    full = [torch.full((B * W + 2, *x.shape[1:]), 7, dtype=x.dtype, device=dev()) for x in states]
    for f, x in zip(full, states):
        f[1:-1] = x.to(dev())
    mmf.mmf_beam_reorder([f[1:-1] for f in full], parents.to(dev()), B, W)
    for f, x in zip(full, reordered(states, parents)):
        assert torch.equal(f[1:-1].cpu(), x) and (f[0] == 7).all() and (f[-1] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
def test_distillation_past_32_bits(mmf, t):
    V, K = 50003, 32
    M = 2 ** 32 // (V * (4 if t == F32 else 2)) + 40
    gen = torch.Generator(device="cuda").manual_seed(2)
    z = torch.empty(M, V, dtype=t, device=dev())
    for i in range(0, M, 2048):
        z[i:i + 2048] = torch.randn(z[i:i + 2048].shape, generator=gen, device=dev()) * 3
    idx = torch.randint(0, V, (M, K), generator=gen, device=dev(), dtype=torch.int32)
    te = torch.randn(M, K, generator=gen, device=dev())
    dl = torch.rand(M, generator=gen, device=dev()) + 0.1
    keep = z[-3:].cpu()
    loss = torch.empty(M, device=dev())
    mmf.mmf_distill_bwd(z, idx, te, 1.5, dl, z, loss)         # in place
    want, dwant, q, _ = distill_reference(keep, idx[-3:].cpu(), te[-3:].cpu(), 1.5, dl[-3:].cpu())
    assert ((loss[-3:].cpu().double() - want).abs() <= 160 * U * 1.5 ** 2 + U * want.abs()).all()
    half = torch.finfo(t).eps / 2
    bound = dl[-3:].cpu().double()[:, None] * 1.5 * (160 * U * q + 2.0 ** -43 * q.amax(1, keepdim=True)) * (1 + half)
    bound = bound + (half + U) * dwant.abs() + 1e-38
    assert ((z[-3:].cpu().double() - dwant).abs() <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,V,K", [(1, 8, 3), (7, 1009, 64), (3, 70003, 100)])
def test_nothing_around_the_gradient_is_written(mmf, M, V, K):
    for t in (F32, BF):
        z, idx, te, dl = (x.to(dev()) for x in distill_inputs(M, V, K, t, F32, V))
        pad, first = 64, None
        full = torch.full((M * V + 2 * pad,), 7, dtype=t, device=dev())
        floss = torch.full((M + 2 * pad,), 7.0, device=dev())
        for _ in range(3):
            mmf.mmf_distill_bwd(z, idx, te, 1.0, dl, full[pad:pad + M * V].reshape(M, V), floss[pad:pad + M])
            mmf.mmf_distill_fwd(z, idx, te, 1.0, floss[pad:pad + M])
            now = torch.cat([full.float(), floss])
            assert first is None or torch.equal(now, first)
            first = now
        assert all((f[:pad] == 7).all() and (f[-pad:] == 7).all() for f in (full, floss))


@pytest.mark.gpu
@pytest.mark.parametrize("tau", [1e-3, 0.05, 30.0, 1e4])
def test_temperatures(mmf, tau):
    """From nearly the best token alone to nearly all alike.  The exponentials'
    arguments are in units of tau, so the bounds hold for every tau."""
    z, idx, te, dl = distill_inputs(4, 3001, 20, F32, F32, 11)
    want, dwant, q, p = distill_reference(z, idx, te, tau, dl)
    loss, dz = torch.empty(4, device=dev()), torch.empty(4, 3001, device=dev())
    mmf.mmf_distill_bwd(z.to(dev()), idx.to(dev()), te.to(dev()), tau, dl.to(dev()), dz, loss)
    tau = float(torch.tensor(tau, dtype=F32))
    # of the loss also each teacher token's ln q, whose argument is rounded: 3 u |z - max| / tau
    far = ((z.double().amax(1) - z.double().amin(1)) / tau + (te.double().amax(1) - te.double().amin(1)) / tau) * 4 * U
    assert ((loss.cpu().double() - want).abs() <= tau * tau * (160 * U + far) + U * want.abs()).all()
    bound = dl.double()[:, None] * tau * (160 * U * q + 2.0 ** -43 * q.amax(1, keepdim=True))
    bound = bound + dl.double()[:, None] * tau * far[:, None] * p + 2 * U * dwant.abs() + 1e-38
    assert ((dz.cpu().double() - dwant).abs() <= bound).all()
