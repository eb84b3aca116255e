"""Distillation and the reordering of beams' states at the sizes from which their
streams pass the caches (256 MB of arrays): every form of bf16 rows, bit for bit
the rows of calls below that size, sampled rows against 64 bits with the bounds of
test_gpu_distill.py; and rows that move in place and into other arrays."""
import pytest
import torch

from _parity import dev, log
from test_gpu_distill import U, reference

BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")
LAST_LEVEL = 256 << 20


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["d_bf16", "d_f32"])
@pytest.mark.parametrize("V", [515, 2000, 4001, 7996, 16003, 31997, 32000, 32774])
def test_streamed_rows(mmf, V, dt):
    size = 2 + (2 if dt == BF else 4)
    M, K = LAST_LEVEL // (V * size) + 9, 24
    log(f"[distill stream] M={M} V={V} {dt}")
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn(M, V, generator=g, device=dev()) * 3).to(BF)
    idx = torch.randint(0, V, (M, K), generator=g, device=dev(), dtype=torch.int32)
    t = torch.randn(M, K, generator=g, device=dev()).to(BF)
    dl = torch.rand(M, generator=g, device=dev()) + 0.1
    sample = [0, 1, 2, 3, 4, 5, 6, M // 2, M - 3, M - 2, M - 1]
    idx[1], dl[2] = -1, 0.0                 # padding
    idx[3, 5:] = idx[3, 0]                  # a token many times
    idx[M - 2, ::2] = idx[M - 2, 1]
    idx[4, :3], idx[4, 3:] = torch.tensor([0, V - 1, V // 2], device=dev(), dtype=torch.int32), -1
    z[5, :V // 2] = -INF                    # tokens that the student is denied
    idx[5] = V - 1 - torch.arange(K, device=dev(), dtype=torch.int32)
    z[1], z[2, 7] = float("nan"), INF       # what padding holds
    tau = 1.5
    loss, dz = torch.full((M,), -1.0, device=dev()), torch.full((M, V), 7.0, dtype=dt, device=dev())
    mmf.mmf_distill_bwd(z, idx, t, tau, dl, dz, loss)
    # below the size, from rows of the same alignment
    some, parts = M // 3 // 8 * 8, torch.full((M, V), 3.0, dtype=dt, device=dev())
    ploss = torch.empty_like(loss)
    for a, b in ((0, some), (some, 2 * some), (2 * some, M)):
        assert (b - a) * V * size < LAST_LEVEL
        mmf.mmf_distill_bwd(z[a:b], idx[a:b], t[a:b], tau, dl[a:b], parts[a:b], ploss[a:b])
    assert torch.equal(dz, parts) and torch.equal(loss.nan_to_num(-9.0), ploss.nan_to_num(-9.0))
    rows = torch.tensor(sample, device=dev())
    ref = z[rows].cpu()
    ref[1] = ref[2] = 0.0
    want, dwant, q, _ = reference(ref, idx[rows].cpu(), t[rows].cpu(), tau, dl[rows].cpu())
    keep = [i for i in range(len(sample)) if i != 2]     # the loss of row 2 is that of its infinity
    assert loss[2].isnan()
    err = (loss[rows].cpu().double() - want).abs()
    assert (err <= 160 * U * tau * tau + U * want.abs())[keep].all()
    half = torch.finfo(dt).eps / 2
    w = dl[rows].cpu().double()[:, None] * tau
    bound = w * (160 * U * q + 2.0 ** -43 * q.amax(1, keepdim=True)) * (1 + half) + (half + U) * dwant.abs() + 1e-38
    assert ((dz[rows].cpu().double() - dwant).abs() <= bound).all()
    if dt == BF:
        mmf.mmf_distill_bwd(z, idx, t, tau, dl, z)       # in place, without the loss
        assert torch.equal(z, dz)


@pytest.mark.gpu
@pytest.mark.parametrize("W", [2, 4, 5, 7, 8, 9, 16, 33, 64])
def test_streamed_states(mmf, W):
    """Two arrays of rows of different sizes, one past 256 MB by itself: in place,
    into others, and one of each."""
    B, words = 3, (LAST_LEVEL // (4 * 3 * W) // 4 + 5) * 4
    log(f"[beam stream] W={W} {4 * words} bytes per row")
    g = torch.Generator(device="cuda").manual_seed(W)
    x = torch.randint(0, 2 ** 31 - 1, (B * W, words), generator=g, dtype=torch.int32, device=dev())
    y = torch.randint(0, 2 ** 31 - 1, (B * W, 260), generator=g, dtype=torch.int32, device=dev())
    parents = torch.randint(0, W, (B, W), generator=g, dtype=torch.int32, device=dev())
    parents[1] = torch.arange(W, device=dev())           # all stay
    parents[2, 0] = W                                    # no beam: stays
    src = parents.long().clamp(0, W - 1)
    src[2, 0] = 0
    src = (src + W * torch.arange(B, device=dev())[:, None]).reshape(-1)
    want_x, want_y = x[src], y[src]
    ox, oy = torch.full_like(x, -1), torch.full_like(y, -1)
    mmf.mmf_beam_reorder([x, y], parents, B, W, [ox, oy])
    assert torch.equal(ox, want_x) and torch.equal(oy, want_y)
    oy.fill_(-1)
    keep = x.clone()
    mmf.mmf_beam_reorder([x, y], parents, B, W, [x, oy])
    assert torch.equal(x, want_x) and torch.equal(oy, want_y)
    x.copy_(keep)
    mmf.mmf_beam_reorder([x, y], parents, B, W)
    assert torch.equal(x, want_x) and torch.equal(y, want_y)
