"""The training operators on a stream that is not the current one.  Every output
starts as NaN (or -1), and the current stream holds some tens of milliseconds
of other work, behind which a call that went there would still be waiting when
the given stream is done and its outputs are compared on it."""
import pytest
import torch

from _parity import dev, log

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def wipe(outs):
    for t in outs:
        t.fill_(float("nan") if t.is_floating_point() else -1)


def check(step, outs):
    """step(stream): on the current stream, then on two others."""
    wipe(outs)
    step(None)
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    assert not any(t.isnan().any() for t in want if t.is_floating_point())
    busy = torch.ones(1 << 29, device=dev())
    for _ in range(2):
        st = torch.cuda.Stream()
        wipe(outs)
        torch.cuda.synchronize()
        for _ in range(50):  # 4 GB each
            busy.mul_(1.0)
        step(st)
        with torch.cuda.stream(st):
            same = [torch.equal(t, w) for t, w in zip(outs, want)]
        assert all(same)
        torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [40, 700])  # the K-split and the tiled contraction
def test_glu(mmf, M):
    K, L = 512, 528
    log(f"[streams] glu M={M} K={K} L={L}")
    gen = torch.Generator(device="cuda").manual_seed(31)
    rand = lambda *s: torch.randn(s, generator=gen, device=dev())  # noqa: E731
    e = lambda *s, dtype=F32: torch.empty(s, dtype=dtype, device=dev())  # noqa: E731
    x, gamma, W, dp = rand(M, K).to(BF), rand(K).abs() + 0.5, rand(2 * L, K) * 0.02, rand(M, L)
    _, q, a, rs, r = mmf.add_act_quant(x, None, gamma)
    p, Wp, ws = e(M, L), e(K // 16, 2 * L, dtype=torch.int32), e(1)
    dx, dW, dgamma, dgu = e(M, K), e(2 * L, K), e(K), e(M, 2 * L, dtype=BF)
    Wg, sg = mmf.ternarize(W[:L].contiguous())
    Wu, su = mmf.ternarize(W[L:].contiguous())
    Wgu, w2 = mmf.glu_pack(Wg, Wu), torch.cat([sg, su])
    n = max(mmf.mmf_glu_train_workspace_bytes(M, K, L), mmf.mmf_glu_bwd_workspace_bytes(M, K, L))

    for work in (e(n, dtype=torch.uint8), None):  # the caller's workspace, or the call's own
        def step(stream):
            mmf.mmf_glu_train_fwd(q, a, rs, W, p, Wp, ws, work, stream)
            mmf.mmf_glu_bwd(dp, x, gamma, r, q, a, rs, Wp, ws, dx, dW, dgamma, work, stream)
            mmf.mmf_glu_gate_bwd(q, a, rs, Wgu, w2, dp, dgu, stream)

        check(step, (p, Wp, ws, dx, dW, dgamma, dgu))


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [((7,), (), (301, 33)), ((300, 401), (7,), (), (3, 5, 77777))], ids=["small", "large"])
def test_norm_and_clip(mmf, sizes):
    log(f"[streams] norm and clip {sizes}")
    gen = torch.Generator(device="cuda").manual_seed(32)
    grads = [torch.randn(s, generator=gen, device=dev()).to(BF if i % 2 else F32) for i, s in enumerate(sizes)]
    outs = [torch.empty_like(g) for g in grads]
    norm = torch.empty(1, device=dev())
    n = mmf.mmf_grad_norm_workspace_bytes([g.numel() for g in grads])
    for work in (torch.empty(n, dtype=torch.uint8, device=dev()), None):
        def step(stream):
            mmf.mmf_grad_norm(grads, norm, work, stream)
            mmf.mmf_grad_clip(grads, norm, 1.0, outs, stream)

        check(step, [norm] + outs)
