"""The GLU channel mixer's training form: mmf_glu_train_fwd and mmf_glu_bwd
against the calls that they join (the same bits), and the gate's gradients
(mmf_glu_gate_bwd) against the formula in 64 bits.

With u = 2^-24: g and u are fl(acc) fl(a w), two roundings each (2u); the
hardware sigmoid carries e_s = s ((1 - s)(|g| + 2) + 3) u and, through g's
error, 2u |g| s (1 - s).  du = dp g s adds three roundings; dg = dp u q(g),
q = s (1 + g (1 - s)), carries e_s (1 + |g|) in q and, per operation, u of its
terms (1 - s rounds to half a step of 1).  Both are rounded once to bf16, half
a step of 2^-8.  The sigmoid's hardware reciprocal gives 0 for results below
the least normal number, MIN = 2^-126 (its operand 1 + e^-g is then above
2^126, at the latest an infinity): e_s is at least that, and so is each
result's error.
"""
import pytest
import torch

from _parity import dev, log

U, MIN = 2.0 ** -24, 2.0 ** -126
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def unpack(Wp, N):
    """Packed words [K/16][N] -> t [N][K] float64."""
    e = torch.arange(16, device=Wp.device, dtype=torch.int32)
    c = (Wp.t().reshape(N, -1, 1) >> (8 * (e % 4) + 2 * (e // 4))) & 3
    return c.reshape(N, -1).double() - 1


def inputs(mmf, seed, M, K, L, dt, xt=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device=dev())  # noqa: E731
    x = rand(M, K).to(xt)
    gamma = torch.rand(K, generator=g, device=dev()) + 0.5
    s, q, a, rs, r = mmf.add_act_quant(x, None, gamma)
    return {"x": x, "gamma": gamma, "q": q, "a": a, "rs": rs, "r": r, "W": rand(2 * L, K) * 0.02,
            "dp": rand(M, L).to(dt)}


def gate64(q, a, tg, tu, ws, dp):
    g = (q.double() @ tg.t()) * a.double()[:, None] * ws[0].double()
    u = (q.double() @ tu.t()) * a.double()[:, None] * ws[1].double()
    dp, s = dp.double(), torch.sigmoid(g)
    es = s * ((1 - s) * (g.abs() + 2) + 3) * U + 2 * U * g.abs() * s * (1 - s) + MIN
    du = dp * g * s
    edu = dp.abs() * (g.abs() * es + 5 * U * (g * s).abs())
    k = s * (1 + g * (1 - s))
    ek = es * (1 + g.abs()) + 3 * U * s * (1 + g.abs()) + 2 * U * (g * s * (1 - s)).abs()
    dg = dp * u * k
    edg = (dp * u).abs() * (ek + 5 * U * k.abs())
    want = torch.cat([dg, du], 1)
    return want, 1.01 * torch.cat([edg, edu], 1) + 2.0 ** -8 * want.abs() + MIN


def guarded(M, N, dtype):
    whole = torch.full((M + 2, N), 33, dtype=dtype, device=dev())
    return whole, whole[1:M + 1]


def check_gate(mmf, M, K, L, dt, path, seed=0):
    log(f"[glu_gate_bwd] M={M} K={K} L={L} dp={dt} path={path}")
    v = inputs(mmf, seed + M + K + L, M, K, L, dt)
    Wg, sg = mmf.ternarize(v["W"][:L].contiguous())
    Wu, su = mmf.ternarize(v["W"][L:].contiguous() * 3.0)  # another scale
    ws = torch.cat([sg, su])
    whole, dgu = guarded(M, 2 * L, BF)
    prev = mmf.mmf_set_path(path)
    try:
        mmf.mmf_glu_gate_bwd(v["q"], v["a"], v["rs"], mmf.glu_pack(Wg, Wu), ws, v["dp"], dgu)
    finally:
        mmf.mmf_set_path(prev)
    torch.cuda.synchronize()
    want, tol = gate64(v["q"], v["a"], unpack(Wg, L), unpack(Wu, L), ws, v["dp"])
    err = (dgu.double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())
    assert (whole[0] == 33).all() and (whole[-1] == 33).all()
    return dgu


# M, K, L and the tile that the planner takes for them on the tiled kernel;
# fewer rows take the K-split kernel on the automatic path
SIZES = [(1, 16, 16, "64x256"), (5, 48, 32, "64x256"), (37, 272, 304, "64x256"), (357, 1040, 2832, "64x256"),
         (1000, 336, 3008, "64x512"), (1100, 528, 4000, "128x512"), (3000, 400, 4112, "128x256_paired"),
         (129, 4112, 48, "64x256")]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,K,L,tile", SIZES)
def test_gate_gradients(mmf, M, K, L, tile, dt):
    assert mmf.mmf_prefill_tile_plan(M, K, 2 * L, mmf.MMF_EPILOGUE_GLU) == tile
    tiled = check_gate(mmf, M, K, L, dt, mmf.MMF_PATH_GEMM)
    assert torch.equal(check_gate(mmf, M, K, L, dt, mmf.MMF_PATH_AUTO), tiled)


# every row and column block count of the K-split kernel's tiles, K of less
# than one step per wave to more than two
@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,K,L", [(1, 2048, 5632), (16, 64, 2048), (17, 2048, 48), (33, 1040, 2832), (48, 528, 16),
                                   (64, 2048, 5632), (100, 2064, 1040), (128, 4112, 3008), (300, 272, 5632)])
def test_gate_gradients_of_few_rows(mmf, M, K, L, dt):
    few = check_gate(mmf, M, K, L, dt, mmf.MMF_PATH_AUTO)
    assert torch.equal(check_gate(mmf, M, K, L, dt, mmf.MMF_PATH_GEMM), few)


@pytest.mark.gpu
def test_row_slices(mmf):
    """q of more than 2^31 bytes: the rows of the second launch as in a call
    of their own."""
    M, K, L, n = 1_060_000, 2048, 32, 300
    g = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8, device=dev())
    a, rs = torch.rand(M, generator=g, device=dev()) * 0.01, q.sum(1, dtype=torch.int32)
    Wp, s = mmf.ternarize(torch.randn((2 * L, K), generator=g, device=dev()))
    dp = torch.randn((M, L), generator=g, device=dev())
    ws, tail = torch.tensor([0.5, 2.0], device=dev()), slice(M - n, M)
    dgu, one = (torch.empty((m, 2 * L), dtype=BF, device=dev()) for m in (M, n))
    mmf.mmf_glu_gate_bwd(q, a, rs, Wp, ws, dp, dgu)
    mmf.mmf_glu_gate_bwd(q[tail], a[tail].clone(), rs[tail].clone(), Wp, ws, dp[tail], one)
    assert torch.equal(dgu[tail], one)


@pytest.mark.gpu
def test_gate_gradients_far_out(mmf):
    """Gates where the sigmoid saturates, gradients of 0."""
    M, K, L = 70, 64, 48
    v = inputs(mmf, 1, M, K, L, F32)
    Wp, s = mmf.ternarize(v["W"])
    Wgu = mmf.glu_pack(Wp[:, :L].contiguous(), Wp[:, L:].contiguous())
    ws = torch.tensor([40.0, 0.5], device=dev())
    v["dp"][::3] = 0
    dgu = torch.empty((M, 2 * L), dtype=BF, device=dev())
    mmf.mmf_glu_gate_bwd(v["q"], v["a"], v["rs"], Wgu, ws, v["dp"], dgu)
    want, tol = gate64(v["q"], v["a"], unpack(Wp, 2 * L)[:L], unpack(Wp, 2 * L)[L:], ws, v["dp"])
    assert ((dgu.double() - want).abs() <= tol).all()
    assert (dgu[::3] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("xt,dt", [(BF, F32), (F32, BF)], ids=["xbf16", "xf32"])
@pytest.mark.parametrize("M,K,L", [(1, 16, 16), (37, 272, 304), (900, 512, 1040)])
def test_forward_and_backward_are_the_calls_they_join(mmf, M, K, L, xt, dt):
    v = inputs(mmf, 2, M, K, L, dt, xt)
    p, Wp, ws = torch.empty((M, L), device=dev()), torch.empty((K // 16, 2 * L), dtype=torch.int32, device=dev()), \
        torch.empty(1, device=dev())
    n = mmf.mmf_glu_train_workspace_bytes(M, K, L)
    work = torch.full((n + 256,), 0xAB, dtype=torch.uint8, device=dev())
    mmf.mmf_glu_train_fwd(v["q"], v["a"], v["rs"], v["W"], p, Wp, ws, work[:n])
    assert (work[n:] == 0xAB).all()
    Wp2, ws2 = mmf.ternarize(v["W"])
    assert torch.equal(Wp, Wp2) and torch.equal(ws, ws2)
    Wgu = mmf.glu_pack(Wp[:, :L].contiguous(), Wp[:, L:].contiguous())
    p2 = torch.empty_like(p)
    mmf.mmf_ternary_gemm_glu(v["q"], v["a"], v["rs"], Wgu, ws.repeat(2), p2)
    assert torch.equal(p, p2)
    assert torch.equal(p, mmf.glu(v["x"], v["gamma"], Wgu, ws.repeat(2)))

    dx, dW, dgamma = (torch.full(s, float("nan"), device=dev()) for s in ((M, K), (2 * L, K), (K,)))
    n = mmf.mmf_glu_bwd_workspace_bytes(M, K, L)
    work = torch.full((n + 256,), 0xAB, dtype=torch.uint8, device=dev())
    mmf.mmf_glu_bwd(v["dp"], v["x"], v["gamma"], v["r"], v["q"], v["a"], v["rs"], Wp, ws, dx, dW, dgamma, work[:n])
    assert (work[n:] == 0xAB).all()
    dgu = torch.empty((M, 2 * L), dtype=BF, device=dev())
    mmf.mmf_glu_gate_bwd(v["q"], v["a"], v["rs"], Wgu, ws.repeat(2), v["dp"], dgu)
    dx2, dW2, dgamma2 = torch.empty_like(dx), torch.empty_like(dW), torch.empty_like(dgamma)
    mmf.mmf_bitlinear_bwd(dgu, v["x"], v["gamma"], v["r"], v["q"], v["a"], Wp, ws, dx2, dW2, None, dgamma2)
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2) and torch.equal(dW, dW2) and torch.equal(dgamma, dgamma2)
    # without dgamma and workspace
    mmf.mmf_glu_bwd(v["dp"], v["x"], v["gamma"], v["r"], v["q"], v["a"], v["rs"], Wp, ws, dx2, dW2, None)
    assert torch.equal(dx, dx2) and torch.equal(dW, dW2)
    # dW: the product of the gate's gradients and the activations in bf16
    Y = (v["q"].float() * v["a"][:, None]).to(BF).double()
    want = dgu.double().t() @ Y
    tol = 2 * M * U * (dgu.double().abs().t() @ Y.abs()) + 1e-38
    assert ((dW.double() - want).abs() <= tol).all()


@pytest.mark.gpu
def test_on_another_stream_and_captured(mmf):
    M, K, L = 200, 512, 528
    v = inputs(mmf, 3, M, K, L, F32)
    p, Wp, ws = torch.zeros((M, L), device=dev()), torch.zeros((K // 16, 2 * L), dtype=torch.int32, device=dev()), \
        torch.zeros(1, device=dev())
    dx, dW, dgamma = (torch.zeros(s, device=dev()) for s in ((M, K), (2 * L, K), (K,)))
    outs = (p, Wp, ws, dx, dW, dgamma)
    n = max(mmf.mmf_glu_train_workspace_bytes(M, K, L), mmf.mmf_glu_bwd_workspace_bytes(M, K, L))
    work = torch.empty(n, dtype=torch.uint8, device=dev())

    def step(stream=None):
        mmf.mmf_glu_train_fwd(v["q"], v["a"], v["rs"], v["W"], p, Wp, ws, work, stream)
        mmf.mmf_glu_bwd(v["dp"], v["x"], v["gamma"], v["r"], v["q"], v["a"], v["rs"], Wp, ws, dx, dW, dgamma, work,
                        stream)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    st = torch.cuda.Stream()
    step(st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_formula_against_differences():
    """dg and du are the gradients of sum(dp SiLU(g) u)."""
    gen = torch.Generator().manual_seed(5)
    dp, g, u = (torch.randn(50, generator=gen, dtype=torch.float64) * 3 for _ in range(3))
    s, h = torch.sigmoid(g), 1e-6
    loss = lambda g, u: dp * g * torch.sigmoid(g) * u  # noqa: E731
    dg, du = dp * u * s * (1 + g * (1 - s)), dp * g * s
    assert ((loss(g + h, u) - loss(g - h, u)) / (2 * h) - dg).abs().max() < 1e-7
    assert ((loss(g, u + h) - loss(g, u - h)) / (2 * h) - du).abs().max() < 1e-7


A, BAD, S = 0x100000, 0x100004, None


def test_refusals(mmf):
    lib = mmf._lib
    wf, wb = mmf.mmf_glu_train_workspace_bytes(4, 32, 48), mmf.mmf_glu_bwd_workspace_bytes(4, 32, 48)
    assert wf > 0 and wb > 0 and wf % 256 == 0 and wb % 256 == 0

    def fwd(q=A, a=A, rs=A, W=A, p=A, Wp=A, s=A, M=4, K=32, L=48, ws=A, n=wf):
        return lib.mmf_glu_train_fwd(q, a, rs, W, p, Wp, s, M, K, L, ws, n, S)

    def gate(q=A, a=A, rs=A, W=A, s=A, dp=A, k=1, o=A, M=4, K=32, L=48):
        return lib.mmf_glu_gate_bwd(q, a, rs, W, s, dp, k, o, M, K, L, S)

    def bwd(dp=A, k=1, x=A, xk=0, g=A, r=A, q=A, a=A, rs=A, Wp=A, s=A, dx=A, dW=A, dg=A, M=4, K=32, L=48, ws=A, n=wb):
        return lib.mmf_glu_bwd(dp, k, x, xk, g, r, q, a, rs, Wp, s, dx, dW, dg, M, K, L, ws, n, S)

    for f in (fwd, gate, bwd):
        assert f(K=24) == 2 and f(L=24) == 2 and f(L=-16) == 2 and f(M=-1) == 2
        assert f(K=256, L=1 << 26) == 2 and f(M=65, K=16, L=1 << 20) == 2  # past the contraction's offsets
        for name in ("q", "a", "rs"):
            assert f(**{name: None}) == 1 and f(**{name: BAD}) == 3
        assert f(q=None, M=0) == 0 and f(q=None, L=0) == 0
    for name in ("W", "p", "Wp"):
        assert fwd(**{name: None}) == 1 and fwd(**{name: BAD}) == 3
    for name in ("W", "dp", "o"):
        assert gate(**{name: None}) == 1 and gate(**{name: BAD}) == 3
    for name in ("dp", "x", "r", "Wp", "dx", "dW"):
        assert bwd(**{name: None}) == 1 and bwd(**{name: BAD}) == 3
    assert fwd(s=None) == 1 and gate(s=None) == 1 and bwd(s=None) == 1 and bwd(g=BAD) == 3 and bwd(dg=BAD) == 3
    assert gate(k=2) == 4 and bwd(k=2) == 4 and bwd(xk=2) == 4
    assert fwd(n=wf - 1) == 6 and bwd(n=wb - 1) == 6 and fwd(ws=A + 16) == 6 and bwd(ws=A + 16) == 6
    assert bwd(K=2048, L=1 << 17) == 2 and mmf.mmf_glu_bwd_workspace_bytes(4, 2048, 1 << 17) == 0  # dW of 2^31 bytes
    assert mmf.mmf_glu_train_workspace_bytes(4, 32, 40) == 0
