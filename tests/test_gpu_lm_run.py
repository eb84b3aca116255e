"""Linear attention, beam search and distillation as a program runs them: on
streams other than the current one, in captured graphs whose inputs change
between replays, two calls at once, and together with the layers around them."""
import pytest
import torch

from _parity import dev, log
from test_gpu_beam import reference as beam_reference
from test_gpu_distill import reference as distill_reference
from test_gpu_linattn import check_bwd, check_fwd
from test_gpu_train_streams import check as check_streams

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def e(*s, dtype=F32):
    return torch.empty(s, dtype=dtype, device=dev())


class Linattn:
    """(B, T, H, dk, dv, type): the forward and the backward."""

    def __init__(self, mmf, gen, dims, t, own_ws):
        B, T, H, dk, dv = self.dims = dims
        r = lambda *s: torch.randn(s, generator=gen, device=dev())  # noqa: E731
        self.mmf, self.decay = mmf, torch.rand(H, generator=gen, device=dev())
        self.ins = [r(B * T, H * (2 * dk + dv)).to(t), r(B, H, dk, dv), r(B * T, H * dv).to(t), r(B, H, dk, dv)]
        self.outs = [e(B * T, H * dv, dtype=t), e(B, H, dk, dv), e(B * T, H * (2 * dk + dv), dtype=BF), e(B, H, dk, dv)]
        n = max(mmf.mmf_linattn_workspace_bytes(*dims), mmf.mmf_linattn_bwd_workspace_bytes(*dims))
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device=dev()) if own_ws else None

    def __call__(self, stream=None):
        (x, s0, do, ds), (o, s, d, g) = self.ins, self.outs
        self.mmf.mmf_linattn_fwd(x, *self.dims, self.decay, 0.25, s0, o, s, self.ws, stream)
        self.mmf.mmf_linattn_bwd(x, *self.dims, self.decay, 0.25, s0, do, ds, d, g, self.ws, stream)


class Beam:
    def __init__(self, mmf, gen, dims, t, own_ws):
        B, W, V, n = self.dims = dims
        self.mmf = mmf
        r = lambda *s: torch.randn(s, generator=gen, device=dev())  # noqa: E731
        self.done = (torch.rand(B, W, generator=gen, device=dev()) < 0.2).to(torch.uint8)
        self.ins = [r(B * W, V).to(t), -r(B, W).abs(), r(B * W, 1024), r(B * W, 4, 8).to(BF)]
        i = torch.int32
        self.outs = [e(B, n), e(B, n, dtype=i), e(B, n, dtype=i), e(B * W, 1024), e(B * W, 4, 8, dtype=BF)]
        self.new_done = e(B, n, dtype=torch.uint8)
        self.ws = (torch.full((mmf.mmf_beam_select_workspace_bytes(*dims),), 255, dtype=torch.uint8, device=dev())
                   if own_ws else None)

    def __call__(self, stream=None):
        (z, s, h, c), (ns, tok, par, h2, c2) = self.ins, self.outs
        B, W, V, n = self.dims
        self.mmf.mmf_beam_select(z, s, self.done, 1, B, W, n, ns, tok, par, self.new_done, self.ws, stream)
        self.mmf.mmf_beam_reorder([h, c], par, B, W, [h2, c2], stream)


class Distill:
    def __init__(self, mmf, gen, dims, t, own_ws):
        M, V, K = dims
        self.mmf = mmf
        r = lambda *s: torch.randn(s, generator=gen, device=dev())  # noqa: E731
        self.ins = [r(M, V).to(t), r(M, K), r(M)]
        self.idx = torch.randint(0, V, (M, K), generator=gen, device=dev(), dtype=torch.int32)
        self.outs = [e(M), e(M, V, dtype=t), e(M)]

    def __call__(self, stream=None):
        (z, t, dl), (loss, dz, loss2) = self.ins, self.outs
        self.mmf.mmf_distill_fwd(z, self.idx, t, 2.0, loss, stream)
        self.mmf.mmf_distill_bwd(z, self.idx, t, 2.0, dl, dz, loss2, stream)


CASES = [(Linattn, (3, 1, 2, 64, 64)), (Linattn, (2, 40, 3, 48, 80)), (Linattn, (1, 1500, 2, 128, 128)),
         (Beam, (3, 4, 5000, 4)), (Beam, (1, 8, 50001, 8)), (Distill, (5, 1000, 16)), (Distill, (3, 70001, 40))]


@pytest.mark.gpu
@pytest.mark.parametrize("own_ws", [True, False], ids=["workspace", "allocated"])
@pytest.mark.parametrize("kind,dims", CASES, ids=[f"{k.__name__}-{d}" for k, d in CASES])
def test_streams(mmf, kind, dims, own_ws):
    log(f"[lm streams] {kind.__name__} {dims} {own_ws}")
    gen = torch.Generator(device="cuda").manual_seed(3)
    step = kind(mmf, gen, dims, BF, own_ws)
    check_streams(step, step.outs)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind,dims", CASES, ids=[f"{k.__name__}-{d}" for k, d in CASES])
def test_captured(mmf, kind, dims, t):
    """Two graphs that share a workspace, replayed in turn with new inputs and
    eager work between; every replay has the bits of the eager call."""
    log(f"[lm graph] {kind.__name__} {dims} {t}")
    gen = torch.Generator(device="cuda").manual_seed(4)
    steps = [kind(mmf, gen, dims, t, True) for _ in range(2)]
    if hasattr(steps[0], "ws"):
        steps[1].ws = steps[0].ws
    graphs = []
    for s in steps:
        s()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s()
    for _ in range(3):
        for s, graph in zip(steps, graphs):
            for x in s.ins:
                x.copy_(torch.randn(x.shape, generator=gen, device=dev()))
            s()
            want = [o.clone() for o in s.outs]
            for o in s.outs:
                o.fill_(-1)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(s.outs, want))


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dims", [CASES[2], CASES[4], CASES[6]], ids=["linattn", "beam", "distill"])
def test_two_at_once(mmf, kind, dims):
    """Two streams, each with memory of its own, not waiting for each other."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    steps = [kind(mmf, gen, dims, BF, i == 0) for i in range(2)]
    for s in steps:
        s()
    torch.cuda.synchronize()
    want = [[o.clone() for o in s.outs] for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    for s in steps:
        for o in s.outs:
            o.fill_(-1)
    torch.cuda.synchronize()
    for _ in range(10):
        for s, st in zip(steps, streams):
            s(st)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.outs, w))


class Layer:
    """A BitLinear's packed weights."""

    def __init__(self, mmf, gen, N, K):
        self.gamma = torch.rand(K, generator=gen, device=dev()) + 0.5
        self.Wp, self.ws = mmf.ternarize(torch.randn(N, K, generator=gen, device=dev()) * 0.05)
        self.mmf = mmf

    def __call__(self, x):
        return self.mmf.bitlinear(x, self.gamma, self.Wp, self.ws)


@pytest.mark.gpu
@pytest.mark.parametrize("H,dk,dv,W,V", [(2, 64, 64, 4, 1000), (3, 32, 48, 7, 5003)])
def test_beam_decoding(mmf, H, dk, dv, W, V):
    """Token mixers whose states are matrices and their MLGRU beside them, decoded
    by beam search: the states that end up at a beam are those of its own tokens,
    and its score is the sum over them."""
    log(f"[lm run] beam H={H} dk={dk} dv={dv} W={W} V={V}")
    gen = torch.Generator(device="cuda").manual_seed(6)
    B, d, steps, end = 2, 256, 12, 3
    embed = torch.randn(V, d, generator=gen, device=dev())
    qkv_of, out_of, head = (Layer(mmf, gen, n, k) for n, k in ((H * (2 * dk + dv), d), (d, H * dv), (V, d)))
    decay = torch.rand(H, generator=gen, device=dev()) * 0.5 + 0.5

    def step(tokens, S, h):
        x = embed[tokens.long()]
        o = e(B * W, H * dv)
        mmf.mmf_linattn_fwd(qkv_of(x), B * W, 1, H, dk, dv, decay, dk ** -0.5, S, o, S)
        y = x + out_of(o)
        # a recurrence beside it: h = (h + y) / 2, a state of another shape and type
        h.copy_(((h.float() + y) / 2).to(h.dtype))
        return head(y + h.float())

    S, h = torch.zeros(B * W, H, dk, dv, device=dev()), torch.zeros(B * W, d, dtype=BF, device=dev())
    hist = torch.zeros(B * W, 16, dtype=torch.int32, device=dev())
    scores = torch.full((B, W), float("-inf"), device=dev())
    scores[:, 0] = 0.0
    done = torch.zeros(B, W, dtype=torch.uint8, device=dev())
    tokens = torch.zeros(B * W, dtype=torch.int32, device=dev())
    for i in range(steps):
        z = step(tokens, S, h)
        ns, tok, par, nd = e(B, W), e(B, W, dtype=torch.int32), e(B, W, dtype=torch.int32), e(B, W, dtype=torch.uint8)
        mmf.mmf_beam_select(z, scores, done, end, B, W, W, ns, tok, par, nd)
        if i == 0:
            want = beam_reference(z.double().cpu().numpy().reshape(B, W, V), scores.cpu().numpy(), done.cpu().numpy(), end, W)
            assert (tok.cpu().numpy() == want["tokens"]).all()
        mmf.mmf_beam_reorder([S, h, hist], par, B, W)
        hist[:, i] = tok.reshape(-1)
        scores, done, tokens = ns, nd, tok.reshape(-1)
        assert (scores.diff(dim=1) <= 0).all()
    # every beam from the start, all rows its own tokens
    for row in range(B * W):
        line = hist[row, :steps].tolist()
        ended = line.index(end) if end in line else None
        assert bool(done.reshape(-1)[row]) == (ended is not None) and (ended is None or set(line[ended:]) == {end})
        S2, h2 = torch.zeros_like(S), torch.zeros_like(h)
        total, token = 0.0, 0
        for i, nxt in enumerate(line):
            z = step(torch.full((B * W,), token, dtype=torch.int32, device=dev()), S2, h2)
            if ended is None or i <= ended:
                total += float(torch.log_softmax(z[row].double(), 0)[nxt])
            token = nxt
        # 2^-17 per step (test_gpu_beam.py) and a rounding of the running score
        score = float(scores.reshape(-1)[row])
        assert abs(score - total) <= steps * (2.0 ** -17 + 2.0 ** -24 * abs(score))
        # the same kernels on the same rows: the same bits
        assert torch.equal(S[row], S2[row]) and torch.equal(h[row], h2[row])


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,dk,dv", [(37, 2, 64, 64), (300, 3, 48, 80)])
def test_training_step(mmf, T, H, dk, dv):
    """Projection, linear attention, output and un-embedding layers trained on a
    teacher's tokens: each link against its formula, and all of it captured."""
    log(f"[lm run] train T={T} H={H} dk={dk} dv={dv}")
    gen = torch.Generator(device="cuda").manual_seed(7)
    B, d, V, K = 2, 128, 1008, 16
    M, wide = B * T, H * (2 * dk + dv)
    r = lambda *s: torch.randn(s, generator=gen, device=dev())  # noqa: E731
    x, decay = r(M, d), torch.rand(H, generator=gen, device=dev())
    idx = torch.randint(0, V, (M, K), generator=gen, device=dev(), dtype=torch.int32)
    t, dl = r(M, K), torch.full((M,), 1.0 / M, device=dev())
    idx[5] = -1                                                # a row of padding

    class Train:
        def __init__(self, N, C):
            self.W, self.gamma = r(N, C) * 0.05, torch.rand(C, generator=gen, device=dev()) + 0.5
            self.y, self.Wp, self.ws = e(M, N), e(C // 16, N, dtype=torch.int32), e(1)
            self.q, self.a, self.rstd = e(M, C, dtype=torch.int8), e(M), e(M)
            self.dx, self.dW, self.dgamma = e(M, C), e(N, C), e(C)

        def fwd(self, v):
            self.x = v
            mmf.mmf_bitlinear_train_fwd(v, self.gamma, self.W, None, self.y, self.Wp, self.ws, self.q, self.a, self.rstd, ws)
            return self.y

        def bwd(self, dy):
            mmf.mmf_bitlinear_bwd(dy, self.x, self.gamma, self.rstd, self.q, self.a, self.Wp, self.ws, self.dx, self.dW, None,
                                  self.dgamma, ws)
            return self.dx

    n = max(mmf.mmf_linattn_workspace_bytes(B, T, H, dk, dv), mmf.mmf_linattn_bwd_workspace_bytes(B, T, H, dk, dv),
            *(f(M, a, b) for f in (mmf.mmf_bitlinear_bwd_workspace_bytes, mmf.mmf_bitlinear_train_workspace_bytes)
              for a, b in ((d, wide), (H * dv, d), (d, V))))
    ws = e(n, dtype=torch.uint8)
    proj, out, head = Train(wide, d), Train(d, H * dv), Train(V, d)
    o, loss, dz, dqkv = e(M, H * dv), e(M), e(M, V, dtype=BF), e(M, wide, dtype=BF)
    dy = e(M, d, dtype=BF)

    def step():
        mmf.mmf_linattn_fwd(proj.fwd(x), B, T, H, dk, dv, decay, dk ** -0.5, None, o, None, ws)
        z = head.fwd(out.fwd(o))
        mmf.mmf_distill_bwd(z, idx, t, 2.0, dl, dz, loss)
        dy.copy_(head.bwd(dz))
        mmf.mmf_linattn_bwd(proj.y, B, T, H, dk, dv, decay, dk ** -0.5, None, out.bwd(dy), None, dqkv, None, ws)
        proj.bwd(dqkv)

    outs = [o, loss, dz, dqkv] + [v for l in (proj, out, head) for v in (l.dx, l.dW, l.dgamma)]
    step()
    torch.cuda.synchronize()
    p = {"qkv": proj.y.cpu(), "decay": decay.cpu(), "s0": None, "ds_last": None, "scale": dk ** -0.5, "dout": out.dx.cpu(),
         "dims": (B, T, H, dk, dv)}
    check_fwd(p, o.cpu(), None)
    check_bwd(p, dqkv.cpu(), None)
    want, dwant, q, _ = distill_reference(head.y.cpu(), idx.cpu(), t.cpu(), 2.0, dl.cpu())
    U = 2.0 ** -24
    assert ((loss.cpu().double() - want).abs() <= 160 * U * 4 + U * want.abs()).all()
    bound = 2.0 / M * (160 * U * q + 2.0 ** -43) * 1.01 + (2.0 ** -8 + U) * dwant.abs() + 1e-38
    assert ((dz.cpu().double() - dwant).abs() <= bound).all()
    assert loss[5] == 0 and (dz[5] == 0).all()
    # the projection's gradient from dqkv: products of bf16 values are exact in
    # fp32, their sums take at most M roundings
    xq = (proj.q.float() * proj.a[:, None]).to(BF).cpu().double()
    g = dqkv.cpu().double().t()
    assert ((proj.dW.cpu().double() - g @ xq).abs() <= (M + 2) * U * (g.abs() @ xq.abs()) + 1e-37).all()
    first = [v.clone() for v in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.copy_(r(M, d))
        step()
        again = [v.clone() for v in outs]
        assert not torch.equal(again[0], first[0])
        for v in outs:
            v.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, again))
