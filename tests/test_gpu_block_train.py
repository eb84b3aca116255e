"""A training step of a whole block of the model, as a user's program would
write it from the entry points: residual addition + quantisation, the MLGRU
token mixer, again residual + quantisation, the GLU channel mixer, the loss's
gradient back through all of it, the global norm and the clipped gradients;
against the same block in 64 bits (CPU, autograd, straight-through quantisers).

Tolerance: the gradients pass through bfloat16 (half a step 2^-8) at the
entry of each layer's backward and in its Yq; the longest way to a gradient
(the token mixer's input projections) has the loss's gradient, the GLU's down-
projection, the gate, the token mixer's output projection and z: with Yq, six
roundings, and each can pass to a result at most once per way in 2-norm.
Quantised activations next to a midpoint may fall to the other side of it,
one of 127 steps of a few values: 2^-8 more for each of the four quantisers.
"""
import pytest
import torch

from _parity import dev

BF, F32 = torch.bfloat16, torch.float32
TOL = (6 + 4) * 2.0 ** -8


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def params(B, T, d, L, seed=0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s, k=1.0: torch.randn(s, generator=g) * k  # noqa: E731
    return {"x": rand(B * T, d), "b": rand(B * T, d), "lb": torch.rand(d, generator=g) * 0.9,
            "gamma1": torch.rand(d, generator=g) + 0.5, "Wfcg": rand(3 * d, d, k=0.05), "bfcg": rand(3 * d, k=0.2),
            "gamma_o": torch.rand(d, generator=g) + 0.5, "Wo": rand(d, d, k=0.05),
            "gamma2": torch.rand(d, generator=g) + 0.5, "Wgu": rand(2 * L, d, k=0.05),
            "gamma_d": torch.rand(L, generator=g) + 0.5, "Wd": rand(d, L, k=0.05), "dout": rand(B * T, d)}


class Block:
    """The framework's side; every buffer made once."""

    def __init__(self, mmf, p, B, T, d, L):
        self.mmf, self.B, self.T, self.d, self.L = mmf, B, T, d, L
        self.p = {k: v.to(dev()) for k, v in p.items()}
        M = B * T
        e = lambda *s, dtype=F32: torch.empty(s, dtype=dtype, device=dev())  # noqa: E731
        i8, i32 = torch.int8, torch.int32
        self.s1, self.q1, self.a1, self.rs1, self.r1 = e(M, d), e(M, d, dtype=i8), e(M), e(M, dtype=i32), e(M)
        self.z, self.Wp1, self.w1 = e(M, 3 * d), e(d // 16, 3 * d, dtype=i32), e(1)
        self.o, self.states = e(M, d), e(mmf.mmf_mlgru_train_states_bytes(B, T, d), dtype=torch.uint8)
        self.y, self.Wp_o, self.w_o, self.q_o, self.a_o, self.r_o = \
            e(M, d), e(d // 16, d, dtype=i32), e(1), e(M, d, dtype=i8), e(M), e(M)
        self.s2, self.q2, self.a2, self.rs2, self.r2 = e(M, d), e(M, d, dtype=i8), e(M), e(M, dtype=i32), e(M)
        self.pp, self.Wp2, self.w2 = e(M, L), e(d // 16, 2 * L, dtype=i32), e(1)
        self.y2, self.Wp_d, self.w_d, self.q_d, self.a_d, self.r_d = \
            e(M, d), e(L // 16, d, dtype=i32), e(1), e(M, L, dtype=i8), e(M), e(M)
        self.out = e(M, d)
        self.dz, self.dp, self.ds2, self.do, self.ds1 = e(M, 3 * d, dtype=BF), e(M, L), e(M, d), e(M, d), e(M, d)
        self.grads = {k: torch.empty_like(self.p[k]) for k in
                      ("Wfcg", "bfcg", "Wo", "Wgu", "Wd", "gamma1", "gamma2", "gamma_o", "gamma_d", "lb")}
        self.norm = e(1)
        n = max(mmf.mmf_bitlinear_train_workspace_bytes(M, d, 3 * d), mmf.mmf_bitlinear_bwd_workspace_bytes(M, d, 3 * d),
                mmf.mmf_bitlinear_train_workspace_bytes(M, L, d), mmf.mmf_bitlinear_bwd_workspace_bytes(M, L, d),
                mmf.mmf_glu_train_workspace_bytes(M, d, L), mmf.mmf_glu_bwd_workspace_bytes(M, d, L),
                mmf.mmf_mlgru_scan_bwd_workspace_bytes(B, T, d),
                mmf.mmf_grad_norm_workspace_bytes([g.numel() for g in self.grads.values()]))
        self.ws = e(n, dtype=torch.uint8)

    def step(self, max_norm):
        m, p, g, B, T, ws = self.mmf, self.p, self.grads, self.B, self.T, self.ws
        # forward
        m.mmf_add_act_quant(p["x"], p["b"], p["gamma1"], self.s1, self.q1, self.a1, self.rs1, self.r1)
        m.mmf_bitlinear_train_fwd(self.s1, p["gamma1"], p["Wfcg"], p["bfcg"], self.z, self.Wp1, self.w1, self.q1,
                                  self.a1, self.r1, ws)
        m.mmf_mlgru_train_scan(self.z, B, T, p["lb"], None, self.o, None, self.states, ws)
        m.mmf_bitlinear_train_fwd(self.o, p["gamma_o"], p["Wo"], None, self.y, self.Wp_o, self.w_o, self.q_o, self.a_o,
                                  self.r_o, ws)
        m.mmf_add_act_quant(self.s1, self.y, p["gamma2"], self.s2, self.q2, self.a2, self.rs2, self.r2)
        m.mmf_glu_train_fwd(self.q2, self.a2, self.rs2, p["Wgu"], self.pp, self.Wp2, self.w2, ws)
        m.mmf_bitlinear_train_fwd(self.pp, p["gamma_d"], p["Wd"], None, self.y2, self.Wp_d, self.w_d, self.q_d,
                                  self.a_d, self.r_d, ws)
        torch.add(self.s2, self.y2, out=self.out)
        # backward
        m.mmf_bitlinear_bwd(p["dout"].to(BF), self.pp, p["gamma_d"], self.r_d, self.q_d, self.a_d, self.Wp_d, self.w_d,
                            self.dp, g["Wd"], None, g["gamma_d"], ws)
        m.mmf_glu_bwd(self.dp, self.s2, p["gamma2"], self.r2, self.q2, self.a2, self.rs2, self.Wp2, self.w2, self.ds2,
                      g["Wgu"], g["gamma2"], ws)
        self.ds2.add_(p["dout"])
        m.mmf_bitlinear_bwd(self.ds2.to(BF), self.o, p["gamma_o"], self.r_o, self.q_o, self.a_o, self.Wp_o, self.w_o,
                            self.do, g["Wo"], None, g["gamma_o"], ws)
        m.mmf_mlgru_scan_bwd(self.z, B, T, p["lb"], self.states, self.do, None, self.dz, None, g["lb"], ws)
        m.mmf_bitlinear_bwd(self.dz, self.s1, p["gamma1"], self.r1, self.q1, self.a1, self.Wp1, self.w1, self.ds1,
                            g["Wfcg"], g["bfcg"], g["gamma1"], ws)
        self.ds1.add_(self.ds2)
        grads = list(g.values())
        m.mmf_grad_norm(grads, self.norm, ws)
        m.mmf_grad_clip(grads, self.norm, max_norm)

    def results(self):
        return {"out": self.out, "x": self.ds1, "norm": self.norm, **self.grads}


def reference(p, B, T, d, L):
    """The block in 64 bits: values and unclipped gradients."""
    v = {k: x.double() for k, x in p.items()}
    leaves = [k for k in v if k not in ("dout", "b")]
    for k in leaves:
        v[k].requires_grad_(True)

    def quant(s, gamma):
        y = s * (1.0 / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-6)) * gamma
        a = y.detach().abs().amax(1, keepdim=True).clamp_min(1e-5)
        return y + ((y * (127.0 / a)).round() * (a / 127.0) - y).detach()

    def layer(s, gamma, W):
        ws = W.detach().abs().mean()
        t = W + ((W / ws).round().clamp(-1, 1) * ws - W).detach()
        return quant(s, gamma) @ t.t()

    s1 = v["x"] + v["b"]
    z = (layer(s1, v["gamma1"], v["Wfcg"]) + v["bfcg"]).reshape(B, T, 3, d)
    f = v["lb"] + (1 - v["lb"]) * torch.sigmoid(z[:, :, 0])
    c = z[:, :, 1] * torch.sigmoid(z[:, :, 1])
    h, hs = torch.zeros((B, d), dtype=torch.float64), []
    for t in range(T):
        h = f[:, t] * h + (1 - f[:, t]) * c[:, t]
        hs.append(h)
    o = (z[:, :, 2] * torch.sigmoid(torch.stack(hs, 1))).reshape(B * T, d)
    s2 = s1 + layer(o, v["gamma_o"], v["Wo"])
    gu = layer(s2, v["gamma2"], v["Wgu"])
    out = s2 + layer(gu[:, :L] * torch.sigmoid(gu[:, :L]) * gu[:, L:], v["gamma_d"], v["Wd"])
    (out * v["dout"]).sum().backward()
    return out.detach(), {k: v[k].grad for k in leaves}


def rel(a, b):
    return float((a.cpu().double() - b).norm() / b.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,d,L", [(2, 70, 128, 352), (1, 9, 64, 160)])
def test_a_step_of_a_block(mmf, B, T, d, L):
    p = params(B, T, d, L)
    out, want = reference(p, B, T, d, L)
    blk = Block(mmf, p, B, T, d, L)
    blk.step(1e9)  # nothing to clip
    torch.cuda.synchronize()
    got = blk.results()
    assert rel(got["out"], out) <= 4 * 2.0 ** -8
    for k, w in want.items():
        if k != "x":
            assert rel(got[k], w) <= TOL, k
    assert rel(got["x"], want["x"]) <= TOL
    total = float(sum(got[k].double().square().sum() for k in blk.grads)) ** 0.5
    assert abs(float(blk.norm) - total) <= 2.0 ** -23 * total
    full = {k: g.clone() for k, g in blk.grads.items()}
    # clipped to a tenth: every gradient, by one factor
    blk.step(total / 10)
    torch.cuda.synchronize()
    for k, g in blk.grads.items():
        assert torch.allclose(g, full[k] * 0.1, rtol=1e-5, atol=0)


@pytest.mark.gpu
def test_a_captured_step_replays(mmf):
    B, T, d, L = 2, 70, 128, 352
    blk = Block(mmf, params(B, T, d, L, 1), B, T, d, L)
    blk.step(1.0)
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in blk.results().items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blk.step(1.0)
    for _ in range(3):
        for v in blk.results().values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in blk.results().items():
            assert torch.equal(v, want[k]), k
