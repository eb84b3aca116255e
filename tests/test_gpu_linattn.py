"""Linear attention with a decay per head against the recurrence in 64 bits.

Error bounds per output, with A the same sums over the magnitudes of their
terms (|q|, |k|, |v|, |l|, |s0|), u = 2^-24 and h = 2^-8 (half a step of bf16):
  - fp32 sums: fewer than 8 roundings per term on its way into a chunk's sums
    and products, then one for each of at most T + 4 joins and the d of the
    query's product: (T + d + 16) u A;
  - fp32 factors as three bf16 parts: 3 x 2^-24 per factor and, for what the
    products leave out, 4 x 2^-24 per product: below 32 u A in all;
  - bf16 outputs: two parts, 3 x 2^-16 for each of the two products that
    follow one another and 2^-16 for each of their three fp32 factors: 9 x
    2^-16 A; then the rounding, h |o|.  fp32 inputs (backward): three factors
    more;
  - the backward's sums are the forward's with the roles exchanged.
"""
import pytest
import torch

from _parity import dev, log

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U, H8 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def inputs(B, T, H, dk, dv, t, seed=0, s0=True, decay=None):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    if decay is None:
        decay = 1.0 - 2.0 ** -(1 + 8 * torch.rand(H, generator=g))
    return {"qkv": rand(B * T, H * (2 * dk + dv)).to(t), "decay": torch.as_tensor(decay, dtype=F32),
            "s0": rand(B, H, dk, dv) if s0 else None, "dout": rand(B * T, H * dv),
            "ds_last": rand(B, H, dk, dv), "scale": dk ** -0.5, "dims": (B, T, H, dk, dv)}


def forward(p, f=lambda x: x):
    """o and the last state in 64 bits; f: applied to every input (abs for A)."""
    B, T, H, dk, dv = p["dims"]
    x = f(p["qkv"].to(F64)).reshape(B, T, -1)
    q, k, v = (y.reshape(B, T, H, -1) for y in x.split([H * dk, H * dk, H * dv], 2))
    l = f(p["decay"].to(F64))[None, :, None, None]
    S = torch.zeros(B, H, dk, dv, dtype=F64) if p["s0"] is None else f(p["s0"].to(F64))
    o = []
    for t in range(T):
        S = l * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        o.append(p["scale"] * (q[:, t, :, :, None] * S).sum(2))
    return torch.stack(o, 1).reshape(B * T, H * dv) if T else torch.zeros(0, H * dv, dtype=F64), S


def backward(p, f=lambda x: x):
    B, T, H, dk, dv = p["dims"]
    x = f(p["qkv"].to(F64)).reshape(B, T, -1)
    q, k, v = (y.reshape(B, T, H, -1) for y in x.split([H * dk, H * dk, H * dv], 2))
    do = f(p["dout"].to(F64)).reshape(B, T, H, dv)
    l, sc = f(p["decay"].to(F64))[None, :, None, None], p["scale"]
    S = torch.zeros(B, H, dk, dv, dtype=F64) if p["s0"] is None else f(p["s0"].to(F64))
    dq, dk_, dv_ = [], [None] * T, [None] * T
    for t in range(T):
        S = l * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        dq.append(sc * (S * do[:, t, :, None, :]).sum(3))
    G = torch.zeros_like(S) if p["ds_last"] is None else f(p["ds_last"].to(F64))
    for t in reversed(range(T)):
        G = G + sc * q[:, t, :, :, None] * do[:, t, :, None, :]
        dk_[t], dv_[t] = (G * v[:, t, :, None, :]).sum(3), (G * k[:, t, :, :, None]).sum(2)
        G = l * G
    rows = lambda xs, w: torch.stack(xs, 1).reshape(B * T, H * w)  # noqa: E731
    return torch.cat([rows(dq, dk), rows(dk_, dk), rows(dv_, dv)], 1), G


def up(x):
    return None if x is None else x.to(dev())


def run_fwd(mmf, p, s_last=True, ws=None, stream=None):
    B, T, H, dk, dv = p["dims"]
    qkv = up(p["qkv"])
    o = torch.full((B * T, H * dv), float("nan"), dtype=qkv.dtype, device=dev())
    s = torch.full((B, H, dk, dv), float("nan"), device=dev()) if s_last else None
    mmf.mmf_linattn_fwd(qkv, B, T, H, dk, dv, up(p["decay"]), p["scale"], up(p["s0"]), o, s, ws, stream)
    torch.cuda.synchronize()
    return o.cpu(), None if s is None else s.cpu()


def run_bwd(mmf, p, do_t=F32, ds0=True):
    B, T, H, dk, dv = p["dims"]
    dqkv = torch.full((B * T, H * (2 * dk + dv)), float("nan"), dtype=BF, device=dev())
    g = torch.full((B, H, dk, dv), float("nan"), device=dev()) if ds0 else None
    mmf.mmf_linattn_bwd(up(p["qkv"]), B, T, H, dk, dv, up(p["decay"]), p["scale"], up(p["s0"]), up(p["dout"]).to(do_t),
                        up(p["ds_last"]), dqkv, g)
    torch.cuda.synchronize()
    return dqkv.cpu(), None if g is None else g.cpu()


def within(got, want, bound, what):
    err = (got.to(F64) - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float((err / bound.clamp_min(1e-300)).max()):.3g} of its bound"


def check_fwd(p, o, s):
    B, T, H, dk, dv = p["dims"]
    (want, S), (A, SA) = forward(p), forward(p, torch.abs)
    f32 = (T + dk + 48) * U
    if o.dtype == F32:
        within(o, want, f32 * A + 1e-37, "o")
    else:
        within(o, want, (f32 + 9 * 2.0 ** -16) * A + H8 * (want.abs() + 9 * 2.0 ** -16 * A) + 1e-37, "o")
    if s is not None:
        within(s, S, f32 * SA + 1e-37, "s_last")


def check_bwd(p, dqkv, g):
    B, T, H, dk, dv = p["dims"]
    (want, G), (A, GA) = backward(p), backward(p, torch.abs)
    f32 = (T + max(dk, dv) + 48) * U + 12 * 2.0 ** -16
    within(dqkv, want, f32 * A + H8 * (want.abs() + f32 * A) + 1e-37, "dqkv")
    if g is not None:
        within(g, G, (T + dk + 48) * U * GA + 1e-37, "ds0")


SHAPES = [(1, 1, 1, 16, 16), (2, 1, 3, 128, 128), (5, 3, 2, 48, 80), (1, 16, 2, 256, 256), (2, 17, 1, 16, 16),
          (1, 33, 2, 64, 64), (2, 64, 1, 128, 64), (1, 65, 3, 64, 128), (1, 127, 1, 80, 112), (3, 200, 2, 112, 48),
          (1, 97, 1, 256, 16), (1, 130, 1, 16, 256), (1, 70, 1, 256, 256), (1, 70, 2, 144, 208), (1, 700, 2, 128, 128),
          (2, 1000, 1, 64, 96)]


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(mmf, shape, t):
    log(f"[linattn] {shape} {t}")
    p = inputs(*shape, t, seed=sum(shape), s0=sum(shape) % 3 != 0)
    check_fwd(p, *run_fwd(mmf, p))


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("do_t", [F32, BF], ids=["do_f32", "do_bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(mmf, shape, t, do_t):
    log(f"[linattn] backward {shape} {t} {do_t}")
    p = inputs(*shape, t, seed=1 + sum(shape), s0=sum(shape) % 3 != 0)
    p["dout"] = p["dout"].to(do_t)
    if sum(shape) % 2:
        p["ds_last"] = None
    check_bwd(p, *run_bwd(mmf, p, do_t))
