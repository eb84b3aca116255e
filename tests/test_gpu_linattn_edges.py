"""Linear attention where it can go wrong: decays of every kind, states in place,
calls without tokens, values that are not finite, rows around the outputs,
offsets past 32 bits, gradients against differences, equal bits on repetition.
Error bounds as derived in test_gpu_linattn.py."""
import pytest
import torch

from _parity import dev, log
from test_gpu_linattn import (BF, F32, F64, H8, U, backward, check_bwd, check_fwd, forward, run_bwd, run_fwd, up, within)
from test_gpu_linattn import inputs as inputs_f32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def inputs(B, T, H, dk, dv, t, **kw):
    """With the gradient of o in the type of qkv."""
    p = inputs_f32(B, T, H, dk, dv, t, **kw)
    p["dout"] = p["dout"].to(t)
    return p


DECAYS = [0.0, 1.0, -1.0, -0.5, 1.02, 1e-30, -1e-6, 2.0 ** -126, 1.0 - 2.0 ** -24, 0.3]


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 5, 40, 129, 450])
def test_decays(mmf, T, t):
    log(f"[linattn] decays T={T} {t}")
    p = inputs(2, T, len(DECAYS), 32, 48, t, seed=T, decay=DECAYS)
    check_fwd(p, *run_fwd(mmf, p))
    check_bwd(p, *run_bwd(mmf, p, t))


@pytest.mark.gpu
@pytest.mark.parametrize("decay", [0.0, 0.9])
@pytest.mark.parametrize("T", [1, 2, 64, 200])
def test_without_states(mmf, T, decay):
    """No state before, none wanted after, no gradient of either."""
    for t in (F32, BF):
        p = inputs(1, T, 3, 64, 64, t, seed=T, s0=False, decay=[decay] * 3)
        p["ds_last"] = None
        check_fwd(p, *run_fwd(mmf, p, s_last=False))
        check_bwd(p, *run_bwd(mmf, p, t, ds0=False))


@pytest.mark.gpu
@pytest.mark.parametrize("B,T", [(0, 5), (3, 0)])
def test_no_tokens_change_nothing(mmf, B, T):
    p = inputs(B, T, 2, 16, 32, F32)
    s = torch.full((B, 2, 16, 32), 7.0, device=dev())
    g = s.clone()
    qkv = up(p["qkv"])
    mmf.mmf_linattn_fwd(qkv, B, T, 2, 16, 32, up(p["decay"]), 1.0, s, torch.empty(0, 64, device=dev()), s)
    mmf.mmf_linattn_bwd(qkv, B, T, 2, 16, 32, up(p["decay"]), 1.0, s, torch.empty(0, 64, device=dev()), g,
                        torch.empty(0, 128, dtype=BF, device=dev()), g)
    assert (s == 7).all() and (g == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(3, 1, 2, 128, 64), (2, 7, 3, 48, 80), (1, 100, 2, 256, 144), (1, 900, 3, 64, 128)])
def test_states_in_place_and_the_same_bits_again(mmf, B, T, H, dk, dv, t):
    log(f"[linattn] in place {B} {T} {H} {dk} {dv} {t}")
    p = inputs(B, T, H, dk, dv, t, seed=T)
    o, s = run_fwd(mmf, p)
    dqkv, g = run_bwd(mmf, p, t)
    qkv, decay, do = up(p["qkv"]), up(p["decay"]), up(p["dout"]).to(t)
    for _ in range(3):
        state, grad = up(p["s0"]), up(p["ds_last"])
        o2, dq2 = torch.empty_like(o, device=dev()), torch.empty_like(dqkv, device=dev())
        mmf.mmf_linattn_bwd(qkv, B, T, H, dk, dv, decay, p["scale"], state, do, grad, dq2, grad)
        mmf.mmf_linattn_fwd(qkv, B, T, H, dk, dv, decay, p["scale"], state, o2, state)
        assert torch.equal(state.cpu(), s) and torch.equal(o2.cpu(), o)
        assert torch.equal(grad.cpu(), g) and torch.equal(dq2.cpu(), dqkv)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 6, 50, 333])
def test_a_sequence_in_parts(mmf, T, t):
    """Token by token, and in two parts, the state carried along."""
    p = inputs(2, T, 2, 64, 48, t, seed=T)
    qkv, decay = up(p["qkv"]).reshape(2, T, -1), up(p["decay"])
    for cuts in ([1] * min(T, 9) + [T - min(T, 9)], [T // 2, T - T // 2]):
        s, at, parts = up(p["s0"]), 0, []
        for n in cuts:
            o = torch.empty(2 * n, 96, dtype=t, device=dev())
            mmf.mmf_linattn_fwd(qkv[:, at:at + n].reshape(2 * n, 352).contiguous(), 2, n, 2, 64, 48, decay, p["scale"], s, o, s)
            parts.append(o.reshape(2, n, 96))
            at += n
        check_fwd(p, torch.cat(parts, 1).reshape(2 * T, 96).cpu(), s.cpu())


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,at", [(1, 0), (6, 3), (100, 0), (100, 70), (700, 300), (64, 63)])
@pytest.mark.parametrize("part", ["q", "k", "v"])
def test_what_is_not_finite_stays_where_it_belongs(mmf, part, T, at, t):
    log(f"[linattn] not finite {part} T={T} at {at} {t}")
    B, H, dk, dv = 2, 2, 32, 48
    p = inputs(B, T, H, dk, dv, t, seed=T + at, decay=[0.9, 0.5])
    clean = p["qkv"]
    o_clean, s_clean = run_fwd(mmf, p)
    d_clean, g_clean = run_bwd(mmf, p, t)
    col = {"q": 0, "k": H * dk, "v": 2 * H * dk}[part] + (dv if part == "v" else dk) + 5   # of head 1
    for value in (float("nan"), float("inf"), -float("inf")):
        p["qkv"] = clean.clone()
        p["qkv"][T + at, col] = value                                                      # sequence 1
        o, s = run_fwd(mmf, p)
        dqkv, g = run_bwd(mmf, p, t)
        want, S = forward(p)
        dwant, G = backward(p)
        heads = lambda x: x.reshape(B, T, H, -1)  # noqa: E731
        # where the formula is not finite, neither is the result
        for got, ref in ((o, want), (s, S), (dqkv, dwant), (g, G)):
            assert not got[~ref.isfinite()].isfinite().any()
        # other sequences and heads: the same bits
        assert torch.equal(heads(o)[0], heads(o_clean)[0]) and torch.equal(heads(o)[1, :, 0], heads(o_clean)[1, :, 0])
        assert torch.equal(s[0], s_clean[0]) and torch.equal(s[1, 0], s_clean[1, 0])
        assert torch.equal(g[0], g_clean[0]) and torch.equal(g[1, 0], g_clean[1, 0])
        for lo, w in ((0, dk), (H * dk, dk), (2 * H * dk, dv)):
            a, b = (heads(x[:, lo:lo + H * w]) for x in (dqkv, d_clean))
            assert torch.equal(a[0], b[0]) and torch.equal(a[1, :, 0], b[1, :, 0])
        # tokens before it, of a query also those behind it: within the bounds of the clean call
        p["qkv"] = clean
        (ref, refS), (A, SA) = forward(p), forward(p, torch.abs)
        f32 = (T + dk + 48) * U
        bound = f32 * A if t == F32 else (f32 + 9 * 2.0 ** -16) * A + H8 * (ref.abs() + 9 * 2.0 ** -16 * A)
        fine = torch.ones(B * T, dtype=torch.bool)
        fine[T + at: T + at + 1 if part == "q" else 2 * T] = False
        within(o[fine], ref[fine], bound[fine] + 1e-37, "o")
        if part == "q":
            within(s, refS, f32 * SA + 1e-37, "s_last")
        dref, dA = backward(p)[0], backward(p, torch.abs)[0]
        b32 = (T + max(dk, dv) + 48) * U + 12 * 2.0 ** -16
        dbound = b32 * dA + H8 * (dref.abs() + b32 * dA) + 1e-37
        before, behind = slice(T, T + at), slice(T + at + 1, 2 * T)
        cols = lambda which: {"q": slice(0, H * dk), "kv": slice(H * dk, None)}[which]  # noqa: E731
        # dq: keys and values reach the later tokens; dk and dv: queries the earlier ones
        keep = [(before, "q"), (behind, "kv")] + ([(behind, "q")] if part == "q" else [(before, "kv")])
        for rows, which in keep:
            within(dqkv[rows, cols(which)], dref[rows, cols(which)], dbound[rows, cols(which)], f"d{which}")


@pytest.mark.gpu
@pytest.mark.parametrize("part", ["q", "k", "v"])
@pytest.mark.parametrize("value", [3.4e38, -3.395e38])
def test_fp32_above_the_largest_bf16(mmf, part, value):
    """Finite, but with no finite first part: as what is not finite."""
    B, T, H, dk, dv, at = 1, 100, 2, 32, 48, 70
    p = inputs(B, T, H, dk, dv, F32, seed=3, decay=[0.9, 0.5])
    ref, A = forward(p)[0], forward(p, torch.abs)[0]
    o_clean = run_fwd(mmf, p)[0]
    p["qkv"][at, {"q": 0, "k": H * dk, "v": 2 * H * dk}[part] + 3] = value   # of head 0
    o, s = run_fwd(mmf, p)
    bound = (T + dk + 48) * U * A + 1e-37
    within(o[:at], ref[:at], bound[:at], "o before")
    if part == "q":
        within(o[at + 1:], ref[at + 1:], bound[at + 1:], "o behind")
    assert torch.equal(o[:, dv:], o_clean[:, dv:]) and s[:, 1].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,at", [(3, 1), (100, 40), (700, 300)])
def test_gradients_that_are_not_finite(mmf, T, at):
    B, H, dk, dv = 2, 2, 32, 48
    p = inputs(B, T, H, dk, dv, F32, seed=T + at, decay=[0.9, 0.5])
    clean = run_bwd(mmf, p)
    good = p["dout"].clone()
    p["dout"][T + at, dv + 3] = float("nan")
    dqkv, g = run_bwd(mmf, p)
    dwant, G = backward(p)
    assert not dqkv[~dwant.isfinite()].isfinite().any() and not g[~G.isfinite()].isfinite().any()
    assert torch.equal(g[0], clean[1][0]) and torch.equal(g[1, 0], clean[1][1, 0])
    assert torch.equal(dqkv[:T], clean[0][:T])
    p["dout"] = good
    dref, dA = backward(p)[0], backward(p, torch.abs)[0]
    b32 = (T + max(dk, dv) + 48) * U + 12 * 2.0 ** -16
    dbound = b32 * dA + H8 * (dref.abs() + b32 * dA) + 1e-37
    rows = slice(T + at + 1, 2 * T)
    within(dqkv[rows], dref[rows], dbound[rows], "behind")
    rows, cols = slice(T, T + at), slice(0, H * dk)
    within(dqkv[rows, cols], dref[rows, cols], dbound[rows, cols], "dq before")


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 1, 1, 16, 16), (2, 5, 3, 80, 112), (3, 99, 2, 144, 16), (1, 517, 1, 128, 128)])
def test_nothing_around_the_outputs_is_written(mmf, B, T, H, dk, dv, t):
    p = inputs(B, T, H, dk, dv, t, seed=T)
    n, pad = B * T, 64

    def guarded(rows, w, dt):
        full = torch.full((rows * w + 2 * pad,), 3.0, dtype=dt, device=dev())
        return full, full[pad:pad + rows * w].reshape(rows, w)

    fo, o = guarded(n, H * dv, t)
    fs, s = guarded(B * H, dk * dv, F32)
    fd, d = guarded(n, H * (2 * dk + dv), BF)
    fg, g = guarded(B * H, dk * dv, F32)
    state = (B, H, dk, dv)
    need = max(mmf.mmf_linattn_workspace_bytes(B, T, H, dk, dv), mmf.mmf_linattn_bwd_workspace_bytes(B, T, H, dk, dv))
    ws = torch.full((need + 512,), 77, dtype=torch.uint8, device=dev())
    mmf.mmf_linattn_fwd(up(p["qkv"]), B, T, H, dk, dv, up(p["decay"]), p["scale"], up(p["s0"]), o, s.reshape(state),
                        ws[:mmf.mmf_linattn_workspace_bytes(B, T, H, dk, dv)])
    check_fwd(p, o.cpu(), s.reshape(state).cpu())
    assert (ws[mmf.mmf_linattn_workspace_bytes(B, T, H, dk, dv):] == 77).all()
    ws.fill_(77)
    mmf.mmf_linattn_bwd(up(p["qkv"]), B, T, H, dk, dv, up(p["decay"]), p["scale"], up(p["s0"]), up(p["dout"]).to(t),
                        up(p["ds_last"]), d, g.reshape(state), ws[:mmf.mmf_linattn_bwd_workspace_bytes(B, T, H, dk, dv)])
    check_bwd(p, d.cpu(), g.reshape(state).cpu())
    assert (ws[mmf.mmf_linattn_bwd_workspace_bytes(B, T, H, dk, dv):] == 77).all()
    for full in (fo, fs, fd, fg):
        assert (full[:pad] == 3).all() and (full[-pad:] == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
def test_rows_past_32_bits(mmf, t):
    """Rows behind 4 GiB of the inputs.  A decay of 1/2 forgets what lies 300
    tokens back (2^-300), so that the last rows are those of the last tokens
    alone, and the first rows' dk and dv those of the first."""
    H, dk, dv = 16, 128, 128
    T = (2 ** 32 // (H * 3 * dk * (4 if t == F32 else 2))) + 1111
    log(f"[linattn] T={T} {t}")
    gen = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.empty(T, H * 3 * dk, dtype=t, device=dev())
    for i in range(0, T, 16384):
        qkv[i:i + 16384] = torch.randn(qkv[i:i + 16384].shape, generator=gen, device=dev())
    do = torch.randn(T, H * dv, generator=gen, device=dev()).to(t)
    decay = torch.full((H,), 0.5, device=dev())
    o, s = torch.empty(T, H * dv, dtype=t, device=dev()), torch.empty(1, H, dk, dv, device=dev())
    mmf.mmf_linattn_fwd(qkv, 1, T, H, dk, dv, decay, 0.125, None, o, s)
    dqkv = torch.empty(T, H * 3 * dk, dtype=BF, device=dev())
    mmf.mmf_linattn_bwd(qkv, 1, T, H, dk, dv, decay, 0.125, None, do, None, dqkv, None)
    n, k, h = 360, 300, 15   # tokens of the reference, those that only lead to it, the last head

    def short(rows):
        x = qkv[rows].reshape(n, 3, H, dk)[:, :, h].reshape(n, 3 * dk).cpu()
        return {"qkv": x, "decay": torch.tensor([0.5]), "s0": None, "ds_last": None, "scale": 0.125,
                "dout": do[rows].reshape(n, H, dv)[:, h].cpu(), "dims": (1, n, 1, dk, dv)}

    last = short(slice(T - n, T))
    (want, S), (A, SA) = forward(last), forward(last, torch.abs)
    f32 = (n + dk + 48) * U   # what lies further back weighs nothing
    bound = f32 * A if t == F32 else (f32 + 9 * 2.0 ** -16) * A + H8 * (want.abs() + 9 * 2.0 ** -16 * A)
    within(o[T - n:].reshape(n, H, dv)[k:, h].cpu(), want[k:], bound[k:] + 1e-37, "o")
    within(s[:, h:].cpu(), S, f32 * SA + 1e-37, "s_last")
    b32 = (n + dk + 48) * U + 12 * 2.0 ** -16

    def grads(p, rows, keep, cols):
        want, A = backward(p)[0], backward(p, torch.abs)[0]
        got = dqkv[rows].reshape(n, 3, H, dk)[:, :, h].reshape(n, 3 * dk).cpu()
        bound = b32 * A + H8 * (want.abs() + b32 * A) + 1e-37
        within(got[keep, cols], want[keep, cols], bound[keep, cols], "dqkv")

    grads(last, slice(T - n, T), slice(k, n), slice(0, 3 * dk))
    grads(short(slice(0, n)), slice(0, n), slice(0, n - k), slice(0, 3 * dk))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 9, 150])
def test_gradients_are_the_slopes(mmf, T):
    """sum(o dout) + sum(s_last ds_last) is linear in each single entry of q, k, v
    and s0: differences of the forward in 64 bits are its slopes."""
    p = inputs(1, T, 2, 16, 32, F32, seed=T)
    dqkv, g = run_bwd(mmf, p)
    A, GA = backward(p, torch.abs)

    def value(x, s0):
        o, S = forward({**p, "qkv": x, "s0": s0})
        return float((o * p["dout"].double()).sum() + (S * p["ds_last"].double()).sum())

    x0, s0 = p["qkv"].double(), p["s0"].double()
    b32 = (T + 80) * U + 12 * 2.0 ** -16
    for t in {0, T // 2, T - 1}:
        for c in (3, 16 + 7, 32 + 5, 48 + 15, 64 + 1, 96 + 31):
            a, b = x0.clone(), x0.clone()
            a[t, c] += 1.0
            b[t, c] -= 1.0
            slope = (value(a, s0) - value(b, s0)) / 2
            assert abs(float(dqkv[t, c]) - slope) <= b32 * float(A[t, c]) * 2 + H8 * abs(slope) + 1e-10 * float(A.max())
    for i in ((0, 0, 0, 0), (0, 1, 15, 31), (0, 0, 7, 20)):
        a, b = s0.clone(), s0.clone()
        a[i] += 1.0
        b[i] -= 1.0
        slope = (value(x0, a) - value(x0, b)) / 2
        assert abs(float(g[i]) - slope) <= (T + 64) * U * float(GA[i]) + 1e-10 * float(GA.max())
