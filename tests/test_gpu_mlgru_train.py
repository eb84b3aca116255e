"""The MLGRU recurrence in training form (mmf_mlgru_train_scan,
mmf_mlgru_scan_bwd) against the equations in 64 bits.

Tolerances, u = 2^-24, from a first-order propagation of fp32 roundings along
the sequence, evaluated in 64 bits beside the values.  The hardware sigmoid
carries e_s = s ((1 - s)(|v| + 2) + 3) u; f = (1 - lb) s + lb and c = z s carry
it and two roundings; a step h' = f h + (1 - f) c passes on f times the error
before it and adds |h| e_f + |c| e_f + (1 - f) e_c and 4 u of its terms; the
gradient's recurrence likewise.  The kernels reach a token's state through the
maps of the runs before it (products of forget gates), whose factors carry the
same relative errors as the steps, once in a run's map and once more in the
join: the tests allow four times the propagated bound.  A value in bf16 adds
half a step, 2^-8 of it.
"""
import pytest
import torch

from _parity import dev, log

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
TINY = 1e-30


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def sig(v):
    s = torch.sigmoid(v)
    return s, s * ((1 - s) * (v.abs() + 2) + 3) * U


def scan64(z, B, T, lb, h0, do, dh):
    """Values and error bounds (float64, CPU): o, h_last, dz, dh0, dlb."""
    d = z.shape[1] // 3
    z = z.double().reshape(B, T, 3, d)
    zf, zc, g = z[:, :, 0], z[:, :, 1], z[:, :, 2]
    lb = torch.zeros(d, dtype=torch.float64) if lb is None else lb.double()
    h = torch.zeros((B, d), dtype=torch.float64) if h0 is None else h0.double()
    do = do.double().reshape(B, T, d)
    sf, esf = sig(zf)
    sc, esc = sig(zc)
    f, c = lb + (1 - lb) * sf, zc * sc
    ef, ec = (1 - lb) * esf + 3 * U * f, zc.abs() * esc + U * c.abs()
    hp, hs, ehp, eh = [], [], [], []
    e = torch.zeros_like(h)
    for t in range(T):
        hp.append(h)
        ehp.append(e)
        n = f[:, t] * h + (1 - f[:, t]) * c[:, t]
        e = f[:, t] * e + (h.abs() + c[:, t].abs()) * (ef[:, t] + U) + (1 - f[:, t]) * ec[:, t] \
            + 4 * U * ((f[:, t] * h).abs() + ((1 - f[:, t]) * c[:, t]).abs())
        h = n
        hs.append(h)
        eh.append(e)
    hp, hs, ehp, eh = (torch.stack(v, 1) for v in (hp, hs, ehp, eh))
    sh, esh = sig(hs)
    o = g * sh
    eo = g.abs() * (sh * (1 - sh) * eh + esh) + U * o.abs()
    own = do * g * sh * (1 - sh)
    # 1 - s rounds to half a step of 1 where s is near 1
    slope = lambda s, es: es * (1 - 2 * s).abs() + 4 * U * s * (1 - s) + U * s  # noqa: E731
    eown = (do * g).abs() * (sh * (1 - sh) * (1 - 2 * sh).abs() * eh + slope(sh, esh))
    G = torch.zeros((B, d), dtype=torch.float64) if dh is None else dh.double()
    eG = torch.zeros_like(G)
    dhs, edh = [None] * T, [None] * T
    for t in range(T - 1, -1, -1):
        dhs[t] = G + own[:, t]
        edh[t] = eG + eown[:, t] + U * dhs[t].abs()
        G = f[:, t] * dhs[t]
        eG = f[:, t] * edh[t] + dhs[t].abs() * ef[:, t] + U * G.abs() + 2 * U * (f[:, t] * own[:, t]).abs()
    dhs, edh = torch.stack(dhs, 1), torch.stack(edh, 1)
    diff = hp - c
    w, ew = dhs * diff, edh * diff.abs() + dhs.abs() * (ehp + ec + U * (hp.abs() + c.abs())) + U * (dhs * diff).abs()
    k = (1 - lb) * sf * (1 - sf)
    df, edf = w * k, ew * k + w.abs() * ((1 - lb) * slope(sf, esf) + 2 * U * k)
    q = sc * (1 + zc * (1 - sc))
    eq = esc * (1 + zc.abs()) * 2 + 4 * U * (sc + (zc * sc).abs()) + 4 * U * q.abs()
    dc = dhs * (1 - f) * q
    edc = edh * (1 - f) * q.abs() + dhs.abs() * ((ef + U) * q.abs() + (1 - f) * eq) + 3 * U * dc.abs()
    dg, edg = do * sh, do.abs() * (sh * (1 - sh) * eh + esh) + U * (do * sh).abs()
    dz, edz = torch.stack([df, dc, dg], 2), torch.stack([edf, edc, edg], 2)
    dl = w * (1 - sf)
    edl = (ew * (1 - sf) + w.abs() * (esf + U) + U * dl.abs()).sum((0, 1)) + U * dl.sum((0, 1)).abs()
    flat = lambda v: v.reshape(B * T, -1)  # noqa: E731
    return {"o": (flat(o), 4 * flat(eo)), "h": (hs[:, -1], 4 * eh[:, -1]),
            "dz": (flat(dz), 4 * flat(edz) + 2.0 ** -8 * flat(dz).abs()), "dh0": (G, 4 * eG),
            "dlb": (dl.sum((0, 1)), 4 * edl)}


def make(seed, B, T, d, dt, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B * T, 3 * d), generator=g) * scale
    return {"z": z, "lb": torch.rand(d, generator=g) * 0.95, "h0": torch.randn((B, d), generator=g) * 0.5,
            "do": torch.randn((B * T, d), generator=g).to(dt), "dh": torch.randn((B, d), generator=g)}


def guarded(rows, cols, dtype):
    whole = torch.full((rows + 2, cols), 55, dtype=dtype, device=dev())
    return whole, whole[1:rows + 1]


def run(mmf, v, B, T, h_last_is_h0=False, dh0_is_dh_last=False):
    d = v["z"].shape[1] // 3
    t = {k: None if x is None else x.to(dev()) for k, x in v.items()}
    wo, o = guarded(B * T, d, F32)
    wz, dz = guarded(B * T, 3 * d, BF)
    h = t["h0"] if h_last_is_h0 else torch.full((B, d), float("nan"), device=dev())
    dh0 = t["dh"] if dh0_is_dh_last else torch.full((B, d), float("nan"), device=dev())
    dlb = torch.full((d,), float("nan"), device=dev())
    n, m = mmf.mmf_mlgru_train_states_bytes(B, T, d), mmf.mmf_mlgru_scan_bwd_workspace_bytes(B, T, d)
    assert m >= mmf.mmf_mlgru_train_scan_workspace_bytes(B, T, d)
    states = torch.full((n + 256,), 0xAB, dtype=torch.uint8, device=dev())
    ws = torch.full((m + 256,), 0xAB, dtype=torch.uint8, device=dev())
    mmf.mmf_mlgru_train_scan(t["z"], B, T, t["lb"], t["h0"], o, h, states[:n], ws[:m])
    mmf.mmf_mlgru_scan_bwd(t["z"], B, T, t["lb"], states[:n], t["do"], t["dh"], dz, dh0, dlb, ws[:m])
    torch.cuda.synchronize()
    for w in (wo, wz):
        assert (w[0] == 55).all() and (w[-1] == 55).all()
    assert (states[n:] == 0xAB).all() and (ws[m:] == 0xAB).all()
    return {"o": o.clone(), "h": h.clone(), "dz": dz.clone(), "dh0": dh0, "dlb": dlb}


def check(mmf, v, B, T, **kw):
    want = scan64(v["z"], B, T, v["lb"], v["h0"], v["do"], v["dh"])
    got = run(mmf, v, B, T, **kw)
    for k, (x, tol) in want.items():
        err = (got[k].cpu().double() - x).abs()
        assert (err <= tol + TINY).all(), f"{k}: {float((err / (tol + TINY)).max()):.3g} of the tolerance"
    return got


# around 8 tokens (a half wave's), 128 (a chunk) and 16 chunks (a run)
SIZES = [(1, 1, 16), (3, 1, 2048), (2, 7, 16), (1, 8, 48), (1, 9, 128), (2, 63, 144), (2, 127, 80), (2, 128, 256),
         (2, 129, 256), (3, 357, 1040), (5, 700, 32), (1, 2048, 64), (2, 2049, 48), (1, 18433, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,T,d", SIZES)
def test_against_the_equations(mmf, B, T, d, dt):
    log(f"[mlgru_train] B={B} T={T} d={d} do={dt}")
    check(mmf, make(B * 7 + T + d, B, T, d, dt), B, T)


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,d", [(2, 5, 32), (2, 200, 144)])
def test_optional_inputs(mmf, B, T, d):
    for drop in ("lb", "h0", "dh"):
        log(f"[mlgru_train] without {drop}")
        v = make(1, B, T, d, F32)
        v[drop] = None
        check(mmf, v, B, T)
    check(mmf, make(2, B, T, d, F32), B, T, h_last_is_h0=True)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [129, 1500, 2500])
def test_state_in_place_over_several_chunks(mmf, T):
    check(mmf, make(6, 2, T, 80, F32), 2, T, h_last_is_h0=True)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 128, 129, 1500, 2500])
def test_gradient_of_the_state_in_place(mmf, T):
    """As for sequences that are passed segment by segment, the last first."""
    check(mmf, make(7, 2, T, 80, F32), 2, T, dh0_is_dh_last=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
def test_past_the_last_level_cache(mmf, dt):
    """Four sequences that together exceed 256 MB, and so pass as streams:
    each as in a call of its own."""
    B, T, d = 4, 2100, 2064
    g = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(s, generator=g, device=dev())  # noqa: E731
    v = {"z": rand(B * T, 3 * d), "lb": torch.rand(d, generator=g, device=dev()) * 0.9, "h0": rand(B, d),
         "do": rand(B * T, d).to(dt), "dh": rand(B, d)}
    a = run(mmf, v, B, T)
    total = torch.zeros(d, device=dev(), dtype=torch.float64)
    for b in range(B):
        s, r = slice(b * T, (b + 1) * T), slice(b, b + 1)
        one = run(mmf, {"z": v["z"][s], "lb": v["lb"], "h0": v["h0"][r], "do": v["do"][s], "dh": v["dh"][r]}, 1, T)
        assert torch.equal(a["o"][s], one["o"]) and torch.equal(a["dz"][s], one["dz"])
        assert torch.equal(a["h"][r], one["h"]) and torch.equal(a["dh0"][r], one["dh0"])
        total += one["dlb"].double()
    # the same fp64 sums, rounded once, or once per sequence
    assert ((a["dlb"].double() - total).abs() <= U * (total.abs() + B * 2 ** 11)).all()


@pytest.mark.gpu
def test_offsets_past_32_bits(mmf):
    """z of 4.4 GB: the last sequence as in a call of its own."""
    B, T, d = 44, 4096, 2048
    g = torch.Generator(device="cuda").manual_seed(10)
    v = {"z": torch.randn((B * T, 3 * d), generator=g, device=dev()), "lb": None,
         "h0": torch.randn((B, d), generator=g, device=dev()),
         "do": torch.randn((B * T, d), generator=g, device=dev()), "dh": None}
    assert v["z"].numel() * 4 > 1 << 32
    a = run(mmf, v, B, T)
    s, r = slice((B - 1) * T, B * T), slice(B - 1, B)
    one = run(mmf, {"z": v["z"][s], "lb": None, "h0": v["h0"][r], "do": v["do"][s], "dh": None}, 1, T)
    assert torch.equal(a["o"][s], one["o"]) and torch.equal(a["dz"][s], one["dz"])
    assert torch.equal(a["h"][r], one["h"]) and torch.equal(a["dh0"][r], one["dh0"])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [60, 300])
def test_saturated_gates(mmf, T):
    """Forget gates of exactly 0 and 1 (long memories), candidates far out."""
    v = make(3, 2, T, 32, F32, scale=4.0)
    v["z"][::3, :32] = 200.0
    v["z"][::7, :16] = -200.0
    v["z"][::5, 32:64] *= 10.0
    v["lb"][:8] = 0.0
    v["lb"][8] = 1.0
    check(mmf, v, 2, T)


@pytest.mark.gpu
def test_optional_outputs_and_repeatability(mmf):
    B, T, d = 2, 333, 144
    v = make(4, B, T, d, F32)
    a, b = run(mmf, v, B, T), run(mmf, v, B, T)
    assert all(torch.equal(a[k], b[k]) for k in a)
    t = {k: x.to(dev()) for k, x in v.items()}
    o, dz = torch.empty((B * T, d), device=dev()), torch.empty((B * T, 3 * d), dtype=BF, device=dev())
    states = torch.empty(mmf.mmf_mlgru_train_states_bytes(B, T, d), dtype=torch.uint8, device=dev())
    # without workspace: allocated in the call
    mmf.mmf_mlgru_train_scan(t["z"], B, T, t["lb"], t["h0"], o, None, states)
    mmf.mmf_mlgru_scan_bwd(t["z"], B, T, t["lb"], states, t["do"], t["dh"], dz, None, None)
    assert torch.equal(o, a["o"]) and torch.equal(dz, a["dz"])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 500])
def test_on_another_stream_and_captured(mmf, T):
    B, d = 2, 272
    v = make(5, B, T, d, BF)
    want = run(mmf, v, B, T)
    t = {k: x.to(dev()) for k, x in v.items()}
    o, h = torch.zeros((B * T, d), device=dev()), torch.zeros((B, d), device=dev())
    dz, dh0 = torch.zeros((B * T, 3 * d), dtype=BF, device=dev()), torch.zeros((B, d), device=dev())
    dlb = torch.zeros(d, device=dev())
    states = torch.empty(mmf.mmf_mlgru_train_states_bytes(B, T, d), dtype=torch.uint8, device=dev())
    ws = torch.empty(mmf.mmf_mlgru_scan_bwd_workspace_bytes(B, T, d) or 256, dtype=torch.uint8, device=dev())
    torch.cuda.synchronize()

    def step(stream=None):
        mmf.mmf_mlgru_train_scan(t["z"], B, T, t["lb"], t["h0"], o, h, states, ws, stream)
        mmf.mmf_mlgru_scan_bwd(t["z"], B, T, t["lb"], states, t["do"], t["dh"], dz, dh0, dlb, ws, stream)

    def same():
        return all(torch.equal(x, want[k]) for k, x in (("o", o), ("h", h), ("dz", dz), ("dh0", dh0), ("dlb", dlb)))

    st = torch.cuda.Stream()
    step(st)
    st.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for x in (o, h, dz, dh0, dlb):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same()


class Held:
    """Device arrays of a problem and its two calls; `ws` may be another's."""

    def __init__(self, mmf, seed, B, T, d, ws=None):
        self.v = make(seed, B, T, d, F32)
        self.t = {k: x.to(dev()) for k, x in self.v.items()}
        self.size = B, T
        self.out = {"o": torch.zeros((B * T, d), device=dev()), "h": torch.zeros((B, d), device=dev()),
                    "dz": torch.zeros((B * T, 3 * d), dtype=BF, device=dev()),
                    "dh0": torch.zeros((B, d), device=dev()), "dlb": torch.zeros(d, device=dev())}
        self.states = torch.empty(mmf.mmf_mlgru_train_states_bytes(B, T, d), dtype=torch.uint8, device=dev())
        n = mmf.mmf_mlgru_scan_bwd_workspace_bytes(B, T, d)
        self.ws = torch.empty(n, dtype=torch.uint8, device=dev()) if ws is None else ws
        assert self.ws.numel() >= n
        self.want = run(mmf, self.v, B, T)

    def step(self, mmf, stream=None):
        t, w, (B, T) = self.t, self.out, self.size
        mmf.mmf_mlgru_train_scan(t["z"], B, T, t["lb"], t["h0"], w["o"], w["h"], self.states, self.ws, stream)
        mmf.mmf_mlgru_scan_bwd(t["z"], B, T, t["lb"], self.states, t["do"], t["dh"], w["dz"], w["dh0"], w["dlb"],
                               self.ws, stream)

    def same(self):
        return all(torch.equal(x, self.want[k]) for k, x in self.out.items())

    def clear(self):
        for x in self.out.values():
            x.zero_()


@pytest.mark.gpu
def test_two_graphs_share_a_workspace(mmf):
    """Replayed in turn on one stream, of different sizes."""
    a = Held(mmf, 11, 2, 2500, 144)
    b = Held(mmf, 12, 3, 300, 80, a.ws)
    graphs = []
    for x in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.step(mmf)
    for _ in range(3):
        for x in (a, b):
            x.clear()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert a.same() and b.same()
        b.clear()
        b.step(mmf)
        torch.cuda.synchronize()
        assert b.same()


@pytest.mark.gpu
def test_two_streams_at_once(mmf):
    """Calls side by side, each with more chunks than fit the chip at once."""
    both = [Held(mmf, 13, 1, 6000, 2048), Held(mmf, 14, 2, 4000, 1040)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for x in both:
            x.clear()
        torch.cuda.synchronize()
        for x, s in zip(both, streams):
            x.step(mmf, s)
        torch.cuda.synchronize()
        assert both[0].same() and both[1].same()


def test_equations_against_differences():
    """The gradients are those of sum(do o') + sum(dh_last h_T)."""
    B, T, d = 2, 5, 2
    g = torch.Generator().manual_seed(8)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    z, h0, do, dh, lb = rand(B * T, 3 * d), rand(B, d), rand(B * T, d), rand(B, d), torch.rand(d, generator=g).double()

    def loss(z, lb, h0):
        r = scan64(z, B, T, lb, h0, do, dh)
        return float((do * r["o"][0]).sum() + (dh * r["h"][0]).sum())

    r = scan64(z, B, T, lb, h0, do, dh)
    for i, (x, want) in enumerate(((z, r["dz"][0]), (lb, r["dlb"][0]), (h0, r["dh0"][0]))):
        for j in range(x.numel()):
            args = [z, lb, h0]
            e = torch.zeros_like(x).reshape(-1)
            e[j] = 1e-6
            e = e.reshape(x.shape)
            args[i] = x + e
            up = loss(*args)
            args[i] = x - e
            assert abs((up - loss(*args)) / 2e-6 - float(want.reshape(-1)[j])) < 1e-7


A, BAD, S = 0x100000, 0x100004, None


def test_refusals(mmf):
    lib = mmf._lib
    sb = mmf.mmf_mlgru_train_states_bytes(2, 200, 32)
    wf, wb = mmf.mmf_mlgru_train_scan_workspace_bytes(2, 200, 32), mmf.mmf_mlgru_scan_bwd_workspace_bytes(2, 200, 32)
    assert sb == 2 * 2 * 32 * 4 and 0 < wf < wb and wb % 256 == 0

    def fwd(z=A, lb=A, h0=A, o=A, h=A, st=A, n=sb, B=2, T=200, d=32, ws=A, wn=wf):
        return lib.mmf_mlgru_train_scan(z, lb, h0, o, h, st, n, B, T, d, ws, wn, S)

    def bwd(z=A, lb=A, st=A, n=sb, do=A, k=1, dh=A, dz=A, dh0=A, dlb=A, B=2, T=200, d=32, ws=A, wn=wb):
        return lib.mmf_mlgru_scan_bwd(z, lb, st, n, do, k, dh, dz, dh0, dlb, B, T, d, ws, wn, S)

    for f in (fwd, bwd):
        for d in (0, -16, 24):
            assert f(d=d) == 2
        assert f(B=-1) == 2 and f(T=-1) == 2 and f(B=1 << 20, T=1 << 12) == 2
        assert f(B=1 << 22, T=129, d=16) == 2          # 2^23 workgroups
        assert f(d=(1 << 20) + 16) == 2
        assert f(n=sb - 1) == 6 and f(st=A + 16) == 6 and f(ws=A + 16) == 6
        assert f(z=None) == 1 and f(st=None) == 1
        assert f(z=None, B=0) == 0 and f(z=None, T=0) == 0
    assert fwd(o=None) == 1 and fwd(wn=wf - 1) == 6
    assert bwd(do=None) == 1 and bwd(dz=None) == 1 and bwd(wn=wb - 1) == 6 and bwd(k=2) == 4
    for name in ("z", "lb", "h0", "o", "h"):
        assert fwd(**{name: BAD}) == 3
    for name in ("z", "lb", "do", "dh", "dz", "dh0", "dlb"):
        assert bwd(**{name: BAD}) == 3
    assert mmf.mmf_mlgru_train_states_bytes(2, 100, 24) == 0
    assert mmf.mmf_mlgru_train_scan_workspace_bytes(7, 128, 32) == 0   # one chunk: no maps


def test_workspace_of_a_batch_serves_smaller_ones(mmf):
    for B, d in ((1, 16), (4, 2048)):
        for f in (mmf.mmf_mlgru_scan_bwd_workspace_bytes, mmf.mmf_mlgru_train_states_bytes):
            sizes = [f(B, T, d) for T in range(1, 600)]
            assert sizes == sorted(sizes)
