"""Residual addition + quantisation (mmf_add_act_quant) and its backward,
against the addition followed by mmf_act_quant_ex (the same bits) and against
the formulas in 64 bits.

With u = 2^-24, forward from the stored s: rstd is the fp32 rounding of an
fp64 root (u, and another u where the sums' order moves it over a border);
a_scale = fl(fl(s r) gamma) / 127 carries four roundings and rstd's two.
Backward, per element: g = fl(gamma dY) (u), t sums fl products in fp64 (u sum
|g s|), the coefficient c = r^3 t / K is rounded once, and ds takes the
roundings of r g, c s, their difference and the residual's addition:
  |err| <= u (2 |r g| + 2 |c s| + r^3 / K sum |g s| |s| + |r g - c s| + |ds|)
to first order (held with 1 % to spare for the products of roundings); the
bf16 copy adds half a step, 2^-8 |ds|... of the value it rounds; dgamma sums
products of two roundings in fp64 and is rounded once.
"""
import pytest
import torch

from _parity import dev, log

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device=dev()) * scale).to(dtype)


def ref64(s, gamma):
    s = s.double()
    r = 1.0 / torch.sqrt(s.square().mean(1) + 1e-6)
    y = s * r[:, None]
    return r, y if gamma is None else y * gamma.double()


def guarded(M, K, dtype):
    """An [M][K] array inside a larger one whose other rows must stay."""
    whole = torch.full((M + 2, K), 77, dtype=dtype, device=dev())
    return whole, whole[1:M + 1]


def check_fwd(mmf, M, K, xt, bt, gamma=True, branch=True, in_place=False, scale=1.0, seed=0):
    log(f"[add_quant] M={M} K={K} x={xt} branch={bt if branch else None} gamma={gamma} in_place={in_place}")
    g = gen(seed + M * 131 + K)
    x = rand(g, M, K, dtype=xt, scale=scale)
    b = rand(g, M, K, dtype=bt, scale=scale) if branch else None
    gm = torch.rand(K, generator=g, device=dev()) + 0.5 if gamma else None
    want_s = (x.float() + b.float()).to(xt) if branch else x.clone()
    ws_, s = guarded(M, K, xt)
    wq, q = guarded(M, K, torch.int8)
    if in_place:
        s.copy_(x)
        x = s
    a, r = (torch.full((M,), float("nan"), device=dev()) for _ in range(2))
    rs = torch.full((M,), 99, dtype=torch.int32, device=dev())
    mmf.mmf_add_act_quant(x, b, gm, s, q, a, rs, r)
    q2, a2, rs2 = torch.empty_like(q), torch.empty_like(a), torch.empty_like(rs)
    mmf.mmf_act_quant_ex(want_s, gm, q2, a2, rs2)
    torch.cuda.synchronize()
    assert torch.equal(s, want_s)
    assert torch.equal(q, q2) and torch.equal(a, a2) and torch.equal(rs, rs2)
    for w in (ws_, wq):
        assert (w[0] == 77).all() and (w[-1] == 77).all()
    r64, y64 = ref64(want_s, gm)
    assert ((r.double() - r64).abs() <= 2 * U * r64).all()
    a64 = y64.abs().amax(1).clamp_min(1e-5) / 127.0
    assert ((a.double() - a64).abs() <= 6.1 * U * a64).all()
    # q: the nearest integer, but for the roundings next to a midpoint
    qs = y64 / a64[:, None]
    assert ((q.double() - qs).abs() <= 0.5 + 127 * 10 * U).all()
    assert torch.equal(rs.long(), q.long().sum(1))


SIZES = [(1, 16), (1, 2048), (3, 48), (64, 256), (65, 256), (45, 5120), (300, 2048), (7, 2064), (130, 8192),
         (66, 8208), (5, 32768), (70, 32768), (3, 32784), (66, 65552)]


@pytest.mark.gpu
@pytest.mark.parametrize("bt", [BF, F32], ids=["bbf16", "bf32"])
@pytest.mark.parametrize("xt", [BF, F32], ids=["xbf16", "xf32"])
@pytest.mark.parametrize("M,K", SIZES)
def test_forward(mmf, M, K, xt, bt):
    check_fwd(mmf, M, K, xt, bt)


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [BF, F32], ids=["xbf16", "xf32"])
@pytest.mark.parametrize("M,K", [(1, 2048), (77, 528), (66, 65552)])
def test_forward_options(mmf, M, K, xt):
    check_fwd(mmf, M, K, xt, F32, gamma=False)
    check_fwd(mmf, M, K, xt, F32, in_place=True)
    check_fwd(mmf, M, K, xt, BF, branch=False)
    check_fwd(mmf, M, K, xt, F32, scale=0.0)      # rows of zeros
    check_fwd(mmf, M, K, xt, F32, scale=1e-6)
    check_fwd(mmf, M, K, xt, BF, scale=1e4)


@pytest.mark.gpu
def test_forward_more_rows_than_a_grid(mmf):
    """4 x 2^20 + 5 rows: the grid's second pass over the rows."""
    check_fwd(mmf, 4 * (1 << 20) + 5, 16, BF, BF)


@pytest.mark.gpu
@pytest.mark.parametrize("xt,bt", [(BF, F32), (F32, F32), (BF, BF)])
def test_forward_past_the_last_level_cache(mmf, xt, bt):
    """More than 256 MB: read and written as streams."""
    check_fwd(mmf, 9001, 8000, xt, bt)
    check_fwd(mmf, 40001, 1040, xt, bt, in_place=True)


@pytest.mark.gpu
def test_offsets_past_32_bits(mmf):
    """Arrays of 4.9 GB: the last rows as in calls of their own."""
    M, K, n = 600_000, 2048, 37
    g = gen(11)
    x, b = rand(g, M, K), rand(g, M, K, dtype=BF)
    s, q, a, rs, r = mmf.add_act_quant(x, b, None)
    tail = slice(M - n, M)
    s2, q2, a2, rs2, r2 = mmf.add_act_quant(x[tail], b[tail], None)
    for u, v in ((s, s2), (q, q2), (a, a2), (rs, rs2), (r, r2)):
        assert torch.equal(u[tail], v)
    ds, dh = torch.empty_like(s), torch.empty((M, K), dtype=BF, device=dev())
    mmf.mmf_add_act_quant_bwd(b, x, s, None, r, ds, dh, None)
    ds2, dh2 = torch.empty_like(s2), torch.empty((n, K), dtype=BF, device=dev())
    mmf.mmf_add_act_quant_bwd(b[tail], x[tail], s2, None, r2, ds2, dh2, None)
    assert torch.equal(ds[tail], ds2) and torch.equal(dh[tail], dh2)


@pytest.mark.gpu
def test_backward_past_the_last_level_cache(mmf):
    check_bwd(mmf, 8001, 2288, BF, F32)
    check_bwd(mmf, 30001, 1040, F32, BF, in_place=True)


@pytest.mark.gpu
def test_forward_without_the_optional_outputs(mmf):
    g = gen(5)
    x, b = rand(g, 9, 256), rand(g, 9, 256)
    q, a = torch.empty((9, 256), dtype=torch.int8, device=dev()), torch.empty(9, device=dev())
    s, q2, a2, rs, r = mmf.add_act_quant(x, b, None)
    s2 = torch.empty_like(s)
    mmf.mmf_add_act_quant(x, b, None, s2, q, a)
    assert torch.equal(q, q2) and torch.equal(a, a2) and torch.equal(s, s2)
    mmf.mmf_add_act_quant(s, None, None, None, q, a)
    assert torch.equal(q, q2) and torch.equal(a, a2)


@pytest.mark.gpu
def test_forward_nan_stays_in_the_stream(mmf):
    """A row that blew up keeps its NaN and infinity in s; the rows beside it
    are as without it."""
    g = gen(6)
    x, b = rand(g, 5, 512, dtype=BF), rand(g, 5, 512)
    s0, q0, a0, rs0, _ = mmf.add_act_quant(x, b, None)
    b[2, 7], b[2, 100] = float("nan"), float("inf")
    s, q, a, rs, _ = mmf.add_act_quant(x, b, None)
    assert s[2, 7].isnan() and s[2, 100] == float("inf")
    for i in (0, 1, 3, 4):
        assert torch.equal(s[i], s0[i]) and torch.equal(q[i], q0[i]) and a[i] == a0[i] and rs[i] == rs0[i]


def bwd64(dy, res, s, gamma, r):
    dy, s, r = dy.double(), s.double(), r.double()[:, None]
    g = dy if gamma is None else dy * gamma.double()
    t = (g * s).sum(1, keepdim=True)
    c = r ** 3 * t / s.shape[1]
    core = r * g - c * s
    ds = core if res is None else core + res.double()
    dgamma = (dy * s * r).sum(0)
    tol = U * (2 * (r * g).abs() + 2 * (c * s).abs() + r ** 3 / s.shape[1] * (g * s).abs().sum(1, keepdim=True) * s.abs()
               + core.abs() + ds.abs()) * 1.01
    return ds, dgamma, tol, 2.02 * U * (dy * s * r).abs().sum(0) + U * dgamma.abs()


def check_bwd(mmf, M, K, st, dt, gamma=True, res=True, in_place=False, half=True, want_dgamma=True):
    log(f"[add_quant_bwd] M={M} K={K} s={st} dy={dt} gamma={gamma} res={res} in_place={in_place}")
    g = gen(M * 17 + K)
    s, dy = rand(g, M, K, dtype=st, scale=2.0), rand(g, M, K, dtype=dt)
    do = rand(g, M, K) if res else None
    gm = torch.rand(K, generator=g, device=dev()) + 0.5 if gamma else None
    r = (s.double().square().mean(1) + 1e-6).rsqrt().float()
    want, wantg, tol, tolg = bwd64(dy, do, s, gm, r)
    whole, ds = guarded(M, K, F32)
    if in_place:
        ds.copy_(do)
        do = ds
    wh, dh = guarded(M, K, BF)
    dg = torch.full((K,), float("nan"), device=dev()) if want_dgamma else None
    need = mmf.mmf_add_act_quant_bwd_workspace_bytes(M, K)
    ws = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device=dev())
    mmf.mmf_add_act_quant_bwd(dy, do, s, gm, r, ds, dh if half else None, dg, ws[:need])
    torch.cuda.synchronize()
    assert ((ds.double() - want).abs() <= tol).all(), float(((ds.double() - want).abs() / tol).max())
    if half:
        assert torch.equal(dh, ds.to(BF))
        assert (wh[0] == 77).all() and (wh[-1] == 77).all()
    assert (whole[0] == 77).all() and (whole[-1] == 77).all() and (ws[need:] == 0xAB).all()
    if want_dgamma:
        assert ((dg.double() - wantg).abs() <= tolg).all()
    return ds.clone(), dg


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["dbf16", "df32"])
@pytest.mark.parametrize("st", [BF, F32], ids=["sbf16", "sf32"])
@pytest.mark.parametrize("M,K", [(1, 16), (1, 2048), (37, 48), (300, 1024), (65, 1040), (1937, 2288), (513, 4112),
                                 (40, 8208), (33, 16384), (9, 16400)])
def test_backward(mmf, M, K, st, dt):
    check_bwd(mmf, M, K, st, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K", [(5000, 256), (200, 2048), (30, 16400)])
def test_backward_options(mmf, M, K):
    check_bwd(mmf, M, K, BF, F32, gamma=False)
    check_bwd(mmf, M, K, BF, F32, res=False)
    check_bwd(mmf, M, K, F32, BF, in_place=True)
    check_bwd(mmf, M, K, F32, F32, half=False, want_dgamma=False)
    a, b = check_bwd(mmf, M, K, BF, F32), check_bwd(mmf, M, K, BF, F32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])  # the same bits on every call


def test_backward_formula_against_differences():
    """The formula's gradients are those of sum(dY y) + sum(ds_out s)."""
    g = torch.Generator().manual_seed(3)
    s, dy, do = (torch.randn((3, 16), generator=g, dtype=torch.float64) for _ in range(3))
    gamma = torch.rand(16, generator=g, dtype=torch.float64) + 0.5

    def loss(s, gamma):
        return float((dy * ref64(s, gamma)[1]).sum() + (do * s).sum())

    ds, dgamma, _, _ = bwd64(dy, do, s, gamma, ref64(s, gamma)[0])
    h = 1e-6
    for i in range(3):
        for k in range(16):
            e = torch.zeros_like(s)
            e[i, k] = h
            assert abs((loss(s + e, gamma) - loss(s - e, gamma)) / (2 * h) - float(ds[i, k])) < 1e-7
    for k in range(16):
        e = torch.zeros_like(gamma)
        e[k] = h
        assert abs((loss(s, gamma + e) - loss(s, gamma - e)) / (2 * h) - float(dgamma[k])) < 1e-7


A, BAD, S = 0x100000, 0x100004, None


def test_refusals(mmf):
    """Bad arguments are refused before anything is enqueued (stand-in
    addresses, never dereferenced)."""
    lib = mmf._lib
    f = lib.mmf_add_act_quant

    def fwd(x=A, xf=0, b=A, bf=1, g=A, s=A, q=A, a=A, rs=A, r=A, M=4, K=32):
        return f(x, xf, b, bf, g, s, q, a, rs, r, M, K, S)

    for K in (0, -16, 24, (1 << 20) + 16):
        assert fwd(K=K) == 2
    assert fwd(M=-1) == 2 and fwd(M=1 << 31) == 2
    assert fwd(xf=2) == 4 and fwd(bf=-1) == 4
    assert fwd(x=None) == 1 and fwd(s=None) == 1 and fwd(q=None) == 1 and fwd(a=None) == 1
    for name in ("x", "b", "g", "s", "q", "a", "rs", "r"):
        assert fwd(**{name: BAD}) == 3
    assert fwd(x=None, b=None, s=None, q=None, a=None, M=0) == 0

    need = mmf.mmf_add_act_quant_bwd_workspace_bytes(4, 32)
    assert need > 0 and need % 256 == 0 and mmf.mmf_add_act_quant_bwd_workspace_bytes(4, 24) == 0

    def bwd(dy=A, df=1, do=A, s=A, sf=0, g=A, r=A, ds=A, dh=A, dg=A, M=4, K=32, ws=A, n=need):
        return lib.mmf_add_act_quant_bwd(dy, df, do, s, sf, g, r, ds, dh, dg, M, K, ws, n, S)

    assert bwd(K=24) == 2 and bwd(M=-1) == 2 and bwd(df=2) == 4 and bwd(sf=3) == 4
    for name in ("dy", "s", "r", "ds"):
        assert bwd(**{name: None}) == 1
    for name in ("dy", "do", "s", "g", "r", "ds", "dh", "dg"):
        assert bwd(**{name: BAD}) == 3
    assert bwd(n=need - 1) == 6 and bwd(ws=A + 16) == 6
    assert bwd(dy=None, M=0) == 0


def test_workspace_of_a_batch_serves_smaller_ones(mmf):
    for K in (16, 1040, 2048, 5120):
        sizes = [mmf.mmf_add_act_quant_bwd_workspace_bytes(M, K) for M in range(1, 5000, 7)]
        assert sizes == sorted(sizes)


def test_binding_refuses_what_it_cannot_take(mmf):
    x = torch.zeros(2, 16)
    with pytest.raises(ValueError, match="HIP device"):
        mmf.mmf_add_act_quant(x, x, None, x, x, x)
    with pytest.raises(TypeError):
        mmf.mmf_add_act_quant(x.half(), x, None, x, x, x)
    with pytest.raises(TypeError):
        mmf.mmf_add_act_quant_bwd(x.half(), None, x, None, x, x, None, None)


@pytest.mark.gpu
def test_binding_refuses_shapes_and_types(mmf):
    x = torch.zeros((2, 32), device=dev())
    q, a = torch.zeros((2, 32), dtype=torch.int8, device=dev()), torch.zeros(2, device=dev())
    for bad in (dict(branch=x[:, ::2]), dict(branch=x[:1]), dict(s=x.bfloat16()), dict(s=None), dict(q=q.int()),
                dict(a=a[:1]), dict(branch=x.double())):
        k = dict(branch=x.clone(), s=x.clone(), q=q, a=a)
        k.update(bad)
        with pytest.raises((TypeError, ValueError)):
            mmf.mmf_add_act_quant(x, k["branch"], None, k["s"], k["q"], k["a"])


@pytest.mark.gpu
def test_on_another_stream_and_captured(mmf):
    """The calls run on the given stream; a captured forward and backward
    replay to the eager results, with eager work between the replays."""
    g = gen(9)
    x, b, dy = rand(g, 33, 2048, dtype=BF), rand(g, 33, 2048), rand(g, 33, 2048)
    s, q, a, rs, r = mmf.add_act_quant(x, b, None)
    ds, dg = torch.empty((33, 2048), device=dev()), torch.empty(2048, device=dev())
    ws = torch.empty(mmf.mmf_add_act_quant_bwd_workspace_bytes(33, 2048), dtype=torch.uint8, device=dev())
    mmf.mmf_add_act_quant_bwd(dy, None, s, None, r, ds, None, dg, ws)
    want = [t.clone() for t in (s, q, a, rs, r, ds, dg)]
    outs = (s, q, a, rs, r, ds, dg)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    torch.cuda.synchronize()
    mmf.mmf_add_act_quant(x, b, None, s, q, a, rs, r, st)
    mmf.mmf_add_act_quant_bwd(dy, None, s, None, r, ds, None, dg, ws, st)
    st.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mmf.mmf_add_act_quant(x, b, None, s, q, a, rs, r)
        mmf.mmf_add_act_quant_bwd(dy, None, s, None, r, ds, None, dg, ws)
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(outs, want))
