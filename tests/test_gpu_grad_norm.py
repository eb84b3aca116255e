"""The norm over a set of gradients and the set scaled to it (mmf_grad_norm,
mmf_grad_clip), against 64 bits and, given the norm, bit for bit.

Squares and sums are fp64 and the root is rounded once to fp32: the norm is
within half a step (u = 2^-24) of the exact one, and 1 % of that for fp64's
own.  The factor and the products are single fp32 operations, so they are
compared bit for bit with the same operations on the CPU."""
import ctypes

import numpy as np
import pytest
import torch

from _parity import dev, log

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def grads_of(seed, counts, bf16=lambda i: False, scale=1.0):
    """Gradients inside guarded buffers: (whole, view) each."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(counts):
        whole = torch.full((n + 24,), 7.0, dtype=BF if bf16(i) else F32, device=dev())
        view = whole[8:8 + n]
        view.copy_(torch.randn(n, generator=g, device=dev()) * scale)
        out.append((whole, view))
    return out


def guards_hold(pairs):
    return all((w[:8] == 7).all() and (w[8 + v.numel():] == 7).all() for w, v in pairs)


def factor(norm, max_norm):
    with np.errstate(all="ignore"):
        c = np.float32(max_norm) / (np.float32(norm) + np.float32(1e-6))
    return np.float32(1.0) if c > 1 else c


def scaled(g, c):
    return (g.cpu().float() * torch.tensor(c)).to(g.dtype)


def check(mmf, counts, max_norm, bf16=lambda i: False, scale=1.0, in_place=False, seed=0):
    log(f"[grad_norm] n={len(counts)} sum={sum(counts)} max_norm={max_norm} in_place={in_place}")
    pairs = grads_of(seed, counts, bf16, scale)
    grads = [v for _, v in pairs]
    before = [g.clone() for g in grads]
    norm = torch.full((1,), float("nan"), device=dev())
    need = mmf.mmf_grad_norm_workspace_bytes(counts)
    ws = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device=dev())
    mmf.mmf_grad_norm(grads, norm, ws[:need])
    want = float(sum(g.double().square().sum() for g in grads)) ** 0.5 if counts else 0.0
    assert abs(float(norm) - want) <= 1.01 * U * want
    assert (ws[need:] == 0xAB).all()
    outs = None
    if not in_place:
        opairs = grads_of(seed + 1, counts, bf16)
        outs = [v for _, v in opairs]
    mmf.mmf_grad_clip(grads, norm, max_norm, outs)
    torch.cuda.synchronize()
    c = factor(float(norm), max_norm)
    for b, g, o in zip(before, grads, grads if in_place else outs):
        assert torch.equal(o.cpu(), scaled(b, c))
        if not in_place:
            assert torch.equal(g, b)
    assert guards_hold(pairs) and (in_place or guards_hold(opairs))
    return norm


COUNTS = [0, 1, 3, 4, 5, 7, 8, 9, 255, 1025, 16383, 16384, 16385, 100001, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True], ids=["out", "in_place"])
@pytest.mark.parametrize("kinds", ["f32", "bf16", "mixed"])
def test_sizes(mmf, kinds, in_place):
    bf = {"f32": lambda i: False, "bf16": lambda i: True, "mixed": lambda i: i % 2 == 0}[kinds]
    for max_norm in (1.0, 0.0, 1e9, float("inf")):
        check(mmf, COUNTS, max_norm, bf, in_place=in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 127, 128, 129, 300])
def test_many_tensors(mmf, n):
    check(mmf, [(37 * i) % 900 + (i % 3) * 8192 for i in range(n)], 0.5, lambda i: i % 5 == 0)


@pytest.mark.gpu
def test_one_large_tensor(mmf):
    check(mmf, [(1 << 26) + 3], 1.0)


@pytest.mark.gpu
def test_offsets_past_32_bits(mmf):
    """One array of 4.4 GB: ones, whose squares sum up exactly."""
    n = 1_100_000_003
    g = torch.ones(n, device=dev())
    norm = torch.zeros(1, device=dev())
    mmf.mmf_grad_norm([g], norm)
    assert abs(float(norm) - n ** 0.5) <= U * n ** 0.5
    mmf.mmf_grad_clip([g], norm, 1.0)
    c = float(factor(float(norm), 1.0))
    assert float(g.min()) == c and float(g.max()) == c


@pytest.mark.gpu
def test_small_and_large_values(mmf):
    """Squares that fp32 could not hold."""
    check(mmf, [1000, 33], 1.0, scale=1e-25)
    check(mmf, [1000, 33], 1.0, scale=1e25)


@pytest.mark.gpu
def test_no_tensors(mmf):
    norm = check(mmf, [], 1.0)
    assert float(norm) == 0.0
    assert float(check(mmf, [0, 0], 1.0)) == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite(mmf, bad):
    """NaN spreads to every output; an infinite norm scales by 0, which
    leaves NaN where the infinity was."""
    g = torch.ones(100, device=dev())
    h = torch.ones(20000, device=dev(), dtype=BF)
    h[19999] = bad
    norm = torch.zeros(1, device=dev())
    mmf.mmf_grad_norm([g, h], norm)
    assert torch.isnan(norm).all() if bad != bad else torch.isinf(norm).all()
    mmf.mmf_grad_clip([g, h], norm, 1.0)
    torch.cuda.synchronize()
    assert torch.isnan(h[19999])
    if bad != bad:
        assert torch.isnan(g).all() and torch.isnan(h).all()
    else:
        assert (g == 0).all() and (h[:19999] == 0).all()


@pytest.mark.gpu
def test_shapes_repeatability_stream_and_capture(mmf):
    gen = torch.Generator(device="cuda").manual_seed(4)
    grads = [torch.randn(s, generator=gen, device=dev()) for s in ((300, 401), (7,), (), (3, 5, 77777))]
    outs = [torch.empty_like(g) for g in grads]
    norm = torch.zeros(1, device=dev())
    ws = torch.empty(mmf.mmf_grad_norm_workspace_bytes([g.numel() for g in grads]), dtype=torch.uint8, device=dev())

    def step(stream=None):
        mmf.mmf_grad_norm(grads, norm, ws, stream)
        mmf.mmf_grad_clip(grads, norm, 1.0, outs, stream)

    step()
    torch.cuda.synchronize()
    want = [norm.clone()] + [o.clone() for o in outs]
    st = torch.cuda.Stream()
    step(st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip([norm] + outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in [norm] + outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([norm] + outs, want))


A, BAD, S = 0x100000, 0x100004, None


def test_refusals(mmf):
    lib = mmf._lib

    def arrays(ptrs, kinds, counts):
        n = len(counts)
        return (ctypes.c_void_p * n)(*ptrs), (ctypes.c_int * n)(*kinds), (ctypes.c_int64 * n)(*counts), n

    def norm(ptrs=(A, A), kinds=(0, 1), counts=(5, 6), out=A, ws=A, wn=1 << 20, n=None):
        p, k, c, m = arrays(ptrs, kinds, counts)
        return lib.mmf_grad_norm(p, k, c, m if n is None else n, out, ws, wn, S)

    def clip(ptrs=(A, A), kinds=(0, 1), counts=(5, 6), norm=A, mx=1.0, outs=(A, A), n=None):
        p, k, c, m = arrays(ptrs, kinds, counts)
        o = None if outs is None else (ctypes.c_void_p * len(outs))(*outs)
        return lib.mmf_grad_clip(p, k, c, m if n is None else n, norm, mx, o, S)

    for f in (norm, clip):
        assert f(counts=(5, -1)) == 2 and f(counts=(5, (1 << 36) + 1)) == 2 and f(n=-1) == 2
        assert f(kinds=(0, 2)) == 4
        assert f(ptrs=(A, None)) == 1 and f(ptrs=(A, BAD)) == 3
    assert norm(out=None) == 1 and norm(out=BAD) == 3
    assert norm(wn=0) == 6 and norm(ws=A + 16) == 6
    assert clip(norm=None) == 1 and clip(norm=BAD) == 3 and clip(outs=None) == 1
    assert clip(outs=(A, None)) == 1 and clip(outs=(BAD, A)) == 3
    assert clip(mx=-1.0) == 7 and clip(mx=float("nan")) == 7
    assert lib.mmf_grad_norm(None, None, None, 1, A, A, 1 << 20, S) == 1
    assert lib.mmf_grad_clip(None, None, None, 0, A, 1.0, None, S) == 0
    assert mmf.mmf_grad_norm_workspace_bytes([1, 0, 16385]) >= 3 * 8
    assert mmf.mmf_grad_norm_workspace_bytes([-1]) == 0 and mmf.mmf_grad_norm_workspace_bytes([]) == 0


@pytest.mark.gpu
def test_a_tensor_in_the_list_twice(mmf):
    """It counts twice in the norm, and is refused where it would be written
    twice; empty tensors may share an address."""
    g, e = torch.ones(100, device=dev()), torch.empty(0, device=dev())
    norm = torch.zeros(1, device=dev())
    mmf.mmf_grad_norm([g, e, g, e], norm)
    assert abs(float(norm) - 200 ** 0.5) <= 2 * U * 200 ** 0.5
    with pytest.raises(ValueError, match="twice"):
        mmf.mmf_grad_clip([g, e, g], norm, 1.0)
    o = torch.empty_like(g)
    with pytest.raises(ValueError, match="twice"):
        mmf.mmf_grad_clip([g, g], norm, 1.0, [o, o])
    p = torch.empty_like(g)
    mmf.mmf_grad_clip([g, e, g, e], norm, 1.0, [o, e, p, e])
    assert torch.equal(o, p) and float(o[0]) == float(factor(float(norm), 1.0))


@pytest.mark.gpu
def test_a_generator_of_tensors(mmf):
    gs = [torch.full((30,), 2.0, device=dev()), torch.full((7,), 1.0, device=dev()).bfloat16()]
    outs = [torch.empty_like(g) for g in gs]
    norm, want = torch.zeros(1, device=dev()), (30 * 4 + 7) ** 0.5
    mmf.mmf_grad_norm((g for g in gs), norm)
    assert abs(float(norm) - want) <= 2 * U * want
    mmf.mmf_grad_clip((g for g in gs), norm, 1.0, (o for o in outs))
    mmf.mmf_grad_clip(dict(enumerate(gs)).values(), norm, 1.0)
    c = factor(float(norm), 1.0)
    assert float(outs[0][29]) == float(gs[0][29]) == float(torch.tensor(2.0) * c)
    assert float(outs[1][6]) == float(gs[1][6]) == float((torch.tensor(1.0) * c).bfloat16())
    for one in (lambda: mmf.mmf_grad_norm(gs[0], norm), lambda: mmf.mmf_grad_clip(gs[0], norm, 1.0),
                lambda: mmf.mmf_grad_clip([gs[0]], norm, 1.0, outs[0])):
        with pytest.raises(TypeError, match="list"):
            one()


@pytest.mark.gpu
def test_binding_refuses(mmf):
    g = torch.zeros((4, 8), device=dev())
    norm = torch.zeros(1, device=dev())
    for bad in ([g.t()], [g, g.half()], [g.cpu()], [g, 3], [g.double()]):
        with pytest.raises((TypeError, ValueError)):
            mmf.mmf_grad_norm(bad, norm)
    for outs in ([g, g], [g.bfloat16()], [g[:2]], [g.t()]):
        with pytest.raises((TypeError, ValueError)):
            mmf.mmf_grad_clip([g], norm, 1.0, outs)
    with pytest.raises((TypeError, ValueError)):
        mmf.mmf_grad_norm([g], norm.double())
