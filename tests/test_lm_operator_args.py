"""Linear attention, beam search and distillation without a GPU: what the calls
refuse (no pointer is dereferenced on these paths) and, behind tests/fake_hip.c,
which kernels they launch, that the largest shapes stay within a launch's limits
and that what they allocate is freed.  fake_hip.c refuses a launch past the
runtime's limits."""
import ctypes
import json
import os
import subprocess
import sys
import tempfile

import pytest
import torch

from record import HERE, LIB, call, kernels, record

A, B, C, D, E, F = (0x10000 * i for i in range(1, 7))
BAD = 0x10004
WS = 0x100000
S = None
OK, NULL, SHAPE, ALIGN, DTYPE, HIP, WORKSPACE, ARG = range(8)


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def linattn(lib, qkv=A, f32=0, decay=B, s0=C, o=D, s_last=E, dims=(2, 100, 3, 32, 48), ws=None, n=0):
    return lib.mmf_linattn_fwd(qkv, f32, decay, 1.0, s0, o, s_last, *dims, ws, n, S)


def linattn_bwd(lib, qkv=A, f32=0, decay=B, s0=C, do=D, do_f32=0, ds=E, dqkv=F, ds0=E, dims=(2, 100, 3, 32, 48), ws=None,
                n=0):
    return lib.mmf_linattn_bwd(qkv, f32, decay, 1.0, s0, do, do_f32, ds, dqkv, ds0, *dims, ws, n, S)


@pytest.mark.parametrize("dims", [(1, 1, 1, 8, 16), (1, 1, 1, 16, 24), (1, 1, 1, 0, 16), (1, 1, 1, 16, -16), (1, 1, 1, 272, 16),
                                  (1, 1, 1, 16, 272), (1, 1, 0, 16, 16), (-1, 1, 1, 16, 16), (1, -1, 1, 16, 16),
                                  (2 ** 20 + 1, 1, 1, 16, 16), (2 ** 18, 1, 5, 16, 16), (1, 1, 2 ** 14, 64, 64),
                                  (2 ** 17 + 1, 1, 1, 256, 256), (4, 2 ** 29, 1, 16, 16), (1, 2 ** 31, 1, 16, 16)], ids=str)
def test_linattn_shapes(mmf, dims):
    lib = mmf._lib
    assert linattn(lib, dims=dims) == SHAPE and linattn_bwd(lib, dims=dims) == SHAPE
    assert mmf.mmf_linattn_workspace_bytes(*dims) == 0 and mmf.mmf_linattn_bwd_workspace_bytes(*dims) == 0


def test_linattn_arguments(mmf):
    lib = mmf._lib
    for name in ("qkv", "decay", "o"):
        assert linattn(lib, **{name: None}) == NULL
    for name in ("qkv", "decay", "s0", "o", "s_last"):
        assert linattn(lib, **{name: BAD}) == ALIGN
    for name in ("qkv", "decay", "do", "dqkv"):
        assert linattn_bwd(lib, **{name: None}) == NULL
    for name in ("qkv", "decay", "s0", "do", "ds", "dqkv", "ds0"):
        assert linattn_bwd(lib, **{name: BAD}) == ALIGN
    assert linattn(lib, f32=2) == linattn_bwd(lib, f32=-1) == linattn_bwd(lib, do_f32=3) == DTYPE
    long = (2, 4000, 3, 32, 48)
    need, need_bwd = mmf.mmf_linattn_workspace_bytes(*long), mmf.mmf_linattn_bwd_workspace_bytes(*long)
    assert need > 0 and need % 256 == 0 and need_bwd > 0 and need_bwd % 256 == 0
    assert linattn(lib, dims=long, ws=WS, n=need - 1) == linattn(lib, dims=long, ws=WS + 16, n=need) == WORKSPACE
    assert linattn_bwd(lib, dims=long, ws=WS, n=need_bwd - 1) == WORKSPACE
    assert linattn_bwd(lib, dims=long, ws=WS + 128, n=need_bwd) == WORKSPACE
    for dims in ((0, 7, 3, 32, 48), (2, 0, 3, 32, 48)):
        assert linattn(lib, None, 0, None, None, None, None, dims) == OK
        assert linattn_bwd(lib, None, 0, None, None, None, 0, None, None, None, dims) == OK


def beam(lib, z=A, f32=0, scores=B, done=C, end=2, ns=D, tokens=E, parents=F, nd=None, dims=(2, 3, 100, 4), ws=None, n=0):
    return lib.mmf_beam_select(z, f32, scores, done, end, ns, tokens, parents, nd, *dims, ws, n, S)


@pytest.mark.parametrize("dims", [(-1, 1, 1, 1), (1, 0, 5, 1), (1, 65, 5, 1), (1, 2, 0, 1), (1, 2, 5, 0), (1, 2, 5, 11),
                                  (1, 2, 100, 65), (1, 1, 2 ** 18 + 1, 1), (2 ** 23 + 1, 1, 1, 1), (2 ** 17, 64, 1025, 1)],
                         ids=str)
def test_beam_shapes(mmf, dims):
    assert beam(mmf._lib, done=None, end=-1, dims=dims) == SHAPE
    assert mmf.mmf_beam_select_workspace_bytes(*dims) == 0


def test_beam_arguments(mmf):
    lib = mmf._lib
    for name in ("z", "scores", "ns", "tokens", "parents"):
        assert beam(lib, **{name: None}) == NULL
    for name in ("z", "scores", "done", "ns", "tokens", "parents", "nd"):
        assert beam(lib, **{name: BAD}) == ALIGN
    assert beam(lib, f32=2) == DTYPE
    assert beam(lib, end=-1) == beam(lib, end=-2, done=None) == beam(lib, end=100) == ARG
    need = mmf.mmf_beam_select_workspace_bytes(2, 3, 100, 4)
    assert need > 0 and need % 256 == 0
    assert beam(lib, ws=WS, n=need - 1) == beam(lib, ws=WS + 16, n=need) == WORKSPACE
    assert beam(lib, None, 0, None, None, -1, None, None, None, None, (0, 3, 100, 4)) == OK


def test_reorder_arguments(mmf):
    lib = mmf._lib
    P, I = ctypes.c_void_p, ctypes.c_int64

    def reorder(src=(A, B), dst=(C, D), rows=(32, 64), parents=E, Bn=2, W=3, count=None):
        n = len(rows)
        return lib.mmf_beam_reorder((P * n)(*src), (P * n)(*dst), (I * n)(*rows), n if count is None else count, parents, Bn, W, S)

    assert reorder(src=(A, None)) == reorder(dst=(None, D)) == reorder(parents=None) == NULL
    assert lib.mmf_beam_reorder(None, None, None, 1, E, 2, 3, S) == NULL
    assert reorder(src=(A, BAD)) == reorder(dst=(BAD, D)) == reorder(parents=BAD) == ALIGN
    assert reorder(rows=(32, 24)) == reorder(rows=(-16, 32)) == reorder(rows=(32, 2 ** 31)) == SHAPE
    assert reorder(rows=(32, 2 ** 30), Bn=9) == SHAPE
    assert reorder(W=0) == reorder(W=65) == reorder(Bn=-1) == reorder(Bn=2 ** 23 + 1) == reorder(count=-1) == SHAPE
    assert lib.mmf_beam_reorder(None, None, None, 0, None, 2, 3, S) == OK
    assert reorder(src=(None, None), dst=(None, None), rows=(0, 0)) == OK
    assert reorder(src=(None, None), dst=(None, None), parents=None, Bn=0) == OK


def distill(lib, z=A, zf=0, idx=B, t=C, tf=0, tau=1.0, loss=D, M=4, V=100, K=5):
    return lib.mmf_distill_fwd(z, zf, idx, t, tf, tau, loss, M, V, K, S)


def distill_bwd(lib, z=A, zf=0, idx=B, t=C, tf=0, tau=1.0, dloss=D, dz=E, df=0, loss=F, M=4, V=100, K=5):
    return lib.mmf_distill_bwd(z, zf, idx, t, tf, tau, dloss, dz, df, loss, M, V, K, S)


def test_distill_arguments(mmf):
    lib = mmf._lib
    for f in (distill, distill_bwd):
        for bad in ({"M": -1}, {"M": 2 ** 22}, {"V": 0}, {"V": 2 ** 24 + 1}, {"K": 0}, {"K": 1025}):
            assert f(lib, **bad) == SHAPE, bad
        for tau in (0.0, -1.0, 1e-39, float("inf"), float("nan")):
            assert f(lib, tau=tau) == ARG
        assert f(lib, zf=2) == f(lib, tf=-1) == DTYPE
    for name in ("z", "idx", "t", "loss"):
        assert distill(lib, **{name: None}) == NULL and distill(lib, **{name: BAD}) == ALIGN
    for name in ("z", "idx", "t", "dloss", "dz"):
        assert distill_bwd(lib, **{name: None}) == NULL and distill_bwd(lib, **{name: BAD}) == ALIGN
    assert distill_bwd(lib, loss=BAD) == ALIGN and distill_bwd(lib, df=2) == DTYPE
    assert distill_bwd(lib, dz=A, df=1) == ARG
    assert distill(lib, None, 0, None, None, 0, 1.0, None, 0) == OK
    assert distill_bwd(lib, None, 0, None, None, 0, 1.0, None, None, 0, None, 0) == OK


def test_binding_refuses_before_the_call(mmf):
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)  # noqa: E731
    half = z(2, 96, t=torch.float16)
    with pytest.raises(TypeError):
        mmf.mmf_linattn_fwd(half, 2, 1, 2, 16, 16, z(2), 1.0, None, half, None)
    with pytest.raises(ValueError):   # not on the GPU
        mmf.mmf_linattn_fwd(z(2, 96), 2, 1, 2, 16, 16, z(2), 1.0, None, z(2, 32), None)
    with pytest.raises(ValueError):   # shape
        mmf.mmf_linattn_bwd(z(2, 95), 2, 1, 2, 16, 16, z(2), 1.0, None, z(2, 32), None, z(2, 96), None)
    for bad in (z(()), z(6), z(6, 0)):
        with pytest.raises(ValueError):
            mmf.mmf_beam_select(bad, z(2, 3), None, -1, 2, 3, 4, z(2, 4), z(2, 4), z(2, 4),
                                None)
    with pytest.raises(TypeError):
        mmf.mmf_beam_reorder(z(6, 4), z(2, 3, t=torch.int32), 2, 3)
    for bad in (z(()), z(5, 4), z(4, 6).t()):
        with pytest.raises((TypeError, ValueError)):
            mmf.mmf_beam_reorder([bad], z(2, 3, t=torch.int32), 2, 3)
    with pytest.raises(ValueError):
        mmf.mmf_distill_fwd(z(4, 10), z(4, t=torch.int32), z(4), 1.0, z(4))
    with pytest.raises(TypeError):
        mmf.mmf_distill_bwd(half, z(2, 3, t=torch.int32), z(2, 3), 1.0, z(2), half)


# ---- launches (addresses made up, never read) ----
BIG = 1 << 60
P = 0x100000000


def fwd_call(f32, dims, ws=P, n=BIG, **kw):  # without `scale`, which goes in another kind of register
    return call("mmf_linattn_fwd", P, f32, P, P, P, P, *dims, ws, n, None, **kw)


def bwd_call(f32, do_f32, dims, ds0=P, ws=P, n=BIG, **kw):
    return call("mmf_linattn_bwd", P, f32, P, P, P, do_f32, P, P, ds0, *dims, ws, n, None, **kw)


def test_few_tokens_go_one_by_one_and_more_as_chunks():
    step, chunk, join = ("linattn_step_kernel", "linattn_chunk_kernel", "linattn_join_kernel")
    bare = lambda r: [k.split("::")[-1] for k in kernels(r)]  # noqa: E731
    dims = lambda T: (2, T, 4, 64, 64)  # noqa: E731
    rs = record([fwd_call(1, dims(8)), fwd_call(1, dims(9)), fwd_call(0, dims(2)), fwd_call(0, dims(3)),
                 fwd_call(1, dims(5000)), bwd_call(0, 0, dims(1), 2 * P), bwd_call(1, 1, dims(128), 2 * P),
                 bwd_call(0, 0, dims(1), P), bwd_call(1, 0, dims(1)), bwd_call(1, 0, dims(1), None), bwd_call(1, 0, dims(5000))])
    assert all(r["status"] == OK and r["allocs"] == r["frees"] == 0 for r in rs)
    sums = [chunk, join, chunk]   # [chunk, chunk]: ds0 in the place of ds_last
    assert [bare(r) for r in rs] == [[step], [chunk], [step], [chunk], sums, [chunk], [chunk], [chunk, chunk], sums, [chunk],
                                    sums]


@pytest.mark.parametrize("dims", [(2 ** 20, 1, 1, 16, 16), (2 ** 20, 70, 1, 64, 128), (2 ** 17, 70, 1, 256, 256),
                                  (1, 70, 7710, 128, 16), (1, 2 ** 31 - 1, 1, 16, 16), (1, 2 ** 31 - 1, 8, 256, 16),
                                  (511, 2 ** 22, 1, 128, 128), (1, 1, 43690, 16, 16)], ids=str)
def test_largest_linattn_shapes_launch(mmf, dims):
    rs = record([fwd_call(0, dims), fwd_call(1, dims), bwd_call(0, 0, dims), bwd_call(1, 1, dims), bwd_call(0, 1, dims, None)])
    assert [r["status"] for r in rs] == [OK] * 5


def test_linattn_workspaces(mmf):
    dims = (2, 5000, 4, 64, 64)
    need, need_bwd = mmf.mmf_linattn_workspace_bytes(*dims), mmf.mmf_linattn_bwd_workspace_bytes(*dims)
    rs = record([fwd_call(0, dims, None, 0), bwd_call(0, 0, dims, P, None, 0), fwd_call(0, dims, P, need),
                 bwd_call(0, 0, dims, P, P, need_bwd), fwd_call(0, dims, None, 0, fail_alloc=True),
                 bwd_call(0, 0, dims, P, None, 0, fail_alloc=True)])
    assert [r["status"] for r in rs] == [OK] * 4 + [HIP] * 2
    assert [(r["allocs"], r["frees"]) for r in rs[:4]] == [(1, 1)] * 2 + [(0, 0)] * 2
    assert all(not r["launches"] for r in rs[4:])


def test_beam_launches(mmf):
    def sel(dims, ws=P, n=BIG, **kw):
        return call("mmf_beam_select", P, 0, P, P, 0, P, P, P, P, *dims, ws, n, None, **kw)

    largest = [(2 ** 23, 1, 1, 1), (2 ** 17, 64, 1024, 64), (2 ** 15, 1, 2 ** 18, 64), (1, 64, 2 ** 18, 64), (1, 1, 1, 1)]
    need = mmf.mmf_beam_select_workspace_bytes(2, 3, 50000, 4)
    rs = record([sel(d) for d in largest] + [sel((2, 3, 50000, 4), None, 0), sel((2, 3, 50000, 4), P, need),
                                            sel((2, 3, 50000, 4), None, 0, fail_alloc=True)])
    assert [r["status"] for r in rs] == [OK] * 7 + [HIP]
    assert all(kernels(r) == ["beam_piece_kernel", "beam_final_kernel"] for r in rs[:7]) and not rs[7]["launches"]
    assert [(r["allocs"], r["frees"]) for r in rs[5:7]] == [(1, 1), (0, 0)]


CHILD = """
import ctypes, json, sys
so, lib = sys.argv[1:3]
fake = ctypes.CDLL(so, mode=ctypes.RTLD_GLOBAL)
mmf = ctypes.CDLL(lib)
fake.fake_reset.argtypes = [ctypes.c_int] * 4 + [ctypes.c_void_p]
P, I = ctypes.c_void_p(0x100000000), ctypes.c_int64
def of(f, *args):
    fake.fake_reset(0, 0, 0, 0, None)
    status = f(*args)
    return status, fake.fake_launches(), fake.fake_allocs()
out = []
for M, V, K in json.loads(sys.argv[3]):
    for kind in (0, 1):
        out.append(of(mmf.mmf_distill_fwd, P, kind, P, P, kind, ctypes.c_float(1.0), P, I(M), I(V), I(K), None))
        for d in (0, 1):
            out.append(of(mmf.mmf_distill_bwd, P, kind, P, P, kind, ctypes.c_float(1.0), P, P if kind == d else
                          ctypes.c_void_p(0x200000000), d, None, I(M), I(V), I(K), None))
for n, rows, B, W in ((1, 2 ** 31 - 16, 4, 64), (3, 2 ** 30, 8, 16), (300, 16, 2 ** 23, 1), (2000, 4096, 5, 7)):
    a, r = (ctypes.c_uint64 * n)(*[0x100000000 * (i + 1) for i in range(n)]), (I * n)(*[rows] * n)
    s = of(mmf.mmf_beam_reorder, a, a, r, I(n), P, I(B), I(W), None)
    out.append((s[0], int(s[1] > 0 and s[1] <= n), s[2]))
print(json.dumps(out))
"""


def test_largest_distill_and_reorder_shapes_launch_and_nothing_is_allocated():
    shapes = [(2 ** 22 - 1, 1, 1), (2 ** 22 - 1, 2 ** 24, 1024), (2 ** 22 - 1, 65536, 16), (1, 2 ** 24, 1)]
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "fake_hip.so")
        subprocess.run(["gcc", "-O1", "-std=c11", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.c"), "-o", so], check=True)
        r = subprocess.run([sys.executable, "-c", CHILD, so, LIB, json.dumps(shapes)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert json.loads(r.stdout) == [[OK, 1, 0]] * (6 * len(shapes) + 4)
