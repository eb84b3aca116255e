"""Linear attention near the ends of fp32's range: what the recurrence in 32 bits
holds, the chunks hold too.  Values of 1e33 with keys of 1e-3 make entries of the
state of 1e30, which decays take down (or, above 1, small ones up) over many
chunks; no factor of its own may stand between a value and the state.  Error
bounds as derived in test_gpu_linattn.py."""
import pytest
import torch

from _parity import log
from test_gpu_linattn import BF, F32, check_bwd, check_fwd, inputs, run_bwd, run_fwd

DECAYS = [0.65, 0.5, 0.8, 0.95, 1.0, 0.3, -0.65]
GROWING = [1.5, 1.1, 1.04, -1.5]


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def scaled(p, q=1.0, k=1.0, v=1.0, s0=1.0, do=1.0, ds=1.0):
    """The inputs with each part in units of its own."""
    _, _, H, dk, dv = p["dims"]
    t = p["qkv"].dtype
    unit = torch.cat([torch.full((H * dk,), q), torch.full((H * dk,), k), torch.full((H * dv,), v)])
    p["qkv"] = (p["qkv"].float() * unit).to(t)
    p["dout"] = (p["dout"].float() * do).to(t)
    p["s0"], p["ds_last"] = p["s0"] * s0, p["ds_last"] * ds
    return p


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [40, 64, 130, 700])
@pytest.mark.parametrize("dk,dv", [(32, 48), (128, 128), (256, 64)])
def test_large_values(mmf, dk, dv, T, t):
    log(f"[linattn] large {dk} {dv} T={T} {t}")
    H = len(DECAYS)
    p = scaled(inputs(1, T, H, dk, dv, t, seed=T, decay=DECAYS), q=1e-3, k=1e-3, v=1e33, s0=1e30)
    o, s = run_fwd(mmf, p)
    assert o.isfinite().all() and s.isfinite().all()
    check_fwd(p, o, s)
    # backward: of q and dout the same, and of v and k
    for part in ({"do": 1e33, "q": 1e-3, "k": 1e-3, "v": 1e-3, "ds": 1e30, "s0": 1e-3},
                 {"q": 1e33, "do": 1e-3, "k": 1e-3, "v": 1e-3, "ds": 1e30, "s0": 1e-3},
                 {"k": 1e33, "v": 1e-3, "do": 1e-3, "q": 1e-3, "s0": 1e30, "ds": 1e-3}):
        p = scaled(inputs(1, T, H, dk, dv, t, seed=T + 1, decay=DECAYS), **part)
        dqkv, g = run_bwd(mmf, p, t)
        assert dqkv.isfinite().all() and g.isfinite().all()
        check_bwd(p, dqkv, g)


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [40, 64, 130])
def test_small_values_that_grow(mmf, T, t):
    H = len(GROWING)
    p = scaled(inputs(1, T, H, 48, 80, t, seed=T, decay=GROWING), k=1e-3, v=1e-26, s0=1e-29)
    check_fwd(p, *run_fwd(mmf, p))
    p = scaled(inputs(1, T, H, 48, 80, t, seed=T + 1, decay=GROWING), q=1e-3, do=1e-26, ds=1e-29, s0=1e-29, k=1e-3, v=1e-26)
    check_bwd(p, *run_bwd(mmf, p, t))
