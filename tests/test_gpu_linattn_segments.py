"""Linear attention whose sequences are cut into segments: a few, many, a short
last one, states of every width joined by a lane per entry and by a lane per
four.  The recurrence in 64 bits runs on the device.  Error bounds as derived in
test_gpu_linattn.py."""
import pytest
import torch

from _parity import dev, log
from record import call, record
from test_gpu_linattn import BF, F32, check_bwd, check_fwd, inputs, run_bwd, run_fwd

# (B, T, H, dk, dv)
SHAPES = [(1, 161, 16, 128, 128), (2, 193, 5, 192, 160), (4, 482, 2, 176, 256), (2, 197, 16, 208, 128), (1, 1500, 2, 128, 128),
          (1, 3000, 1, 128, 128), (1, 900, 2, 256, 208), (1, 2000, 1, 16, 256), (1, 1111, 3, 256, 16)]
# states of 2^20 entries and more (of both directions' states, of S and of its
# gradient, together), which a lane joins four by four; the last has segments
# forward alone
WIDE = [(4, 2048, 16, 128, 128), (2, 1025, 8, 256, 256), (2, 700, 16, 128, 128), (1, 1100, 16, 256, 144), (4, 700, 16, 128, 128)]


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def on_device(p):
    return {k: v.to(dev()) if isinstance(v, torch.Tensor) else v for k, v in p.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("t", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES + WIDE, ids=str)
def test_forward_in_segments(mmf, shape, t):
    log(f"[linattn] segments {shape} {t}")
    p = on_device(inputs(*shape, t, seed=sum(shape)))
    check_fwd(p, *(x.to(dev()) for x in run_fwd(mmf, p)))


@pytest.mark.gpu
@pytest.mark.parametrize("t,do_t", [(F32, F32), (BF, BF), (F32, BF), (BF, F32)], ids=["f32", "bf16", "f32-bf16", "bf16-f32"])
@pytest.mark.parametrize("shape", SHAPES + WIDE, ids=str)
def test_backward_in_segments(mmf, shape, t, do_t):
    log(f"[linattn] segments, backward {shape} {t} {do_t}")
    p = on_device(inputs(*shape, t, seed=1 + sum(shape)))
    p["dout"] = p["dout"].to(do_t)
    check_bwd(p, *(x.to(dev()) for x in run_bwd(mmf, p, do_t)))
    p["ds_last"] = None
    check_bwd(p, run_bwd(mmf, p, do_t, ds0=False)[0].to(dev()), None)


def test_the_shapes_take_the_joins_that_they_are_meant_for():
    P, BIG = 0x100000000, 1 << 60
    calls = []
    for dims in SHAPES + WIDE:
        for f32 in (0, 1):
            calls.append(call("mmf_linattn_fwd", P, f32, P, P, P, P, *dims, P, BIG, None))
            calls.append(call("mmf_linattn_bwd", P, f32, P, P, P, f32, P, P, 2 * P, *dims, P, BIG, None))
    rs = record(calls)
    joins = [[l["kernel"][-3:] for l in r["launches"] if "join" in l["kernel"]] for r in rs]
    few, wide = joins[:4 * len(SHAPES)], joins[4 * len(SHAPES):]
    assert all(few) and few.count(["<1>"]) >= 20
    assert wide[:8] == [["<4>"]] * 8 and wide[9:16:2] == [["<4>"]] * 4 and wide[16:] == [["<4>"], []] * 2
