"""The gradient of the forget gate's lower bound (dlb of mmf_mlgru_scan_bwd)
is a sum in 64 bits from its first term on.

Terms that cancel: with f = 0 (zf far out, no bound) a token's state is its
candidate and its gradient its own, so a term is
  do g s(h) (1 - s(h)) (h_{t-1} - c)
and the tokens at even places take c = 32 (s(h) = 1 in fp32: term 0), those at
odd places c = 0 behind h = 32: term 8 do g.  Every eight tokens hold X, 1, 1,
-X with X = 2^40 times 8: a sum in 32 bits loses the ones.  The two large terms
go through the same operations and differ in sign alone, so in 64 bits they
leave exactly the small ones.

Tolerance, u = 2^-24: a small term takes s and 1 - s (4 u and 5 u of hardware
sigmoid at 0), h = 32 s(32) (4 u) and four products, and the sum is rounded
once: 18 u of the result.
"""
import pytest
import torch

from _parity import dev, log

U = 2.0 ** -24
X = 2.0 ** 40


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,T,d", [(1, 8, 16), (2, 128, 80), (3, 264, 48), (1, 4096, 16)])
def test_terms_that_cancel(B, T, d, dt):
    import paper_2406_02528_amd as mmf
    log(f"[dlb] B={B} T={T} d={d} do={dt}")
    z = torch.zeros((B, T, 3, d), device=dev())
    z[:, :, 0] = -200.0
    z[:, 0::2, 1] = 32.0
    z[:, :, 2] = 1.0
    do = torch.zeros((B, T, d), device=dev())
    for i, v in ((1, X), (3, 1.0), (5, 1.0), (7, -X)):
        do[:, i::8] = v
    z, do = z.reshape(B * T, 3 * d).contiguous(), do.reshape(B * T, d).to(dt)
    o, dz = torch.empty((B * T, d), device=dev()), torch.empty((B * T, 3 * d), dtype=torch.bfloat16, device=dev())
    dlb = torch.full((d,), float("nan"), device=dev())
    states = torch.empty(mmf.mmf_mlgru_train_states_bytes(B, T, d), dtype=torch.uint8, device=dev())
    mmf.mmf_mlgru_train_scan(z, B, T, None, None, o, None, states)
    mmf.mmf_mlgru_scan_bwd(z, B, T, None, states, do, None, dz, None, dlb)
    want = B * (T // 8) * 2 * 8.0
    assert ((dlb.double() - want).abs() <= 18 * U * want).all(), dlb[:4]
