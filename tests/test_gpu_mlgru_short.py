"""Large batches of short sequences (one chunk of tokens each), whose arrays
pass the caches as streams: each sequence as in a call of its own, which goes
through them, bit for bit."""
import pytest
import torch

from _parity import dev, log

BF, F32 = torch.bfloat16, torch.float32


def run(mmf, v, B, T):
    d = v["do"].shape[1]
    whole = [torch.full((B * T + 2, n), 55, dtype=t, device=dev()) for n, t in ((d, F32), (3 * d, BF))]
    o, dz = (w[1:B * T + 1] for w in whole)
    h, dh0, dlb = (torch.full(s, float("nan"), device=dev()) for s in ((B, d), (B, d), (d,)))
    states = torch.empty(mmf.mmf_mlgru_train_states_bytes(B, T, d), dtype=torch.uint8, device=dev())
    mmf.mmf_mlgru_train_scan(v["z"], B, T, v["lb"], v["h0"], o, h, states)
    mmf.mmf_mlgru_scan_bwd(v["z"], B, T, v["lb"], states, v["do"], v["dh"], dz, dh0, dlb)
    torch.cuda.synchronize()
    assert all((w[0] == 55).all() and (w[-1] == 55).all() for w in whole)
    assert not dlb.isnan().any()
    return o, h, dz, dh0


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,T,d", [(260, 128, 528), (600, 37, 1040), (8200, 1, 2064)])
def test_sequences_of_one_chunk(B, T, d, dt):
    import paper_2406_02528_amd as mmf
    log(f"[mlgru_train] B={B} T={T} d={d} do={dt}")
    assert B * T * d * 16 > 256 << 20
    g = torch.Generator(device="cuda").manual_seed(B + T)
    rand = lambda *s: torch.randn(s, generator=g, device=dev())  # noqa: E731
    v = {"z": rand(B * T, 3 * d), "lb": torch.rand(d, generator=g, device=dev()) * 0.9, "h0": rand(B, d),
         "do": rand(B * T, d).to(dt), "dh": rand(B, d)}
    o, h, dz, dh0 = run(mmf, v, B, T)
    for b in (0, 1, B // 2, B - 1):
        s, r = slice(b * T, (b + 1) * T), slice(b, b + 1)
        one = run(mmf, {"z": v["z"][s], "lb": v["lb"], "h0": v["h0"][r], "do": v["do"][s], "dh": v["dh"][r]}, 1, T)
        assert all(torch.equal(x, y) for x, y in zip((o[s], h[r], dz[s], dh0[r]), one))
