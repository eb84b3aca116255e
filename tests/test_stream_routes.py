"""Which form of the recurrence's kernels a call takes at and below the size from
which arrays pass the caches as streams (host side only: tests/record.py
records the launches of the built library)."""
import pytest

from record import call, record

A = 0x100000000  # made-up 256-byte aligned device address, never dereferenced
BIG = 1 << 60


def forms(B, T, d):
    """(many chunks, streams) of the forward and of the backward from a bf16 and an fp32 gradient."""
    calls = [call("mmf_mlgru_train_scan", A, A, A, A, A, A, BIG, B, T, d, A, BIG, None)]
    calls += [call("mmf_mlgru_scan_bwd", A, A, A, BIG, A, f32, A, A, A, None, B, T, d, A, BIG, None) for f32 in (0, 1)]
    out = []
    for r in record(calls):
        assert r["status"] == 0
        (name,) = [l["kernel"] for l in r["launches"] if "clear" not in l["kernel"]]
        out.append(tuple(a.strip() == "true" for a in name[:-1].split("<")[1].split(",")[-2:]))
    return out


# sequences of one chunk of 128 tokens, of fewer tokens, and of several chunks
@pytest.mark.parametrize("T", [1, 100, 128, 129, 2048])
def test_streams_from_the_last_level_cache_on(T):
    d, llc = 2048, 256 << 20
    many = T > 128
    for i, per in enumerate((16, 20, 22)):  # bytes per token and channel
        most = (llc - 1) // (per * T * d)   # sequences that stay below it
        assert forms(most, T, d)[i] == (many, False)
        assert forms(most + 1, T, d)[i] == (many, True)
