"""How many waves of the residual addition + quantisation share a row (host side
only: tests/record.py records the launches of the built library)."""
import pytest

from record import call, record

A = 0x100000000  # made-up 256-byte aligned device address, never dereferenced


def waves(M, K, x_f32, b_f32):
    (r,) = record([call("mmf_add_act_quant", A, x_f32, A, b_f32, A, A, A, A, A, A, M, K, None)])
    (l,) = r["launches"]
    return int(l["kernel"].split("<")[1].split(",")[3])


@pytest.mark.parametrize("x_f32,b_f32", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_waves_per_row(x_f32, b_f32):
    two = 1024 if x_f32 == b_f32 == 0 else 512  # two vectors of eight or of four values per lane of a wave
    for M in (1, 64, 256):
        assert [waves(M, K, x_f32, b_f32) for K in (16, two, two + 16, 2048)] == [1, 1, 4, 4]
    for M in (257, 16384):
        assert [waves(M, K, x_f32, b_f32) for K in (16, two + 16, 2048)] == [1, 1, 1]
    for M in (1, 64, 256, 257, 16384):
        assert [waves(M, K, x_f32, b_f32) for K in (2064, 5120, 8192, 8208, 32784)] == [4, 4, 4, 16, 16]
