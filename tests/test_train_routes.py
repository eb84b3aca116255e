"""The kernels that the training operators launch (host side only:
tests/record.py records the launches of the built library)."""
import pytest

from record import GEMM, call, kernels, record

A = 0x100000000  # made-up 256-byte aligned device address, never dereferenced
BIG = 1 << 60


def add(M, K, xf=0, bf=1):
    return call("mmf_add_act_quant", A, xf, A, bf, A, A, A, A, A, A, M, K, None)


def add_bwd(M, K, dgamma=A, ws=A):
    return call("mmf_add_act_quant_bwd", A, 1, A, A, 0, A, A, A, A, dgamma, M, K, ws, BIG if ws else 0, None)


def scan(B, T, d, ws=A):
    return call("mmf_mlgru_train_scan", A, A, A, A, A, A, BIG, B, T, d, ws, BIG if ws else 0, None)


def scan_bwd(B, T, d, dlb=A, ws=A):
    return call("mmf_mlgru_scan_bwd", A, A, A, BIG, A, 1, A, A, A, dlb, B, T, d, ws, BIG if ws else 0, None)


def test_very_many_rows_launch():
    """The most rows that the shapes allow stay inside the runtime's limits."""
    M = (1 << 31) - 1
    for r in record([add(M, 16), add(M, 2064), add(M, 1 << 20, 1, 0), add_bwd(M, 16), add_bwd(M, 1 << 20)]):
        assert r["status"] == 0 and r["launches"]


@pytest.mark.parametrize("K", [16, 2048, 2064, 8192, 8208, 32768, 32784, 1 << 20])
def test_addition_is_one_launch(K):
    for r in record([add(M, K, xf, bf) for M in (1, 64, 65, 5000) for xf in (0, 1) for bf in (0, 1)]):
        assert r["status"] == 0 and kernels(r) == ["add_quant_kernel"] and r["allocs"] == 0


def test_backward_without_dgamma_needs_no_scratch():
    a, b, c = record([add_bwd(300, 2048, None, None), add_bwd(300, 2048, A, None), add_bwd(300, 2048)])
    assert kernels(a) == ["add_quant_bwd_kernel"] and a["allocs"] == 0
    assert kernels(b) == ["add_quant_bwd_kernel", "col_final_kernel"] and (b["allocs"], b["frees"]) == (1, 1)
    assert kernels(c) == kernels(b) and c["allocs"] == 0


def test_recurrence_of_one_chunk_and_of_many():
    one, many, bone, bmany, bno = record([scan(3, 128, 2048, None), scan(1, 129, 2048), scan_bwd(3, 128, 2048, None, None),
                                          scan_bwd(1, 129, 2048), scan_bwd(1, 129, 2048, None)])
    assert kernels(one) == ["mlgru_train_fwd_kernel"] and one["allocs"] == 0
    assert kernels(many) == ["mlgru_train_clear_kernel", "mlgru_train_fwd_kernel"]
    assert kernels(bone) == ["mlgru_train_bwd_kernel"] and bone["allocs"] == 0
    assert kernels(bmany) == ["mlgru_train_clear_kernel", "mlgru_train_bwd_kernel", "col_final_kernel"]
    assert kernels(bno) == kernels(bmany)[:2]
    # a workgroup per 128 tokens and 64 channels
    assert many["launches"][1]["grid"] == [2 * 32, 1, 1] and many["launches"][1]["block"] == [512, 1, 1]


def test_recurrence_at_its_limits_launches():
    for r in record([scan(1, (1 << 22) * 128, 16), scan(1 << 22, 128, 16), scan_bwd(1, 1 << 15, 1 << 20),
                     scan_bwd(1 << 22, 1, 64)]):
        assert r["status"] == 0


def test_glu_backward_joins_its_stages():
    M, K, L = 1000, 2048, 5632
    (r,) = record([call("mmf_glu_bwd", A, 1, A, 0, A, A, A, A, A, A, A, A, A, A, M, K, L, A, BIG, None)])
    names = kernels(r)
    assert r["status"] == 0 and names[:2] == ["glu_pack_kernel", "gemm_kernel"]
    (b,) = record([call("mmf_bitlinear_bwd", A, A, 0, A, A, A, A, A, A, A, A, None, A, M, K, 2 * L, A, BIG, None)])
    assert names[2:] == kernels(b)


def test_gate_gradients_of_few_rows_split_k():
    """On the kernels that the forward's contraction takes."""
    for M, K, L in ((1, 2048, 5632), (16, 64, 2048), (17, 2048, 48), (64, 2048, 5632), (300, 2048, 5632),
                    (1000, 2048, 5632), (300, 512, 512)):
        for dp in (0, 1):
            fwd, bwd, tiled = record([
                call("mmf_ternary_gemm_glu", A, A, A, A, A, A, M, K, L, None),
                call("mmf_glu_gate_bwd", A, A, A, A, A, A, dp, A, M, K, L, None),
                call("mmf_glu_gate_bwd", A, A, A, A, A, A, dp, A, M, K, L, None, path=GEMM)])
            assert kernels(fwd) == kernels(bwd) and bwd["status"] == 0 and kernels(tiled) == ["gemm_kernel"]
            assert fwd["launches"][0]["grid"] == bwd["launches"][0]["grid"]


def test_failing_allocations_are_reported():
    for r in record([dict(c, fail=True) for c in (add_bwd(300, 2048, A, None), scan(1, 129, 64, None),
                                                  scan_bwd(1, 129, 64, A, None))]):
        assert r["status"] == 5 and not r["launches"]
