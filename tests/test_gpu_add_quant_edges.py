"""The residual addition + quantisation at the edges of its contract."""
import pytest
import torch

from _parity import dev, log

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def mmf():
    import paper_2406_02528_amd as m
    return m


def bits(t):
    return t.view(torch.int16 if t.dtype == BF else torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True], ids=["out", "in_place"])
@pytest.mark.parametrize("xt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 2048), (70, 2064), (66, 8208), (2, 32784)])
def test_without_a_branch_the_stream_is_copied_bit_for_bit(mmf, M, K, xt, in_place):
    """s = x, zeros of either sign, subnormal and infinite values among them
    (the branch's type does not matter: there is none)."""
    log(f"[add_quant] copy M={M} K={K} x={xt} in_place={in_place}")
    gen = torch.Generator(device="cuda").manual_seed(M + K)
    x = torch.randn((M, K), generator=gen, device=dev()).to(xt)
    x[:, ::3] = -0.0
    x[:, 1::7] = 0.0
    x[:, 2::11] = -torch.finfo(xt).tiny / 4
    x[-1, 5] = -float("inf")
    want = x.clone()
    s = x if in_place else torch.full_like(x, 9.0)
    q, a = torch.empty((M, K), dtype=torch.int8, device=dev()), torch.empty(M, device=dev())
    for f32 in (0, 1):
        st = mmf._lib.mmf_add_act_quant(x.data_ptr(), xt == F32, None, f32, None, s.data_ptr(), q.data_ptr(),
                                        a.data_ptr(), None, None, M, K, torch.cuda.current_stream().cuda_stream)
        assert st == 0
        assert torch.equal(bits(s), bits(want))


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("K", [16, 512, 2048, 2064, 8208, 32784])
def test_rows_that_are_not_finite(mmf, K, xt):
    """A NaN or an infinity stays in s and shows in rstd; q and a_scale are
    finite, those that mmf_act_quant_ex gives for s; other rows do not notice."""
    M = 7
    log(f"[add_quant] not finite M={M} K={K} x={xt}")
    gen = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn((M, K), generator=gen, device=dev()).to(xt)
    b = torch.randn((M, K), generator=gen, device=dev())
    gamma = torch.rand(K, generator=gen, device=dev()) + 0.5
    clean = mmf.add_act_quant(x, b, gamma)
    nan, inf = float("nan"), float("inf")
    b[1, K // 2] = nan
    b[3, 3], b[3, K - 1] = inf, -inf
    b[5, 0], b[5, 9] = inf, nan
    x[6, 2], b[6, 2] = inf, -inf  # their sum is a NaN
    s, q, a, rs, r = mmf.add_act_quant(x, b, gamma)
    assert s[1, K // 2].isnan() and s[6, 2].isnan() and s[5, 9].isnan()
    assert s[3, 3] == inf and s[3, K - 1] == -inf and s[5, 0] == inf
    assert r[1].isnan() and r[5].isnan() and r[6].isnan() and r[3] == 0
    assert a.isfinite().all() and torch.equal(rs.long(), q.long().sum(1))
    q2, a2, rs2 = torch.empty_like(q), torch.empty_like(a), torch.empty_like(rs)
    mmf.mmf_act_quant_ex(s, gamma, q2, a2, rs2)
    assert torch.equal(q, q2) and torch.equal(a, a2) and torch.equal(rs, rs2)
    for i in (0, 2, 4):
        assert all(torch.equal(u[i], v[i]) for u, v in zip((s, q, a, rs, r), clean))
