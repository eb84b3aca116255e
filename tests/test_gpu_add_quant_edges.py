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
