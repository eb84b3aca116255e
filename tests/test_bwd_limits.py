"""The backward's host side at the ends of its range of widths (no GPU: the
calls return before anything is enqueued)."""
import paper_2406_02528_amd as mmf

A, S = 0x100000, None


def test_no_out_features_is_a_noop():
    lib = mmf._lib
    for M in (0, 4, 300):
        assert lib.mmf_bitlinear_bwd(None, None, 0, None, None, None, None, None, None, None, None, None, None, M, 16,
                                     0, None, 0, S) == 0
        lib.mmf_bitlinear_bwd_workspace_bytes(M, 16, 0)


def test_rows_too_long_for_a_part_of_the_tokens_are_refused():
    """dO rows of which 129 pass 2^31 bytes: no split of dW's token range
    reaches them with 32-bit offsets."""
    lib = mmf._lib
    for N in ((1 << 23) - 8, (1 << 31) // 258 + 8):
        assert lib.mmf_bitlinear_bwd_workspace_bytes(300, 16, N) == 0
        assert lib.mmf_bitlinear_bwd(A, A, 0, None, A, A, A, A, A, A, A, None, None, 300, 16, N, None, 0, S) == 2
    assert lib.mmf_bitlinear_bwd_workspace_bytes(300, 16, (1 << 31) // 258 - 8) > 0
