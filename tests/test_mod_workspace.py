"""The workspace of a backward call with a position bias, by the formula that the header states: no GPU."""
import pytest

from paper_2604_27124_amd import binding as A


def stated(B, L_q, L_k, H, reach):
    rows, keys = -(-L_q // 32), -(-L_k // 64)
    E = 32 * (min((2 * reach + 62) // 32 + 2, rows + 2 * keys) + 2)
    return 4 * B * H * (rows + 1) * E


@pytest.mark.parametrize("B,L_q,L_k,H,d,reach", [
    (2, 256, 256, 2, 64, 128), (4, 8192, 8192, 12, 64, 256), (4, 8192, 8192, 12, 64, 1024), (4, 8192, 8192, 12, 64, 8192), (1, 65536, 65536, 16, 64, 65536),
    (6, 513, 3001, 4, 128, 1000), (1, 1, 1, 1, 64, 0), (3, 33, 5000, 2, 128, 1 << 24), (256, 512, 512, 12, 64, 128)])
def test_workspace_is_what_the_header_says(B, L_q, L_k, H, d, reach):
    assert A.sigmoid_attn_rel_bwd_workspace_bytes(B, L_q, L_k, H, d, reach) == stated(B, L_q, L_k, H, reach)


def test_it_grows_with_both_lengths_at_a_large_reach():
    size = lambda L: A.sigmoid_attn_rel_bwd_workspace_bytes(1, L, L, 16, 64, L)
    assert 3.9 < size(65536) / size(32768) < 4.1 and 15 * 2 ** 30 < size(65536) < 17 * 2 ** 30
    near = lambda L: A.sigmoid_attn_rel_bwd_workspace_bytes(1, L, L, 16, 64, 128)
    assert 1.9 < near(65536) / near(32768) < 2.1
