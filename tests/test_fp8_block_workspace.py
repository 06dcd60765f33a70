"""Workspace sizes of block-scaled backwards that the call refuses are 0 (CPU only)."""
import pytest

import paper_2504_14960_amd as moe

LIMIT = 1 << 22


@pytest.mark.parametrize("R,H,F,E", [(8, 128, 128, 257), (8, 100, 128, 4), (8, 128, 200, 4), (LIMIT + 1, 128, 128, 4), (8, LIMIT + 128, 128, 4),
                                     (8, 128, LIMIT // 2 + 128, 4), ((1 << 31) - 1, 256, 128, 256)])
def test_none_for_calls_that_are_refused(R, H, F, E):
    assert moe.expert_backward_fp8_block_workspace_bytes(R, H, F, E) == 0
    call = moe.lib().moe_grouped_gemm_swiglu_fp8_block_backward
    assert call(*[4096] * 7, R, H, F, E, *[4096] * 9, 1 << 50, None) == 2


@pytest.mark.parametrize("R,H,F,E", [(0, 128, 128, 4), (8, 128, 128, 256), (LIMIT, 128, 128, 4), (8, LIMIT, 128, 4), (8, 128, LIMIT // 2, 4)])
def test_a_size_for_the_largest_calls(R, H, F, E):
    assert moe.expert_backward_fp8_block_workspace_bytes(R, H, F, E) >= R * (H + 6 * F) + 4 * (E + 1)
