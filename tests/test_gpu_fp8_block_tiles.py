"""The block-scaled expert FFN where a workgroup has several output tiles one after the other, in every height of the tiles and at
every place of the four-tile word of scales; contractions of many blocks, layers of many experts, more rows than a tile where the
contraction is a single block; and its weight gradients in the tiles that layers of many rows take.  Each against the oracle, by
the same comparison as the smaller layers."""
import pytest

import paper_2504_14960_amd as moe
import test_gpu_fp8_block as base

pytestmark = pytest.mark.gpu


def _with_options(options, check):
    try:
        for name, value in options.items():
            moe.set_option(name, value)
        check()
    finally:
        for name in options:
            moe.set_option(name, -1 if name == "gemm_idle_skip" else 0)


# blocks along the contraction: gate/up and dh H / 128, down F / 128, dx 2F / 128, each of 2, 3, 4, 5 and 8 among them
LAYERS = [(256, 384), (384, 512), (512, 640), (640, 1024), (1024, 256)]
# a tile of one row, empty experts, and remainders on both sides of half a tile
UNEVEN = [300, 1, 0, 520, 64, 0, 129]


@pytest.mark.parametrize("workgroups,skip", [(8, 0), (13, 1)])
@pytest.mark.parametrize("height", [128, 192, 256])
@pytest.mark.parametrize("H,F", LAYERS)
def test_several_tiles_to_a_workgroup(H, F, height, workgroups, skip):
    options = dict(gemm_workgroups=workgroups, gemm_tile_rows=height, gemm_idle_skip=skip)
    _with_options(options, lambda: base.test_forward(UNEVEN, H, F))
    _with_options(options, lambda: base.test_backward(UNEVEN, H, F))


@pytest.mark.parametrize("rows,H,F,workgroups", [([300, 0, 1, 257, 640, 128, 129, 400, 250, 260, 90, 45], 1024, 1408, 0), ([513, 40, 700], 512, 384, 8),
                                                 ([0, 1000, 900], 384, 640, 13)])
def test_weight_gradients_in_large_tiles(rows, H, F, workgroups):
    _with_options(dict(gemm_workgroups=workgroups), lambda: base.test_backward(rows, H, F))


@pytest.mark.parametrize("rows,H,F", [([2] * 256, 256, 128), ([40, 0, 3, 1] * 64, 256, 256), ([70, 3], 8192, 256), ([5, 2], 256, 8192), ([200, 90], 256, 6144),
                                      ([70, 200, 64, 0, 129], 128, 128), ([65, 130], 128, 512)])
def test_many_experts_long_contractions_and_single_blocks(rows, H, F):
    base.test_forward(rows, H, F)
    base.test_backward(rows, H, F)
