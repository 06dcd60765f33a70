"""Weight gradients of the block-scaled backward where a scale is the smallest there is: what a code and its scale stand for is a bf16
value from a scale of 2^-124 on, and below that to within half of bf16's smallest step, 2^-133."""
import numpy as np
import pytest
import torch

import test_gpu_fp8_block as base
from oracle import fp8_block as fb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,H,F", [([40], 256, 128), ([70, 9], 256, 384)])
@pytest.mark.parametrize("scale", [1, 2, 3, 4])
def test_weight_gradients_of_the_smallest_scales(rows, H, F, scale):
    """Scale bytes 1 to 4: 2^-126 to 2^-123."""
    R = sum(rows)
    q, x, xs, offsets = base._layer(rows, H, F, 11)
    h, hs, gu, _ = base._forward(q, x, xs, offsets)
    rng = np.random.default_rng(scale)
    for codes, scales in ((x, xs), (h, hs)):
        c = rng.integers(0, 256, size=tuple(codes.shape)).astype(np.uint8)      # all codes, the smallest too, but NaN
        codes.copy_(torch.from_numpy(np.where((c & 127) == 127, 0, c)))
        scales.fill_(scale)
    dy = (base._values((R, H), 12) * 2.0 ** 60).to(torch.bfloat16).cuda()
    _, dw = base._backward(q, x, xs, h, hs, gu, dy, offsets)
    xv, hv, lo = fb.rows_value(base._np(x), base._np(xs)), fb.rows_value(base._np(h), base._np(hs)), 0
    lost = 0.0 if scale >= 3 else 2.0 ** -134
    for e, n in enumerate(rows):
        r = slice(lo, lo + n)
        lo += n
        dyv = base._np(dy)[r]
        want, off = base._product(dyv.T, hv[r].T, codes=False)
        off = off + lost * abs(dyv).sum(0)[:, None]
        assert (abs(base._np(dw[2])[e] - want) <= off + base.BF16 * (abs(want) + off)).all()
        # dg | du: as test_backward bounds them
        g, u = base._np(gu)[r, :F], base._np(gu)[r, F:]
        dh, eh = base._product(fb.rows_value(*fb.quantize_rows(dyv)), base._expert(q, "wd_t", e))
        s = fb.sigmoid(g)
        factor = (abs(u) * s * (1 + abs(g) * (1 - s)), abs(g) * s)
        near = (abs(u) * s * (1 + abs(g)), abs(g) * s)
        for k, d in enumerate((dh * u * s * (1 + g * (1 - s)), dh * g * s)):
            err = factor[k] * eh + near[k] * abs(dh) * (24 + 8 * abs(g)) * base.F32 + base.BF16 * abs(d)
            want, off = base._product(d.T, xv[r].T, codes=False)
            off = off + err.T @ abs(xv[r]) + lost * (abs(d) + err).sum(0)[:, None]
            assert (abs(base._np(dw[k])[e] - want) <= off + base.BF16 * (abs(want) + off)).all()
