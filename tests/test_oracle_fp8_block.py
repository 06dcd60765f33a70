"""The block-scaled E4M3 oracle against what the format is (CPU only), and the refusals of the calls."""
import numpy as np
import pytest
import torch

import paper_2504_14960_amd as moe
from oracle import fp8_block as fb


def test_values_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(fb.VALUES, codes.view(torch.float8_e4m3fn).double().numpy())
    np.testing.assert_array_equal(fb.scale_value(codes.numpy()), codes.view(torch.float8_e8m0fnu).double().numpy())


def test_codes_are_torchs_roundings():
    x = torch.from_numpy(np.random.default_rng(0).normal(size=4096) * np.exp2(np.linspace(-12, 7, 4096))).float().clamp(-448, 448)
    np.testing.assert_array_equal(fb.codes_of(fb.to_e4m3(x.double().numpy())), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("top,byte", [(448.0, 127), (448.0 * (1 + 2.0 ** -23), 128), (449.0, 128), (224.0, 126), (0.0, 1), (1e-45, 1),
                                      (448 * 2.0 ** -126, 1), (448 * 2.0 ** -125, 2), (3.4028234663852886e38, 247), (np.inf, 255), (np.nan, 255)])
def test_scale_is_the_smallest_that_leaves_448(top, byte):
    assert fb.scale_bytes(np.float64(top)) == byte
    if byte not in (1, 255):
        assert top / fb.scale_value(np.uint8(byte)) <= 448 < top / fb.scale_value(np.uint8(byte - 1))


def test_scale_stride():
    assert [moe.fp8_block_scale_stride(c) for c in (128, 256, 512, 640, 1408, 4096)] == [4, 4, 4, 8, 12, 32]
    assert all(moe.fp8_block_scale_stride(c) == fb.stride(c) for c in range(128, 20000, 128))
    assert moe.fp8_block_scale_stride(0) == moe.fp8_block_scale_stride(-128) == 0


# ---- refusals: nothing is launched ----
P = 4096


@pytest.mark.parametrize("args,status", [
    ((P, 2, 4, 128, P, P), 1), ((P, 1, -1, 128, P, P), 1), ((P, 1, 4, 0, P, P), 1), ((P, 1, 4, 96, P, P), 2), ((P, 1, 4, 1 << 23, P, P), 2),
    ((None, 1, 4, 128, P, P), 1),
    ((P + 8, 1, 4, 128, P, P), 1), ((P, 1, 4, 128, None, P), 1), ((P, 1, 4, 128, P + 4, P), 1), ((P, 1, 4, 128, P, None), 1),
    ((P, 1, 4, 128, P, P + 2), 1), ((None, 1, 0, 128, None, None), 0),
])
def test_quantize_refusals(args, status):
    assert moe.lib().moe_fp8_block_quantize(*args, None) == status


def _weights(**kw):
    a = dict(wg=P, wu=P, wd=P, dt=1, H=128, F=256, E=4, g=P, gs=P, u=P, us=P, d=P, ds=P, t=P, ts=P, dt_=P, dts=P)
    a.update(kw)
    return moe.lib().moe_expert_weights_fp8_block(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=5), 1), (dict(H=0), 1), (dict(E=0), 1), (dict(E=257), 2), (dict(H=192), 2), (dict(F=130), 2), (dict(H=1 << 23), 2),
    (dict(F=1 << 22), 2), (dict(wg=None), 1), (dict(wu=P + 2), 1), (dict(g=None), 1), (dict(gs=None), 1), (dict(ds=P + 1), 1),
    (dict(t=None), 1), (dict(dts=None), 1),
    (dict(g=None, gs=None, u=None, us=None, d=None, ds=None, t=None, ts=None, dt_=None, dts=None), 1),
])
def test_weights_refusals(kw, status):
    assert _weights(**kw) == status


def _permute(**kw):
    a = dict(x=P, idx=P, T=4, H=256, E=8, K=2, cap=0, c=P, s=P, n=P, off=P, roa=P, aor=P, ws=P, bytes=1 << 20)
    a.update(kw)
    return moe.lib().moe_permute_fp8_block(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(H=64), 2), (dict(H=136), 2), (dict(H=1 << 23), 2), (dict(T=-1), 1), (dict(K=9), 1), (dict(E=300), 2), (dict(x=None), 1), (dict(c=None), 1),
    (dict(s=None), 1), (dict(s=P + 2), 1), (dict(idx=None), 1), (dict(roa=None), 1), (dict(aor=None), 1), (dict(n=None), 1),
    (dict(off=None), 1), (dict(ws=None), 3), (dict(bytes=8), 3),
])
def test_permute_refusals(kw, status):
    assert _permute(**kw) == status


def _ffn(**kw):
    a = dict(x=P, xs=P, off=P, R=4, H=256, F=128, E=4, g=P, gs=P, u=P, us=P, d=P, ds=P, h=P, hs=P, gu=None, y=P)
    a.update(kw)
    return moe.lib().moe_grouped_gemm_swiglu_fp8_block(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(R=-1), 1), (dict(H=0), 1), (dict(E=257), 2), (dict(H=100), 2), (dict(F=200), 2), (dict(x=None), 1), (dict(xs=None), 1),
    (dict(xs=P + 1), 1), (dict(off=None), 1), (dict(g=None), 1), (dict(us=None), 1), (dict(d=None), 1), (dict(ds=None), 1),
    (dict(h=None), 1), (dict(hs=None), 1), (dict(gu=P + 2), 1), (dict(y=None), 1), (dict(R=0, x=None, y=None), 0),
])
def test_ffn_refusals(kw, status):
    assert _ffn(**kw) == status


def _backward(**kw):
    a = dict(x=P, xs=P, h=P, hs=P, gu=P, dy=P, off=P, R=4, H=256, F=128, E=4, t=P, ts=P, d=P, ds=P, dx=P, dg=P, du=P, dd=P, ws=P,
             bytes=1 << 30)
    a.update(kw)
    return moe.lib().moe_grouped_gemm_swiglu_fp8_block_backward(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(R=-1), 1), (dict(E=0), 1), (dict(H=64), 2), (dict(x=None), 1), (dict(xs=None), 1), (dict(h=None), 1), (dict(hs=P + 3), 1),
    (dict(gu=None), 1), (dict(dy=None), 1), (dict(off=None), 1), (dict(t=None), 1), (dict(ts=None), 1), (dict(d=None), 1),
    (dict(ds=None), 1), (dict(dx=None), 1), (dict(dg=None), 1), (dict(du=None), 1), (dict(dd=P + 8), 1), (dict(ws=None), 3),
    (dict(bytes=100), 3), (dict(R=(1 << 22) + 1, bytes=1 << 50), 2),
])
def test_backward_refusals(kw, status):
    assert _backward(**kw) == status


def test_backward_workspace():
    size = moe.expert_backward_fp8_block_workspace_bytes
    assert size(-1, 128, 128, 4) == size(8, 0, 128, 4) == size(8, 128, -1, 4) == size(8, 128, 128, 0) == 0
    assert size(1000, 1024, 512, 8) >= 1000 * (1024 + 6 * 512)


def test_binding_refuses_other_types_and_sizes():
    c, s = torch.empty((4, 256), dtype=torch.uint8), torch.empty((4, 4), dtype=torch.uint8)
    with pytest.raises(ValueError):
        moe.fp8_block_quantize(torch.zeros((4, 256)), c[:, :128], s)
    with pytest.raises(TypeError):
        moe.fp8_block_quantize(torch.zeros((4, 256)), c.to(torch.int32), s)
    with pytest.raises(ValueError):
        moe.fp8_block_quantize(torch.zeros((4, 256)), c, s[:, :2])
    with pytest.raises(ValueError):       # not on the device
        moe.fp8_block_quantize(torch.zeros((4, 256)), c, s)
