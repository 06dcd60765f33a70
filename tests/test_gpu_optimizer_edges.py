"""Gradient norm and AdamW at the edges: numbers that fp32 cannot hold, arguments of other types, lists that one launch does not
hold.  Tolerances are those of test_gpu_optimizer, which derives them."""
import numpy as np
import pytest

from oracle import training as o
from test_gpu_optimizer import ADAM_EPS, B1, B2, EPS, LR, Tensors, _bf16, _dev


def _row(**kw):
    from paper_2504_14960_amd.binding import _AdamWTensor
    return (_AdamWTensor * 1)(_AdamWTensor(**{**dict(
        param=0x1000, master=0, grad=0x2000, exp_avg=0x3000, exp_avg_sq=0x4000, exp_avg_scale=0, exp_avg_sq_scale=0, n=100,
        weight_decay=0.0, lr_scale=1.0, param_dt=0, grad_dt=0, state=0), **kw}))


def test_an_eps_that_fp32_does_not_hold_is_refused():
    """Rounded to 0, or taken as 0 by a reciprocal, it would leave 0 / 0 where a gradient has always been 0."""
    import paper_2504_14960_amd as moe
    L = moe.lib()
    for eps in (5e-324, 1e-300, 1e-46, 1e-45, 1e-39, 1.17e-38, 1e39, 1e300):
        assert L.moe_adamw_step(_row(), 1, 1e-3, 0.9, 0.99, eps, 1, 0, None, None) == 1 and b"eps" in L.moe_last_error(), eps
    for eps in (2.0 ** -126, 1e-8, 1.0, 3e38):
        assert L.moe_adamw_step(_row(), 0, 1e-3, 0.9, 0.99, eps, 1, 0, None, None) == 0, eps


@pytest.mark.gpu
@pytest.mark.parametrize("param", ["f32", "master", "bf16"])
@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_weights_without_gradients_at_the_smallest_eps(param, state):
    import torch
    import paper_2504_14960_amd as moe
    t = Tensors([1000, 33], [(param, "f32", state)] * 2, fresh=True)
    for d in t.dev:
        d["g"].zero_()
    before = [{k: x.clone() for k, x in d.items() if x is not None} for d in t.dev]
    for step in (1, 2):
        moe.adamw_step(t.list, 0.0, B1, B2, 2.0 ** -126, step, seed=step)
        moe.adamw_step(moe.AdamWTensors([d["p"] for d in t.dev], [d["g"] for d in t.dev], [d["m"] for d in t.dev],
                                        [d["v"] for d in t.dev], masters=[d["master"] for d in t.dev],
                                        exp_avg_scales=[d["ms"] for d in t.dev], exp_avg_sq_scales=[d["vs"] for d in t.dev]),
                       LR, B1, B2, 2.0 ** -126, step, seed=step)
    torch.cuda.synchronize()
    for a, d in zip(before, t.dev):
        for k in ("p", "master"):
            assert k not in a or torch.equal(a[k], d[k]), k


def test_rates_that_fp32_does_not_hold_are_refused():
    """An infinite rate times a moment of 0 would be NaN."""
    import paper_2504_14960_amd as moe
    L = moe.lib()
    for lr, kw in ((1e39, {}), (1e300, dict(lr_scale=1e30)), (1e10, dict(lr_scale=1e30)), (1e30, dict(weight_decay=1e30)),
                   (1e38, {})):
        assert L.moe_adamw_step(_row(**kw), 1, lr, 0.9, 0.99, 1e-8, 1, 0, None, None) == 1, (lr, kw)
        assert b"lr" in L.moe_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("kind,count", [(("f32", "f32", "f32"), 145), (("f32", "bf16", "f32"), 71), (("master", "bf16", "f32"), 125),
                                        (("master", "f32", "f32"), 61), (("bf16", "bf16", "f32"), 150), (("bf16", "f32", "f32"), 141),
                                        (("f32", "f32", "8bit"), 110), (("master", "bf16", "8bit"), 95), (("bf16", "bf16", "8bit"), 107)],
                         ids=lambda x: "-".join(x) if isinstance(x, tuple) else str(x))
def test_one_kind_of_tensors_in_several_launches(kind, count):
    """Lists of one kind past what a launch holds (70 tensors of fp32 states without masters, 60 with, 52 and 46 of 8-bit ones):
    the limits on tensors and on words, a place in the list that goes on behind a launch."""
    rng = np.random.default_rng(count)
    sizes = [int(n) for n in rng.integers(0, 2500, count)]
    t = Tensors(sizes, [kind] * count, seed=count)
    t.step(3, 99)
    t.check(3, 99)


@pytest.mark.gpu
@pytest.mark.parametrize("dtypes", [["f32"], ["bf16"], ["bf16", "f32", "f32"]], ids="-".join)
def test_norm_of_lists_of_more_runs_than_workgroups(dtypes):
    """A workgroup goes from one tensor to the next, over several of one run, over some of none, and over types."""
    import torch
    import paper_2504_14960_amd as moe
    rng = np.random.default_rng(len(dtypes))
    sizes = [300_001, 0, 1, 5000, 0, 0, 900_000, 31, 4096, 8192, 1_200_003] * 7 + [2_000_000]
    kinds = [dtypes[i % len(dtypes)] for i in range(len(sizes))]
    runs = sum(-(-n * (2 if k == "bf16" else 4) // 16384) for n, k in zip(sizes, kinds))
    assert runs > 1024
    # every tensor adds about as much as the others: one left out, taken twice or read as the other type would show
    g = [(rng.standard_normal(n) * (2000.0 / max(n, 1)) ** 0.5).astype(np.float32) for n in sizes]
    g = [_bf16(x) if k == "bf16" else x for x, k in zip(g, kinds)]
    out = torch.zeros(2, device="cuda")
    ws = torch.full((moe.grad_norm_workspace_bytes(len(sizes)),), 0xff, dtype=torch.uint8, device="cuda")
    moe.grad_norm(moe.GradTensors([_dev(x, k == "bf16") for x, k in zip(g, kinds)]), out, ws, max_norm=1.0)
    np.testing.assert_allclose(out.cpu().numpy(), o.grad_norm(g, 1.0), rtol=4 * EPS)


@pytest.mark.gpu
def test_states_in_the_types_they_are_read_as():
    """float8_e4m3fn states and float8_e8m0fnu scales are the same bytes as uint8 ones."""
    import torch
    import paper_2504_14960_amd as moe
    a, b = (Tensors([1000, 33], [("bf16", "bf16", "8bit")] * 2, seed=3) for _ in range(2))
    as_type = lambda k, t: [d[k].view(t) for d in b.dev]  # noqa: E731
    e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    typed = moe.AdamWTensors([d["p"] for d in b.dev], [d["g"] for d in b.dev], as_type("m", e4m3), as_type("v", e4m3),
                             exp_avg_scales=as_type("ms", e8m0), exp_avg_sq_scales=as_type("vs", e8m0), weight_decays=b.decays,
                             lr_scales=b.lr_scales)
    a.step(5, 17)
    moe.adamw_step(typed, LR, B1, B2, ADAM_EPS, 5, seed=17)
    for x, y in zip(a.dev, b.dev):
        for k in ("p", "m", "v", "ms", "vs"):
            assert torch.equal(x[k], y[k]), k


def test_types_of_states_are_checked():
    import torch
    import paper_2504_14960_amd as moe
    x, s = torch.zeros(64), torch.zeros(2, dtype=torch.uint8)
    small, scale = x.to(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu)
    with pytest.raises(ValueError, match="device tensors"):          # the types are right, the place is not
        moe.AdamWTensors([x], [x], [small], [small], exp_avg_scales=[scale], exp_avg_sq_scales=[s])
    with pytest.raises(ValueError, match="need exp_avg_scales"):
        moe.AdamWTensors([x], [x], [small], [small])
    with pytest.raises(TypeError, match="exp_avg must be .*float8_e4m3fn"):
        moe.AdamWTensors([x], [x], [x.to(torch.float8_e5m2)], [small], exp_avg_scales=[scale], exp_avg_sq_scales=[scale])
    with pytest.raises(TypeError, match="exp_avg_sq must be"):
        moe.AdamWTensors([x], [x], [small], [x], exp_avg_scales=[scale], exp_avg_sq_scales=[scale])
    with pytest.raises(TypeError, match="exp_avg_sq_scale must be"):
        moe.AdamWTensors([x], [x], [small], [small], exp_avg_scales=[scale], exp_avg_sq_scales=[torch.ones(2)])


def test_a_step_takes_adamw_tensors_only():
    """The rows of a list of gradients are shorter than those of a step."""
    import paper_2504_14960_amd as moe
    for wrong in (moe.GradTensors([]), [], None):
        with pytest.raises(TypeError, match="AdamWTensors"):
            moe.adamw_step(wrong, LR, B1, B2, ADAM_EPS, 1)
    import torch
    with pytest.raises(TypeError, match="GradTensors"):
        moe.grad_norm([], torch.zeros(2), torch.zeros(8, dtype=torch.uint8))


def test_streams_without_the_short_way(monkeypatch):
    """torch's own short way to the stream's handle is not public: where it is missing, the public one is taken."""
    import torch
    from paper_2504_14960_amd import binding

    class Stream:
        cuda_stream = 1234

    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream())
    assert binding._stream() == 1234
