"""Gradient norm and AdamW against the float64 oracle: every combination of types, sizes around blocks and workgroups, lists
longer than one launch, states in 8 bits bit for bit.

Tolerances.  eps = 2^-24.  The moments are fp32 operations in a given order, each rounded: they are equal, bit for bit, to
the same operations in numpy, and so are the 8-bit codes made from them.  A new weight is within one rounding of p * decay
(eps |p|), of the update's factors (a square root, a product, a sum, a division, a product, constants rounded to fp32: 8 eps
of the update) and of the final difference (eps of the result)."""
import ctypes as C

import numpy as np
import pytest

from oracle import training as o

EPS = 2.0 ** -24
LR, B1, B2, ADAM_EPS, DECAY = 3e-3, 0.9, 0.999, 1e-8, 0.1
SIZES = [0, 1, 7, 8, 31, 32, 33, 63, 255, 256, 257, 2047, 2048, 2049, 5000, 70001]


def _bf16(x):
    """Nearest bf16 values of fp32 ones, as fp32."""
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def _dev(a, bf16=False):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.bfloat16() if bf16 else t


class Tensors:
    """A list of tensors on both sides; ``kinds``: (param, grad, state) of each."""

    def __init__(self, sizes, kinds, seed=0, fresh=False):
        import paper_2504_14960_amd as moe
        rng = np.random.default_rng(seed)
        self.host, self.dev, self.kinds = [], [], kinds
        for i, (n, (param, grad, state)) in enumerate(zip(sizes, kinds)):
            p = (rng.standard_normal(n) * 0.02).astype(np.float32)
            size = np.exp(rng.standard_normal(n) * 2).astype(np.float32)
            g = (rng.standard_normal(n) * 1e-3).astype(np.float32) * size
            m = (rng.standard_normal(n) * 3e-4).astype(np.float32) * size * (not fresh)
            v = np.square((rng.standard_normal(n) * 1e-3).astype(np.float32) * size) * np.float32(not fresh)
            p, g = _bf16(p) if param == "bf16" else p, _bf16(g) if grad == "bf16" else g
            h = dict(p=p, g=g, m=m, v=v)
            d = dict(g=_dev(g, grad == "bf16"), master=_dev(p) if param == "master" else None, p=_dev(p, param != "f32"),
                     m=_dev(m), v=_dev(v), ms=None, vs=None)
            if state == "8bit":
                u = rng.integers(0, 65536, n)
                for k in "mv":
                    codes, scales = o.mxfp8(h[k], u, k == "v")
                    h[k], h[k + "c"], h[k + "s"] = o.mxfp8_values(codes, scales).astype(np.float32), codes, scales
                    d[k], d[k + "s"] = _dev(codes), _dev(scales)
            self.host.append(h)
            self.dev.append(d)
        column = lambda k: [d[k] for d in self.dev]  # noqa: E731
        self.decays = [DECAY if i % 3 else 0.0 for i in range(len(sizes))]
        self.lr_scales = [1.0 if i % 2 else 0.5 for i in range(len(sizes))]
        self.list = moe.AdamWTensors(column("p"), column("g"), column("m"), column("v"), masters=column("master"),
                                     exp_avg_scales=column("ms"), exp_avg_sq_scales=column("vs"), weight_decays=self.decays,
                                     lr_scales=self.lr_scales)

    def step(self, step, seed, scale=None):
        import paper_2504_14960_amd as moe
        moe.adamw_step(self.list, LR, B1, B2, ADAM_EPS, step, seed=seed, grad_scale=scale)

    def check(self, step, seed, scale=1.0):
        """Compares one step taken from what ``host`` holds."""
        import torch
        torch.cuda.synchronize()
        for i, (h, d, (param, _, state)) in enumerate(zip(self.host, self.dev, self.kinds)):
            n = len(h["p"])
            where = f"tensor {i} of {n} elements, {self.kinds[i]}"
            g = h["g"] * np.float32(scale)
            m, v = o.moments32(g, h["m"], h["v"], B1, B2)
            bits = o.random_bits(seed, i, np.arange(n))
            if state == "8bit":
                for k, x, u in (("m", m, bits & np.uint32(0xffff)), ("v", v, bits >> np.uint32(16))):
                    codes, scales = o.mxfp8(x, u.astype(np.int64), k == "v")
                    np.testing.assert_array_equal(d[k + "s"].cpu().numpy(), scales, err_msg=where)
                    np.testing.assert_array_equal(d[k].cpu().numpy(), codes, err_msg=where)
            else:
                np.testing.assert_array_equal(d["m"].cpu().numpy(), m, err_msg=where)
                np.testing.assert_array_equal(d["v"].cpu().numpy(), v, err_msg=where)
            # from the moments as the interface rounds them: where beta1 m and (1 - beta1) g cancel, their roundings are far
            # more than eps of what is left
            p64 = o.adamw_weight(h["p"], m, v, LR * self.lr_scales[i], B1, B2, ADAM_EPS, step, self.decays[i])
            update = abs(p64 - h["p"] * (1 - LR * self.lr_scales[i] * self.decays[i]))
            tol = EPS * (2 * abs(h["p"]) + 10 * update + abs(p64)) + 1e-37
            got = d["p"].float().cpu().numpy() if d["master"] is None else d["master"].cpu().numpy()
            if param == "bf16":
                # the same bits round a larger value no lower; both ends may differ by some codes where p nearly vanishes
                ends = [(o.bf16_stochastic(p64 + d, bits).astype(np.uint32) << 16).view(np.float32) for d in (-tol, tol)]
                assert ((np.minimum(*ends) <= got) & (got <= np.maximum(*ends))).all(), where
            else:
                assert (abs(got - p64) <= tol).all(), (where, (abs(got - p64) / tol).max() if n else 0)
            if param == "master":
                np.testing.assert_array_equal(d["p"].float().cpu().numpy(), _bf16(got), err_msg=where)


ALL = [(p, g, s) for p in ("f32", "master", "bf16") for g in ("f32", "bf16") for s in ("f32", "8bit")]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ALL, ids="-".join)
def test_every_combination_of_types_over_many_sizes(kind):
    import torch
    t = Tensors(SIZES, [kind] * len(SIZES))
    scale = torch.tensor([0.37], device="cuda")
    t.step(7, 123, scale)
    t.check(7, 123, np.float32(0.37))


@pytest.mark.gpu
def test_lists_longer_than_a_launch_with_types_mixed():
    rng = np.random.default_rng(3)
    sizes = [int(n) for n in rng.integers(0, 3000, 131)]
    t = Tensors(sizes, [ALL[i % len(ALL)] for i in range(len(sizes))], seed=4)
    t.step(1, 0xffffffff)
    t.check(1, 0xffffffff)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [("f32", "f32", "f32"), ("bf16", "bf16", "8bit"), ("master", "bf16", "8bit")], ids="-".join)
def test_fresh_states(kind):
    """The first step from states of zeros: m / sqrt(v) is the sign of the gradient."""
    t = Tensors([1000, 33], [kind] * 2, fresh=True)
    t.step(1, 5)
    t.check(1, 5)


@pytest.mark.gpu
def test_zero_scales_are_fresh_states():
    import torch
    import paper_2504_14960_amd as moe
    g = torch.randn(100, device="cuda")
    p = torch.zeros(100, device="cuda")
    state = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (100, 100, 4, 4)]
    moe.adamw_step(moe.AdamWTensors([p], [g], [state[0]], [state[1]], exp_avg_scales=[state[2]], exp_avg_sq_scales=[state[3]]),
                   1e-2, B1, B2, ADAM_EPS, 1)
    assert torch.allclose(p, -1e-2 * g.sign(), rtol=1e-4)
    assert (state[1][g != 0] > 0).all()


@pytest.mark.gpu
def test_zero_gradients_and_zero_learning_rate():
    import torch
    import paper_2504_14960_amd as moe
    for dtype in (torch.float32, torch.bfloat16):
        p = torch.randn(500, device="cuda").to(dtype)
        keep, g = p.clone(), torch.zeros(500, device="cuda")
        m, v = torch.zeros(500, device="cuda"), torch.zeros(500, device="cuda")
        t = moe.AdamWTensors([p], [g], [m], [v], weight_decays=[0.1])
        moe.adamw_step(t, 0.0, B1, B2, ADAM_EPS, 1, seed=3)
        assert torch.equal(p, keep) and not m.any() and not v.any()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [("f32", "bf16", "f32"), ("master", "f32", "8bit"), ("bf16", "f32", "8bit")], ids="-".join)
def test_a_nan_scale_changes_nothing(kind):
    import torch
    t = Tensors([3000, 5], [kind] * 2)
    before = [{k: x.clone() for k, x in d.items() if x is not None} for d in t.dev]
    t.step(3, 1, torch.full((1,), float("nan"), device="cuda"))
    for a, d in zip(before, t.dev):
        for k, x in a.items():
            assert torch.equal(x, d[k]), k


@pytest.mark.gpu
def test_gradients_that_are_not_finite_stay_where_they_are():
    """fp32 states: their own elements.  8 bits: their blocks of 32, which then stand for NaN."""
    import torch
    for state in ("f32", "8bit"):
        t = Tensors([200], [("f32", "f32", state)])
        t.dev[0]["g"][40] = float("nan")
        t.dev[0]["g"][100] = float("inf")
        t.step(2, 9)
        p = t.dev[0]["p"].cpu().numpy()
        assert np.isnan(p[[40, 100]]).all() and np.isfinite(np.delete(p, [40, 100])).all()
        if state == "8bit":
            for k, ks in (("m", "ms"), ("v", "vs")):
                scales, codes = t.dev[0][ks].cpu().numpy(), t.dev[0][k].cpu().numpy()
                assert list(np.nonzero(scales == 255)[0]) == [1, 3] and (codes[32:64] == 0x7f).all()
            t.dev[0]["g"].zero_()
            t.step(3, 10)
            p = t.dev[0]["p"].cpu().numpy()
            assert np.isnan(p[32:64]).all() and np.isnan(p[96:128]).all() and np.isfinite(p[:32]).all()
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_extreme_values_in_8_bits():
    """The largest and the smallest fp32 numbers, blocks of one sign, of zeros, of one value."""
    import torch
    import paper_2504_14960_amd as moe
    rng = np.random.default_rng(6)
    g = (rng.standard_normal(32 * 40) * np.repeat(10.0 ** rng.uniform(-22, 18, 40), 32)).astype(np.float32)
    g[:32], g[32:64], g[64:96] = 0.0, -1.0, np.float32(1e-45)
    g[96:128] = np.where(np.arange(32) == 5, 1.0, 1e-12)
    n = len(g)
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(n // 32, dtype=torch.uint8, device="cuda"), torch.zeros(n // 32, dtype=torch.uint8, device="cuda")
    moe.adamw_step(moe.AdamWTensors([p], [_dev(g)], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs]), LR, B1, B2,
                   ADAM_EPS, 1, seed=77)
    m32, v32 = o.moments32(g, np.zeros(n), np.zeros(n), B1, B2)
    bits = o.random_bits(77, 0, np.arange(n))
    for got, scale, x, u, keep in ((m, ms, m32, bits & np.uint32(0xffff), False), (v, vs, v32, bits >> np.uint32(16), True)):
        codes, scales = o.mxfp8(x, u.astype(np.int64), keep)
        np.testing.assert_array_equal(scale.cpu().numpy(), scales)
        np.testing.assert_array_equal(got.cpu().numpy(), codes)
    assert np.isfinite(p.cpu().numpy()).all()


@pytest.mark.gpu
def test_8_bit_moments_follow_a_gradient_without_bias():
    """A thousand steps of beta2 = 0.999 towards a new level, over 4096 elements.  The true second moment reaches 1 - 0.999^1000
    of the gradient's square.  Rounding adds at most a step of 1/8 of the value a time, with probability under 0.001 * 8 of
    moving, so a relative variance under 1000 * 0.008 / 64 = 1/8 in an element and a standard error under 0.006 in the mean:
    3 % is five of them.  To the nearest, nothing would move once v is above 1/60 of its level."""
    import torch
    import paper_2504_14960_amd as moe
    n = 4096
    g = torch.full((n,), 1e-3, device="cuda")
    g[::2] = -1e-3
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(n // 32, dtype=torch.uint8, device="cuda"), torch.zeros(n // 32, dtype=torch.uint8, device="cuda")
    t = moe.AdamWTensors([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
    for step in range(1, 1001):
        moe.adamw_step(t, 0.0, B1, B2, ADAM_EPS, step, seed=step)
    got_v = o.mxfp8_values(v.cpu().numpy(), vs.cpu().numpy())
    got_m = o.mxfp8_values(m.cpu().numpy(), ms.cpu().numpy())
    assert abs(got_v.mean() / (1e-6 * (1 - B2 ** 1000)) - 1) < 0.03
    # m settles in a few steps; its rounding errors are a step of 1/8 at most, so the mean's is under 0.125 / 64
    assert abs((got_m * np.sign(g.cpu().numpy())).mean() / 1e-3 - 1) < 0.01


@pytest.mark.gpu
def test_bf16_weights_alone_follow_small_updates_without_bias():
    """A hundred steps of 1e-4 from 1: far below half the distance 2^-8 of bf16 values under 1.  The mean of 65536 weights has
    a standard error of about sqrt(100 * 1e-4 / 2^-8) 2^-8 / 256 = 2.4e-5; 2e-4 is eight of them."""
    import torch
    import paper_2504_14960_amd as moe
    n = 65536
    p = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g, m, v = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    t = moe.AdamWTensors([p], [g], [m], [v])
    for step in range(1, 101):
        moe.adamw_step(t, 1e-4, B1, B2, ADAM_EPS, step, seed=step)
    assert abs(float(p.double().mean()) - 0.99) < 2e-4


@pytest.mark.gpu
def test_a_tensor_of_more_than_2_to_the_32_elements():
    """Its last elements, whose offsets pass 32 bits, and those around element 2^32."""
    import torch
    import paper_2504_14960_amd as moe
    n = (1 << 32) + 4133
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    at = slice((1 << 32) - 4096, n)
    rng = np.random.default_rng(8)
    g_host = _bf16(rng.standard_normal(n - at.start).astype(np.float32))
    g[at] = _dev(g_host, True)
    out = torch.zeros(2, device="cuda")
    t = moe.AdamWTensors([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
    moe.grad_norm(t, out, torch.empty(moe.grad_norm_workspace_bytes(1), dtype=torch.uint8, device="cuda"))
    moe.adamw_step(t, LR, B1, B2, ADAM_EPS, 1, seed=5)
    torch.cuda.synchronize()
    assert abs(float(out[0]) / o.grad_norm([g_host])[0] - 1) < 4 * EPS
    m32, v32 = o.moments32(g_host, 0 * g_host, 0 * g_host, B1, B2)
    bits = o.random_bits(5, 0, np.arange(at.start, n, dtype=np.int64))
    blocks = slice(at.start // 32, None)
    for got, scale, x, u, keep in ((m, ms, m32, bits & np.uint32(0xffff), False), (v, vs, v32, bits >> np.uint32(16), True)):
        codes, scales = o.mxfp8(x, u.astype(np.int64), keep)
        np.testing.assert_array_equal(scale[blocks].cpu().numpy(), scales)
        np.testing.assert_array_equal(got[at].cpu().numpy(), codes)
    assert int(torch.count_nonzero(p[:1 << 31])) == 0
    moved = p[at].float().cpu().numpy()
    assert (np.sign(moved) == -np.sign(g_host)).all() and (abs(abs(moved) / LR - 1) < 2.0 ** -7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[1], [0, 0], [], [5, 0, 33], SIZES, [300_000], [17] * 200, [3_000_001, 9, 64]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grad_norm(sizes, dtype):
    import torch
    import paper_2504_14960_amd as moe
    rng = np.random.default_rng(len(sizes))
    g = [(rng.standard_normal(n) * 10.0 ** rng.uniform(-3, 1)).astype(np.float32) for n in sizes]
    g = [_bf16(x) for x in g] if dtype == "bf16" else g
    lists = moe.GradTensors([_dev(x, dtype == "bf16") for x in g])
    out = torch.full((2,), -7.0, device="cuda")
    ws = torch.full((moe.grad_norm_workspace_bytes(len(sizes)),), 0xff, dtype=torch.uint8, device="cuda")
    for max_norm, mult in ((0.0, 1.0), (1e-2, 0.25), (1e9, -2.0)):
        moe.grad_norm(lists, out, ws, max_norm=max_norm, multiplier=mult)
        want = o.grad_norm(g, np.float32(max_norm), mult)
        np.testing.assert_allclose(out.cpu().numpy(), want, rtol=4 * EPS, atol=1e-37)


@pytest.mark.gpu
def test_grad_norm_of_extreme_and_not_finite_gradients():
    import torch
    import paper_2504_14960_amd as moe
    out = torch.zeros(2, device="cuda")
    ws = torch.empty(moe.grad_norm_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    for value, norm in ((1e30, 1e30 * np.sqrt(5000)), (1e-30, 1e-30 * np.sqrt(5000)), (3e38, np.inf), (float("inf"), np.inf), (float("nan"), np.nan)):
        g = torch.full((5000,), value, device="cuda")
        moe.grad_norm(moe.GradTensors([g, g[:0]]), out, ws, max_norm=1.0)
        got = out.cpu().numpy()
        np.testing.assert_allclose(got[0], np.float32(norm), rtol=4 * EPS)
        assert np.isnan(got[1]) == (not np.isfinite(norm))


@pytest.mark.gpu
def test_same_inputs_same_bits_on_any_stream():
    import torch
    import paper_2504_14960_amd as moe
    kinds = [ALL[i % len(ALL)] for i in range(60)]
    a, b = (Tensors([1500 + 77 * i for i in range(60)], kinds, seed=2) for _ in range(2))
    ws = torch.empty(moe.grad_norm_workspace_bytes(60), dtype=torch.uint8, device="cuda")
    out = torch.zeros((2, 2), device="cuda")
    torch.cuda.synchronize()
    moe.grad_norm(a.list, out[0], ws, max_norm=0.1)
    a.step(4, 11, out[0, 1:])
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        moe.grad_norm(b.list, out[1], ws, max_norm=0.1)
        b.step(4, 11, out[1, 1:])
        torch.cuda.current_stream().synchronize()
    assert torch.equal(out[0], out[1]) and float(out[0, 1]) < 1
    for x, y in zip(a.dev, b.dev):
        for k in x:
            assert x[k] is None or torch.equal(x[k], y[k])


@pytest.mark.gpu
def test_norm_and_step_replayed_in_a_graph():
    """Each replay steps from what the last one left, with the step and seed it was captured with, as eager calls do."""
    import torch
    import paper_2504_14960_amd as moe
    kinds = [ALL[i % len(ALL)] for i in range(80)]
    eager, captured = (Tensors([700 + 31 * i for i in range(80)], kinds, seed=5) for _ in range(2))
    ws = torch.empty(moe.grad_norm_workspace_bytes(80), dtype=torch.uint8, device="cuda")
    out = torch.zeros((2, 2), device="cuda")

    def step(t, o):
        moe.grad_norm(t.list, o, ws, max_norm=0.1)
        t.step(4, 11, o[1:])

    step(eager, out[0])
    step(captured, out[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured, out[1])
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        step(eager, out[0])
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1])
        for x, y in zip(eager.dev, captured.dev):
            for k in x:
                assert x[k] is None or torch.equal(x[k], y[k])


def _refuse(fn, word, status=1):
    import paper_2504_14960_amd as moe
    L = moe.lib()
    assert fn() == status and word in L.moe_last_error(), L.moe_last_error()


def test_refusals():
    import paper_2504_14960_amd as moe
    from paper_2504_14960_amd.binding import _AdamWTensor, _GradTensor
    L = moe.lib()
    good = dict(param=0x1000, master=0, grad=0x2000, exp_avg=0x3000, exp_avg_sq=0x4000, exp_avg_scale=0, exp_avg_sq_scale=0,
                n=100, weight_decay=0.0, lr_scale=1.0, param_dt=0, grad_dt=0, state=0)

    def step(count=1, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, t=1, scale=None, tensors=True, **kw):
        row = (_AdamWTensor * 1)(_AdamWTensor(**{**good, **kw}))
        return L.moe_adamw_step(row if tensors else None, count, lr, b1, b2, eps, t, 0, scale, None)

    for kw, word in [(dict(count=-1), b"count"), (dict(tensors=False), b"NULL"), (dict(t=0), b"step"), (dict(lr=-1.0), b"lr"),
                     (dict(lr=float("nan")), b"lr"), (dict(b1=1.0), b"beta"), (dict(b2=-0.1), b"beta"), (dict(eps=0.0), b"eps"),
                     (dict(scale=C.c_void_p(0x1001)), b"grad_scale"), (dict(n=-1), b"n=-1"), (dict(param=0), b"param is NULL"),
                     (dict(grad=0x2002), b"aligned"), (dict(exp_avg=0), b"exp_avg"), (dict(exp_avg_sq=0x4008), b"aligned"),
                     (dict(master=0x5000), b"master"), (dict(param_dt=1, master=0x5004), b"aligned"),
                     (dict(param_dt=2), b"param_dt"), (dict(grad_dt=-1), b"grad_dt"), (dict(state=2), b"state"),
                     (dict(state=1), b"scales"), (dict(weight_decay=float("inf")), b"finite"), (dict(lr_scale=float("nan")), b"finite")]:
        _refuse(lambda: step(**kw), word)
    _refuse(lambda: step(n=1 << 40), b"limit", 2)
    _refuse(lambda: step(count=(1 << 26) + 1), b"limit", 2)
    assert step(count=0, tensors=False) == 0 and step(n=0, param=0, grad=0) == 0

    def norm(count=1, max_norm=1.0, mult=1.0, out=0x1000, ws=0x2000, size=1 << 20, grad=0x3000, n=10, dt=0):
        row = (_GradTensor * 1)(_GradTensor(grad, n, dt))
        return L.moe_grad_norm(row, count, max_norm, mult, C.c_void_p(out), C.c_void_p(ws), size, None)

    for kw, word in [(dict(count=-1), b"count"), (dict(max_norm=float("nan")), b"max_norm"), (dict(mult=float("inf")), b"finite"),
                     (dict(out=0), b"out"), (dict(out=0x1001), b"out"), (dict(grad=0), b"grad"), (dict(grad=0x3008), b"aligned"),
                     (dict(n=-3), b"n=-3"), (dict(dt=7), b"dt"), (dict(ws=0x2004), b"aligned")]:
        _refuse(lambda: norm(**kw), word)
    _refuse(lambda: norm(count=(1 << 26) + 1), b"limit", 2)
    _refuse(lambda: norm(size=8), b"workspace", 3)
    _refuse(lambda: norm(ws=0), b"workspace", 3)
    assert moe.grad_norm_workspace_bytes(0) > 0 and moe.grad_norm_workspace_bytes(-1) == 0


def test_lists_are_checked_when_they_are_built():
    import torch
    import paper_2504_14960_amd as moe
    x = torch.zeros(64)
    with pytest.raises(ValueError, match="device tensors"):
        moe.GradTensors([x])
    with pytest.raises(ValueError, match="as many entries"):
        moe.AdamWTensors([x], [x, x], [x], [x])
    with pytest.raises(ValueError, match="exp_avg must have 64"):
        moe.AdamWTensors([x], [x], [x[:3]], [x])
    with pytest.raises(TypeError, match="exp_avg_sq"):
        moe.AdamWTensors([x], [x], [x], [x.byte()])
    with pytest.raises(ValueError, match="need exp_avg_scales"):
        moe.AdamWTensors([x], [x], [x.byte()], [x.byte()])
    with pytest.raises(ValueError, match="8-bit states only"):
        moe.AdamWTensors([x], [x], [x], [x], exp_avg_scales=[x.byte()])
