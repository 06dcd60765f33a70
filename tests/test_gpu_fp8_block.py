"""The expert FFN in E4M3 with a scale for every block of 128 on the GPU against the oracle: codes and scales bit for bit, products
within their roundings."""
import numpy as np
import pytest
import torch

import paper_2504_14960_amd as moe
from oracle import fp8_block as fb

pytestmark = pytest.mark.gpu
BF16 = 2.0 ** -8      # half a step, relative
F32 = 2.0 ** -24


def _bytes(*shape, fill=0xa5):
    return torch.full(shape, fill, dtype=torch.uint8, device="cuda")


def _np(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _values(shape, seed, spread=1.0):
    """Values whose size differs from block to block."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=shape) * np.exp(spread * rng.normal(size=shape[:-1] + (shape[-1] // 128, 1))).repeat(128, -1).reshape(shape)
    return torch.from_numpy(x).float()


# ---- quantisation ----
@pytest.mark.parametrize("rows,C", [(1, 128), (3, 384), (64, 512), (65, 640), (7, 1408), (301, 2048), (2, 16384)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows(rows, C, dtype):
    x = _values((rows, C), rows + C, 3.0).to(dtype).cuda()
    codes, scales = _bytes(rows, C), _bytes(rows, fb.stride(C))
    moe.fp8_block_quantize(x, codes, scales)
    c, b = fb.quantize_rows(_np(x))
    np.testing.assert_array_equal(_np(codes), c)
    np.testing.assert_array_equal(_np(scales)[:, :C // 128], b)
    assert (_np(scales)[:, C // 128:] == 0xa5).all()          # what lies behind a row's scales is left alone


def test_rows_at_the_ends_of_the_range():
    x = torch.zeros((9, 256))
    x[0, :4] = torch.tensor([448.0, 449.0, -1e-30, 0.0])
    x[1, 200] = 3.4028234663852886e38
    x[2, 3] = float("inf")
    x[3, 3], x[3, 130] = float("nan"), 2.0
    x[4, 5] = -float("inf")
    x[5, :128] = torch.arange(128) * 2.0 ** -149              # denormal values
    x[6, :128] = 448 * 2.0 ** -126
    x[7, :128] = torch.linspace(-448, 448, 128)
    x[8] = -0.0
    codes, scales = _bytes(9, 256), _bytes(9, 4)
    moe.fp8_block_quantize(x.cuda(), codes, scales)
    c, b = fb.quantize_rows(x.double().numpy())
    np.testing.assert_array_equal(_np(codes), c)
    np.testing.assert_array_equal(_np(scales)[:, :2], b)
    assert b[2, 0] == b[3, 0] == b[4, 0] == 255 and b[3, 1] != 255 and (c[2, :128] == 0x7f).all()


def _quantized_weights(w, layout=True):
    E, F, H = w[0].shape
    f = dict(gate=(E, F, H), up=(E, F, H), down=(E, H, F))
    t = dict(wgu_t=(E, H, 2 * F), wd_t=(E, F, H))
    out = {}
    for k, (e, n, c) in {**f, **(t if layout else {})}.items():
        out[k], out[k + "_scales"] = _bytes(e, n, c), _bytes(e, n // 128, fb.stride(c))
    moe.expert_weights_fp8_block(*w, *out.values())
    return out


@pytest.mark.parametrize("E,H,F", [(1, 128, 128), (3, 256, 384), (2, 1408, 640), (5, 512, 1152)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weights_in_both_layouts(E, H, F, dtype):
    w = [(_values(s, i + E, 2.0) * 0.02).to(dtype).cuda() for i, s in enumerate(((E, F, H), (E, F, H), (E, H, F)))]
    w[0][0, 3, 5] = float("inf")
    got = {k: _np(v) for k, v in _quantized_weights(w).items()}
    for e in range(E):
        c, b = zip(*(fb.quantize_square(_np(t[e])) for t in w))
        for name, i in (("gate", 0), ("up", 1), ("down", 2)):
            np.testing.assert_array_equal(got[name][e], c[i])
            np.testing.assert_array_equal(got[name + "_scales"][e][:, :b[i].shape[1]], b[i])
            assert (got[name + "_scales"][e][:, b[i].shape[1]:] == 0xa5).all()
        np.testing.assert_array_equal(got["wgu_t"][e], np.concatenate([c[0].T, c[1].T], 1))
        np.testing.assert_array_equal(got["wd_t"][e], c[2].T)
        np.testing.assert_array_equal(got["wgu_t_scales"][e][:, :2 * F // 128], np.concatenate([b[0].T, b[1].T], 1))
        np.testing.assert_array_equal(got["wd_t_scales"][e][:, :H // 128], b[2].T)


def test_weights_in_one_layout_only():
    E, H, F = 2, 256, 128
    w = [_values(s, i).cuda() for i, s in enumerate(((E, F, H), (E, F, H), (E, H, F)))]
    both = _quantized_weights(w)
    only = _quantized_weights(w, layout=False)
    for k, v in only.items():
        assert torch.equal(v, both[k])
    t = {k: _bytes(*both[k].shape) for k in ("wgu_t", "wgu_t_scales", "wd_t", "wd_t_scales")}
    moe.expert_weights_fp8_block(*w, *[None] * 6, *t.values())
    for k, v in t.items():
        assert torch.equal(v, both[k])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weights_of_more_than_the_caches_hold(dtype):
    """151 MB of codes in one call against the two layouts in calls of their own."""
    E, H, F = 4, 4096, 1536
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = [(torch.randn(s, generator=gen, device="cuda") * 0.02).to(dtype) for s in ((E, F, H), (E, F, H), (E, H, F))]
    both = _quantized_weights(w)
    halves = _quantized_weights(w, layout=False)
    halves.update({k: _bytes(*both[k].shape) for k in ("wgu_t", "wgu_t_scales", "wd_t", "wd_t_scales")})
    moe.expert_weights_fp8_block(*w, *[None] * 6, *list(halves.values())[6:])
    for k, v in both.items():
        assert torch.equal(v, halves[k]), k


@pytest.mark.parametrize("T,H,E,K,capacity", [(1, 128, 8, 2, 0), (5, 384, 4, 4, 0), (64, 1408, 64, 8, 0), (777, 512, 12, 3, 150), (3000, 256, 8, 2, 0),
                                              (9000, 128, 64, 6, 700), (1500, 6144, 8, 2, 0), (300, 16384, 16, 1, 0), (20000, 256, 8, 2, 0),
                                              (1100, 8192, 64, 2, 0), (1030, 4096, 16, 1, 50), (5, 8192, 8, 3, 0)])
def test_permute_is_permute_and_quantisation(T, H, E, K, capacity):
    gen = torch.Generator().manual_seed(T)
    x = (torch.randn((T, H), generator=gen) * torch.exp(torch.randn((T, 1), generator=gen))).to(torch.bfloat16).cuda()
    idx = torch.rand((T, E), generator=gen).topk(K).indices.to(torch.int32).cuda()
    idx[0, 0] = -1                                            # a dropped assignment
    R = moe.max_rows(T, K, E, capacity)
    ws = torch.empty(moe.permute_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")

    def maps():
        return [torch.full((n,), -5, dtype=torch.int32, device="cuda") for n in (E, E + 1, T * K, R)]
    a, b = maps(), maps()
    xp = torch.zeros((R, H), dtype=torch.bfloat16, device="cuda")
    moe.permute(x, idx, E, capacity, xp, *a, ws)
    codes, scales = _bytes(R, H), _bytes(R, fb.stride(H))
    moe.permute_fp8_block(x, idx, E, capacity, codes, scales, *b, ws)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    n = int(a[1][-1])
    c, s = _bytes(R, H), _bytes(R, fb.stride(H))
    moe.fp8_block_quantize(xp[:n], c[:n], s[:n])
    assert torch.equal(codes, c) and torch.equal(scales, s)   # rows behind the last one too


# ---- products ----
def _layer(rows, H, F, seed, r_max=None, spread=1.0):
    """Quantised rows and weights of a layer, on the device and as the oracle's values."""
    E, R = len(rows), sum(rows)
    w = [(_values(s, seed + i, 0.5) / np.sqrt(s[2])).cuda() for i, s in enumerate(((E, F, H), (E, F, H), (E, H, F)))]
    q = _quantized_weights(w)
    n = R if r_max is None else r_max
    x, xs = _bytes(n, H), _bytes(n, fb.stride(H))
    moe.fp8_block_quantize(_values((n, H), seed + 9, spread).cuda(), x, xs)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
    return q, x, xs, offsets


def _expert(q, name, e):
    return fb.square_value(_np(q[name][e]), _np(q[name + "_scales"][e]))


def _forward(q, x, xs, offsets, save=True):
    E, F, H = q["gate"].shape
    R = len(x)
    h, hs = _bytes(R, F), _bytes(R, fb.stride(F))
    gu = torch.full((R, 2 * F), 7.0, dtype=torch.bfloat16, device="cuda") if save else None
    y = torch.full((R, H), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.grouped_gemm_swiglu_fp8_block(x, xs, offsets, q["gate"], q["gate_scales"], q["up"], q["up_scales"], q["down"], q["down_scales"],
                                      h, hs, gu, y)
    return h, hs, gu, y


def _product(a, b, codes=True):
    """a b^T and what it may be off.  fp32 accumulation: a rounding for every term, of what is added up.  Products of codes: the
    matrix instruction adds the products of eight neighbouring codes with what lies 2^13 below the largest of them cut off, so
    that each of the other seven loses less than 2^-13 of it: 7 * 2^-13 sum_g max_g |a b|, where max_g <= sqrt(sum_g (a b)^2), and the sum
    over the K / 8 groups is at most sqrt(K / 8 * sum (a b)^2)."""
    K = a.shape[1]
    off = (K + 8) * F32 * 2 * (abs(a) @ abs(b.T))
    if codes:
        off = off + 7 * 2.0 ** -13 * np.sqrt(K / 8 * ((a * a) @ (b * b).T))
    return a @ b.T, off


ROWS = [
    ([1], 128, 128), ([1], 256, 384), ([3, 0, 17, 1], 256, 128), ([16, 16], 512, 256), ([33, 64, 65, 0, 0, 5], 384, 640),
    ([130, 1, 250], 1408, 256), ([0, 0, 300], 256, 1408), ([257], 640, 384), ([2] * 64, 256, 256), ([513, 40, 700], 512, 384),
    ([1000, 900, 1100, 1000], 256, 512), ([7] * 31 + [600], 384, 256),
]


@pytest.mark.parametrize("rows,H,F", ROWS)
def test_forward(rows, H, F):
    R = sum(rows)
    q, x, xs, offsets = _layer(rows, H, F, R + H, r_max=R + 5)
    h, hs, gu, y = _forward(q, x, xs, offsets)
    xv, lo = fb.rows_value(_np(x), _np(xs)), 0
    for e, n in enumerate(rows):
        r = slice(lo, lo + n)
        lo += n
        if n == 0:
            continue
        g, eg = _product(xv[r], _expert(q, "gate", e))
        u, eu = _product(xv[r], _expert(q, "up", e))
        assert (abs(_np(gu)[r, :F] - g) <= eg + BF16 * abs(g)).all() and (abs(_np(gu)[r, F:] - u) <= eu + BF16 * abs(u)).all()
        # silu's slope is at most 1.1; the exponential is off by a step of its argument's size, the rest by a few roundings
        hv = g * fb.sigmoid(g) * u
        err = 1.1 * abs(u) * eg + abs(g * fb.sigmoid(g)) * eu + abs(hv) * (16 + 4 * abs(g)) * F32
        small, large = fb.quantized_range(hv, err)
        got = fb.rows_value(_np(h)[r], _np(hs)[r])
        assert (small <= got).all() and (got <= large).all()
        yv, ey = _product(got, _expert(q, "down", e))
        assert (abs(_np(y)[r] - yv) <= ey + BF16 * abs(yv)).all()
        # all together: a rounding to bf16, and what is cut off (random: at most 1e-4 measured) far below it
        assert np.linalg.norm(_np(y)[r] - yv) <= (BF16 + 2.0 ** -11) * np.linalg.norm(yv)
    assert (_np(y)[R:] == 7).all() and (_np(gu)[R:] == 7).all() and (_np(h)[R:] == 0xa5).all() and (_np(hs)[R:] == 0xa5).all()
    assert (_np(hs)[:, F // 128:] == 0xa5).all()
    # the two halves are the whole, and g | u need not be kept
    h2, hs2, y2 = _bytes(*h.shape), _bytes(*hs.shape), torch.full_like(y, 7.0)
    moe.expert_gate_up_fp8_block(x, xs, offsets, q["gate"], q["gate_scales"], q["up"], q["up_scales"], h2, hs2)
    moe.expert_down_fp8_block(h2, hs2, offsets, q["down"], q["down_scales"], y2)
    assert torch.equal(h, h2) and torch.equal(hs, hs2) and torch.equal(y, y2)


@pytest.mark.parametrize("rows", [[4, 9], [300, 280]])
def test_a_row_that_is_not_finite_stays_alone(rows):
    H, F = 384, 256
    q, x, xs, offsets = _layer(rows, H, F, 1)
    clean = _forward(q, x, xs, offsets)
    x[2, 130:140], xs[2, 1] = 0x7f, 255                       # a block as quantisation leaves it
    x[5, 7] = 0x7f                                            # and a NaN of its own
    h, hs, gu, y = _forward(q, x, xs, offsets)
    bad = torch.zeros(len(x), dtype=torch.bool, device="cuda")
    bad[[2, 5]] = True
    assert y[bad].isnan().all() and gu[bad].isnan().all() and (hs[bad][:, :2] == 255).all() and (h[bad] == 0x7f).all()
    for got, want in zip((h, hs, gu, y), clean):
        assert torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("rows", [[5, 3], [290, 260]])
def test_scales_far_apart(rows):
    """Blocks of 2^-40 and of 2^40 beside one another, along rows and contraction."""
    H, F = 512, 256
    q, x, xs, offsets = _layer(rows, H, F, 2, spread=0.0)
    xs[:, 1] -= 40
    xs[1::2, 2] += 40
    q["gate_scales"][:, :, 2] -= 40
    q["up_scales"][:, 1, :] -= 30
    h, hs, gu, y = _forward(q, x, xs, offsets)
    xv, lo = fb.rows_value(_np(x), _np(xs)), 0
    for e, n in enumerate(rows):
        r = slice(lo, lo + n)
        lo += n
        for k, name in enumerate(("gate", "up")):
            v, err = _product(xv[r], _expert(q, name, e))
            assert (abs(_np(gu)[r, k * F:(k + 1) * F] - v) <= err + BF16 * abs(v)).all()
        yv, ey = _product(fb.rows_value(_np(h)[r], _np(hs)[r]), _expert(q, "down", e))
        assert (abs(_np(y)[r] - yv) <= ey + BF16 * abs(yv)).all()


def _backward(q, x, xs, h, hs, gu, dy, offsets):
    E, F, H = q["gate"].shape
    R = len(x)
    dx = torch.full((R, H), 7.0, dtype=torch.bfloat16, device="cuda")
    dw = [torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((E, F, H), (E, F, H), (E, H, F))]
    ws = torch.full((moe.expert_backward_fp8_block_workspace_bytes(R, H, F, E),), 0xff, dtype=torch.uint8, device="cuda")
    moe.grouped_gemm_swiglu_fp8_block_backward(x, xs, h, hs, gu, dy, offsets, q["wgu_t"], q["wgu_t_scales"], q["wd_t"],
                                               q["wd_t_scales"], dx, *dw, ws)
    return dx, dw


@pytest.mark.parametrize("rows,H,F", ROWS)
def test_backward(rows, H, F):
    R = sum(rows)
    q, x, xs, offsets = _layer(rows, H, F, R + F, r_max=R + 3)
    h, hs, gu, _ = _forward(q, x, xs, offsets)
    dy = (_values((R + 3, H), 77) * 1e-3).to(torch.bfloat16).cuda()
    dx, dw = _backward(q, x, xs, h, hs, gu, dy, offsets)
    xv, hv, guv, lo = fb.rows_value(_np(x), _np(xs)), fb.rows_value(_np(h)[:R], _np(hs)[:R]), _np(gu), 0
    for e, n in enumerate(rows):
        r = slice(lo, lo + n)
        lo += n
        if n == 0:
            assert all((_np(t)[e] == 0).all() for t in dw)
            continue
        dyv, g, u = _np(dy)[r], guv[r, :F], guv[r, F:]
        dyq = fb.rows_value(*fb.quantize_rows(dyv))
        dh, eh = _product(dyq, _expert(q, "wd_t", e))
        s = fb.sigmoid(g)
        d = np.concatenate([dh * u * s * (1 + g * (1 - s)), dh * g * s], 1)
        # the factors of dh, then what they are off: the exponential's argument, and the difference 1 - s, of up to 1
        factor = np.concatenate([abs(u) * s * (1 + abs(g) * (1 - s)), abs(g) * s], 1)
        near = np.concatenate([abs(u) * s * (1 + abs(g)), abs(g) * s], 1)
        err = factor * np.tile(eh, (1, 2)) + near * np.tile(abs(dh) * (24 + 8 * abs(g)), (1, 2)) * F32
        small, large = fb.quantized_range(d, err)
        wgu = _expert(q, "wgu_t", e)
        middle, slack = (small + large) / 2, (large - small) / 2
        dxv, ex = _product(middle, wgu)
        bound = ex + slack @ abs(wgu.T)
        assert (abs(_np(dx)[r] - dxv) <= bound + BF16 * (abs(dxv) + bound)).all()
        want, ew = _product(dyv.T, hv[r].T, codes=False)
        assert (abs(_np(dw[2])[e] - want) <= ew + BF16 * abs(want)).all()
        for k in range(2):
            dk = d[:, k * F:(k + 1) * F]
            want, ew = _product(dk.T, xv[r].T, codes=False)
            off = (err[:, k * F:(k + 1) * F] + BF16 * abs(dk)).T @ abs(xv[r])
            assert (abs(_np(dw[k])[e] - want) <= ew + off + BF16 * (abs(want) + off)).all()
    assert (_np(dx)[R:] == 7).all()


def test_backward_of_no_rows_is_zero():
    q, x, xs, offsets = _layer([0, 0], 256, 128, 3)
    dx, dw = _backward(q, x, xs, _bytes(0, 128), _bytes(0, 4), torch.empty((0, 256), dtype=torch.bfloat16, device="cuda"),
                       torch.empty((0, 256), dtype=torch.bfloat16, device="cuda"), offsets)
    assert all((t == 0).all() for t in dw)


def test_gradients_are_differences_of_the_unrounded_layer():
    """dx against differences of the forward on bf16 values in 64 bits, within what the 8-bit roundings of dy and of dg | du leave
    (each at most 2^-4 of a value, so the two at most 2^-3 of what is added up; typically far less)."""
    rows, H, F = [20, 12], 256, 128
    q, x, xs, offsets = _layer(rows, H, F, 5)
    h, hs, gu, _ = _forward(q, x, xs, offsets)
    dy = _values((32, H), 6).to(torch.bfloat16).cuda()
    dx, _ = _backward(q, x, xs, h, hs, gu, dy, offsets)
    xv, lo, rng = fb.rows_value(_np(x), _np(xs)), 0, np.random.default_rng(0)
    for e, n in enumerate(rows):
        w = [_expert(q, k, e) for k in ("gate", "up", "down")]

        def value(v):
            g, u = v @ w[0].T, v @ w[1].T
            return ((g * fb.sigmoid(g) * u) @ w[2].T * _np(dy)[lo:lo + n]).sum(1)
        for _ in range(4):
            way = rng.normal(size=(n, H))
            step = 1e-5
            slope = (value(xv[lo:lo + n] + step * way) - value(xv[lo:lo + n] - step * way)) / (2 * step)
            got = (_np(dx)[lo:lo + n] * way).sum(1)
            size = np.sqrt((_np(dx)[lo:lo + n] ** 2).sum(1))
            assert np.linalg.norm(got - slope) <= 2.0 ** -3 * np.linalg.norm(size)
        lo += n


def test_the_path_in_a_graph_and_on_another_stream():
    """Permute, FFN and backward of a step captured and replayed with new tokens, against the plain calls."""
    T, H, E, K, F = 200, 256, 8, 2, 384
    q = _layer([1] * E, H, F, 4)[0]
    R = T * K

    def buffers():
        b = dict(x=torch.empty((T, H), dtype=torch.bfloat16, device="cuda"), idx=torch.empty((T, K), dtype=torch.int32, device="cuda"),
                 c=_bytes(R, H), s=_bytes(R, fb.stride(H)), h=_bytes(R, F), hs=_bytes(R, fb.stride(F)),
                 gu=torch.empty((R, 2 * F), dtype=torch.bfloat16, device="cuda"), y=torch.empty((R, H), dtype=torch.bfloat16, device="cuda"),
                 dx=torch.empty((R, H), dtype=torch.bfloat16, device="cuda"),
                 ws=torch.empty(moe.permute_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda"),
                 bws=torch.empty(moe.expert_backward_fp8_block_workspace_bytes(R, H, F, E), dtype=torch.uint8, device="cuda"))
        b["maps"] = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (E, E + 1, R, R)]
        b["dw"] = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((E, F, H), (E, F, H), (E, H, F))]
        return b

    def step(b):
        moe.permute_fp8_block(b["x"], b["idx"], E, 0, b["c"], b["s"], *b["maps"], b["ws"])
        off = b["maps"][1]
        moe.grouped_gemm_swiglu_fp8_block(b["c"], b["s"], off, q["gate"], q["gate_scales"], q["up"], q["up_scales"], q["down"],
                                          q["down_scales"], b["h"], b["hs"], b["gu"], b["y"])
        moe.grouped_gemm_swiglu_fp8_block_backward(b["c"], b["s"], b["h"], b["hs"], b["gu"], b["y"], off, q["wgu_t"], q["wgu_t_scales"],
                                                   q["wd_t"], q["wd_t_scales"], b["dx"], *b["dw"], b["bws"])

    def fill(b, seed):
        gen = torch.Generator().manual_seed(seed)
        b["x"].copy_(torch.randn((T, H), generator=gen).to(torch.bfloat16))
        b["idx"].copy_(torch.rand((T, E), generator=gen).topk(K).indices.to(torch.int32))
    a, b = buffers(), buffers()
    fill(b, 0)
    step(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    other = torch.cuda.Stream()
    for seed in range(1, 4):
        fill(a, seed)
        fill(b, seed)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            step(a)
        graph.replay()
        torch.cuda.synchronize()
        for k in ("c", "s", "h", "gu", "y", "dx"):
            assert torch.equal(a[k], b[k]), k
        for p, r in zip(a["maps"] + a["dw"], b["maps"] + b["dw"]):
            assert torch.equal(p, r)


def test_tensors_of_the_formats_own_types():
    rows, H, F = [5, 9], 256, 128
    q, x, xs, offsets = _layer(rows, H, F, 8)
    want = _forward(q, x, xs, offsets)
    typed = {k: v.view(torch.float8_e8m0fnu if k.endswith("scales") else torch.float8_e4m3fn) for k, v in q.items()}
    got = _forward(typed, x.view(torch.float8_e4m3fn), xs.view(torch.float8_e8m0fnu), offsets)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
