"""Routing by scores on the GPU against the oracle: selection exactly, gates and gradients within their roundings."""
import numpy as np
import pytest
import torch

import paper_2504_14960_amd as moe
from oracle import routing

pytestmark = pytest.mark.gpu
ULP = 2.0 ** -24     # half a step of fp32, relative


def _logits(T, E, seed, masked=0.0):
    rng = np.random.default_rng(seed)
    x = (rng.normal(size=(T, E)) * 1.5 + rng.normal(size=E) * 0.5).astype(np.float32)
    if masked:
        x[rng.random((T, E)) < 0.1] = -np.inf
        x[rng.random(T) < masked] = -np.inf
        x[rng.random((T, E)) < 0.02] = np.nan
    return x


def _select(x, K, score, bias=None, **kw):
    T, E = x.shape
    idx = torch.full((T, K), -7, dtype=torch.int32, device="cuda")
    gate = torch.full((T, K), float("nan"), device="cuda")
    moe.router_select(None, None, None, torch.from_numpy(x).cuda(), K, idx, gate, score=score,
                      select_bias=None if bias is None else torch.from_numpy(bias).cuda(), **kw)
    return idx.cpu().numpy(), gate.cpu().numpy().astype(np.float64)


def _check(x, K, score, bias=None, groups=1, topk_groups=1, group_best=2, renormalize=True, scale=1.0):
    idx, gate = _select(x, K, score, bias, n_groups=groups, topk_groups=topk_groups, group_best=group_best, renormalize=renormalize,
                        gate_scale=scale)
    want, g = routing.select(x, K, score, bias, groups, topk_groups, group_best, renormalize, scale)
    np.testing.assert_array_equal(idx, want)
    # score, sum (4: the softmax's exponentials and their sum), quotient, scale: at most eight roundings; underflow at the end
    assert (abs(gate - g) <= 8 * ULP * g + 2.0 ** -148 * max(1, scale)).all()


SHAPES = [  # T, E, K, groups, topk_groups, group_best
    (1, 2, 1, 1, 1, 1), (1, 8, 2, 1, 1, 2), (3, 1, 1, 1, 1, 2), (77, 8, 8, 2, 2, 2), (65, 16, 4, 4, 2, 1), (129, 60, 4, 1, 1, 2),
    (33, 60, 6, 5, 2, 2), (64, 64, 8, 8, 4, 2), (1, 64, 8, 8, 4, 2), (501, 64, 6, 1, 1, 1), (40, 72, 9, 6, 3, 2), (255, 128, 8, 4, 2, 2),
    (31, 160, 6, 8, 3, 1), (300, 256, 8, 8, 4, 2), (5, 256, 64, 4, 2, 2), (9, 256, 12, 256, 20, 2), (17, 255, 5, 51, 7, 2),
    (21, 37, 8, 1, 1, 2), (19, 250, 10, 2, 1, 2), (100, 33, 3, 11, 2, 2), (2, 192, 64, 3, 3, 1), (67, 4, 4, 1, 1, 2),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
@pytest.mark.parametrize("biased", [False, True])
def test_selection_and_gates(shape, score, biased):
    T, E, K, groups, topk_groups, best = shape
    x = _logits(T, E, T + E)
    bias = (np.random.default_rng(5).normal(size=E) * 0.1).astype(np.float32) if biased else None
    _check(x, K, score, bias, groups, topk_groups, best, renormalize=biased, scale=2.5 if biased else 1.0)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
def test_masked_experts_and_empty_rows(shape, score):
    T, E, K, groups, topk_groups, best = shape
    bias = (np.random.default_rng(6).normal(size=E) * 0.1).astype(np.float32)
    bias[0] = -np.inf
    if E > 4:
        bias[3] = np.nan
    _check(_logits(T, E, 3 * T + E, masked=0.3), K, score, bias, groups, topk_groups, best)


@pytest.mark.parametrize("E,groups,topk_groups", [(8, 1, 1), (64, 8, 3), (256, 8, 4), (60, 5, 2), (200, 4, 3)])
@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
def test_many_tokens_with_many_equal_and_nearly_equal_keys(E, groups, topk_groups, score):
    """Logits of a few values and their neighbours: ties of keys and of groups, and keys one step apart."""
    rng = np.random.default_rng(E)
    x = rng.integers(-3, 4, size=(4000, E)).astype(np.float32) * np.float32(0.25)
    x = np.where(rng.random(x.shape) < 0.3, np.nextafter(x, np.float32(9)), x)
    bias = (rng.integers(-1, 2, size=E) * 0.125).astype(np.float32)
    K = min(8, topk_groups * (E // groups))
    _check(x, K, score, bias, groups, topk_groups, 2)
    _check(x, K, score, None, groups, topk_groups, 1, renormalize=False)


@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
@pytest.mark.parametrize("E,groups,topk_groups", [(6, 1, 1), (64, 8, 4), (256, 1, 1)])
def test_extreme_logits_and_biases(score, E, groups, topk_groups):
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(200, E)) * rng.choice([1e-30, 1.0, 50.0, 1e5, 3e38], size=(200, 1))).astype(np.float32)
    x[::7, 1] = np.inf
    x[::5, 2] = np.inf
    x[::3, 3] = -np.finfo(np.float32).max
    bias = np.where(rng.random(E) < 0.3, rng.normal(size=E) * 1e30, rng.normal(size=E)).astype(np.float32)
    _check(x, min(4, E), score, bias, groups, topk_groups, 2)
    _check(x, min(4, E), score, None, groups, topk_groups, 2, renormalize=False)


def test_large_biases_that_cancel_in_a_group():
    """Pairs of experts with biases of +b and -b: a group's value is what is left of two far larger keys."""
    rng = np.random.default_rng(2)
    for b in (3.0, 1e3, 1e6, 1e7):
        x = (rng.normal(size=(3000, 16)) * 2).astype(np.float32)
        bias = np.tile([b, -b], 8).astype(np.float32)
        _check(x, 3, routing.SIGMOID, bias, groups=8, topk_groups=2, group_best=2)


@pytest.mark.parametrize("K", [4, 12])
@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
def test_biases_whose_sums_overflow(K, score):
    rng = np.random.default_rng(7)
    top = np.finfo(np.float32).max
    for seed in range(6):
        bias = rng.choice(np.array([3e38, -3e38, 2e38, -2e38, np.inf, -np.inf, top, -top, 0.1, 0, 1e30, -2e30], dtype=np.float32), size=32)
        _check(_logits(40, 32, seed, masked=0.1), K, score, bias, groups=8, topk_groups=4, group_best=2)
        _check(_logits(40, 32, seed, masked=0.1), K, score, bias)


@pytest.mark.parametrize("K", [3, 9])
def test_infinite_logits_beside_the_largest_finite_one(K):
    rng = np.random.default_rng(8)
    x = rng.choice(np.array([np.inf, np.finfo(np.float32).max, 1.0, -np.inf, np.nan], dtype=np.float32), size=(300, 12))
    for bias in (None, (rng.normal(size=12) * 3).astype(np.float32)):
        _check(x, K, routing.SOFTMAX, bias, renormalize=False)


def test_infinite_biases_choose_first_in_order():
    x = _logits(50, 16, 4)
    bias = np.zeros(16, dtype=np.float32)
    bias[[3, 9]] = np.inf
    idx, _ = _select(x, 3, moe.MOE_SCORE_SIGMOID, bias)
    assert (idx[:, :2] == [3, 9]).all()


@pytest.mark.parametrize("E,groups,topk_groups,K", [(256, 8, 4, 8), (256, 1, 1, 8), (64, 1, 1, 6), (8, 1, 1, 2), (60, 1, 1, 4), (160, 8, 3, 6)])
@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
def test_many_tokens(E, groups, topk_groups, K, score):
    x = _logits(20011, E, E + K, masked=0.05)
    bias = (np.random.default_rng(8).normal(size=E) * 0.05).astype(np.float32)
    _check(x, K, score, bias, groups, topk_groups, 2, scale=2.5)


@pytest.mark.parametrize("T,E,groups,topk_groups,K,score", [(131072, 64, 1, 1, 6, routing.SIGMOID), (131073, 64, 8, 3, 8, routing.SOFTMAX),
                                                            (140001, 128, 4, 2, 8, routing.SIGMOID), (1 << 20, 8, 1, 1, 2, routing.SIGMOID)])
def test_so_many_tokens_that_doubtful_ones_come_later(T, E, groups, topk_groups, K, score):
    """Rows of many equal and nearly equal keys among others; the same tokens in calls of few tokens."""
    rng = np.random.default_rng(T)
    x = _logits(T, E, 5)
    x[::50] = rng.integers(-3, 4, size=x[::50].shape).astype(np.float32) * np.float32(0.25)
    x[7::1000] = -np.inf
    bias = (rng.integers(-1, 2, size=E) * 0.125).astype(np.float32)
    kw = dict(n_groups=groups, topk_groups=topk_groups)
    idx, gate = _select(x, K, score, bias, **kw)
    assert (idx[7::1000] == -1).all() and (gate[7::1000] == 0).all()
    for lo in range(0, T, 65536):
        i, g = _select(x[lo:lo + 65536], K, score, bias, **kw)
        np.testing.assert_array_equal(idx[lo:lo + 65536], i)
        np.testing.assert_array_equal(gate[lo:lo + 65536], g)
    some = np.concatenate([np.arange(0, T, 50), np.arange(T - 3, T), rng.integers(0, T, 2000)])
    want, g = routing.select(x[some], K, score, bias, groups, topk_groups, 2, True, 1.0)
    np.testing.assert_array_equal(idx[some], want)
    assert (abs(gate[some] - g) <= 8 * ULP * g + 2.0 ** -148).all()


@pytest.mark.parametrize("dtype,T,H,E", [(torch.bfloat16, 1, 64, 8), (torch.bfloat16, 100, 1000, 12), (torch.bfloat16, 2100, 512, 64),
                                         (torch.bfloat16, 300, 256, 200), (torch.float32, 50, 132, 8), (torch.float32, 1500, 256, 32)])
def test_from_tokens(dtype, T, H, E):
    """The logits are moe_router_topk's bit for bit, and the selection is that of those logits."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, H), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((E, H), generator=gen, device="cuda") * 0.1).to(dtype)
    lb = torch.randn(E, generator=gen, device="cuda")
    a, b = torch.empty((T, E), device="cuda"), torch.empty((T, E), device="cuda")
    idx, gate = torch.empty((T, 2), dtype=torch.int32, device="cuda"), torch.empty((T, 2), device="cuda")
    moe.router_topk(x, w, lb, a, 2, True, idx, gate)
    moe.router_select(x, w, lb, b, 2, idx, gate, renormalize=False)
    assert torch.equal(a, b)
    want, g = routing.select(b.cpu().numpy(), 2, routing.SIGMOID, renormalize=False)
    np.testing.assert_array_equal(idx.cpu().numpy(), want)
    assert (abs(gate.cpu().numpy() - g) <= 8 * ULP * g).all()


# ---- gradient ----
def _backward(x, idx, dgate, score, renormalize, scale, addend=None):
    T, E = x.shape
    d = torch.full((T, E), float("nan"), device="cuda")
    moe.router_select_backward(None, None, torch.from_numpy(x).cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(dgate).cuda(), d,
                               None, None, None, None, score=score, renormalize=renormalize, gate_scale=scale,
                               dlogits_addend=None if addend is None else torch.from_numpy(addend).cuda())
    return d.cpu().numpy().astype(np.float64)


def _tolerance(x):
    """Roundings of a softmax's or sigmoid's part of the gradient: exponentials (2, and the argument's, a step of the largest
    distance), their sum over up to 256 (10), quotients and products (12)."""
    f = np.where(np.isfinite(x), x, np.nan)
    with np.errstate(all="ignore"):
        far = np.nan_to_num(np.nanmax(f, 1) - np.nanmin(f, 1)) if f.size else np.zeros(len(x))
    return (24 + 2 * np.minimum(far, 110))[:, None] * ULP


@pytest.mark.filterwarnings("ignore:All-NaN")
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_gradient(shape, score, renormalize, masked):
    T, E, K = shape[:3]
    x = _logits(T, E, T * 5 + E, masked)
    idx, _ = routing.select(x, K, score)
    rng = np.random.default_rng(T)
    dgate = rng.normal(size=(T, K)).astype(np.float32)
    dgate[idx < 0] = np.nan                                    # not looked at
    got = _backward(x, idx, dgate, score, renormalize, 2.5)
    want, size = routing.select_backward(x, idx, np.nan_to_num(dgate), score, renormalize, 2.5)
    assert (abs(got - want) <= _tolerance(x) * size + 2.0 ** -140).all()
    addend = rng.normal(size=(T, E)).astype(np.float32)
    more = _backward(x, idx, dgate, score, renormalize, 2.5, addend)
    np.testing.assert_array_equal(more.astype(np.float32), got.astype(np.float32) + addend)


@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
def test_gradient_of_repeated_and_foreign_slots(score):
    x = _logits(9, 20, 2)
    idx = np.tile(np.array([3, 3, -1, 20, 19, 3], dtype=np.int32), (9, 1))
    dgate = np.random.default_rng(0).normal(size=idx.shape).astype(np.float32)
    for renormalize in (False, True):
        got = _backward(x, idx, dgate, score, renormalize, 1.0)
        want, size = routing.select_backward(x, idx, dgate, score, renormalize, 1.0)
        assert (abs(got - want) <= _tolerance(x) * size).all()


@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
def test_gradient_of_extreme_logits(score):
    x = np.zeros((4, 8), dtype=np.float32)
    x[0] = [-1e30] * 8
    x[1] = [200, -200, 90, -90, 0, 1, 2, 3]
    x[2, :2] = np.inf
    x[3] = -np.inf
    idx = np.tile(np.array([0, 1], dtype=np.int32), (4, 1))
    dgate = np.array([[1.0, -2.0]] * 4, dtype=np.float32)
    for renormalize in (False, True):
        got = _backward(x, idx, dgate, score, renormalize, 1.0)
        want, size = routing.select_backward(x, idx, dgate, score, renormalize, 1.0)
        assert (abs(got - want) <= 300 * ULP * size + 2.0 ** -140).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_reaches_tokens_and_weights_as_in_router_backward(dtype):
    T, H, E, K = 333, 256, 24, 4
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((T, H), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((E, H), generator=gen, device="cuda") * 0.1).to(dtype)
    logits, idx, gate = torch.empty((T, E), device="cuda"), torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    moe.router_select(x, w, None, logits, K, idx, gate)
    dgate, addend = torch.randn((T, K), generator=gen, device="cuda"), torch.randn((T, E), generator=gen, device="cuda")
    ws = torch.empty(moe.router_backward_workspace_bytes(T, H, E), dtype=torch.uint8, device="cuda")
    d, dx, dw, db = torch.empty((T, E), device="cuda"), torch.empty_like(x), torch.empty((E, H), device="cuda"), torch.empty(E, device="cuda")
    moe.router_select_backward(x, w, logits, idx, dgate, d, dx, dw, db, ws, dlogits_addend=addend)
    d64, x64, w64 = (t.double().cpu().numpy() for t in (d, x, w))
    for got, want, size, terms in ((dx, d64 @ w64, abs(d64) @ abs(w64), E), (dw, d64.T @ x64, abs(d64.T) @ abs(x64), T),
                                   (db, d64.sum(0), abs(d64).sum(0), T)):
        last = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
        assert (abs(got.double().cpu().numpy() - want) <= terms * ULP * size + last * abs(want)).all()
    only = torch.empty((T, E), device="cuda")
    moe.router_select_backward(None, None, logits, idx, dgate, only, None, None, None, None, dlogits_addend=addend)
    assert torch.equal(only, d)


# ---- bias ----
@pytest.mark.parametrize("rows,E", [(1, 1), (1, 8), (1, 64), (3, 60), (64, 256), (65, 200), (500, 7), (4096, 256)])
def test_bias_update(rows, E):
    rng = np.random.default_rng(rows + E)
    counts = rng.integers(0, 50, size=(rows, E)).astype(np.int32)
    bias = rng.normal(size=E).astype(np.float32)
    got = torch.from_numpy(bias).cuda()
    ws = torch.empty(moe.router_bias_update_workspace_bytes(rows, E), dtype=torch.uint8, device="cuda")
    moe.router_bias_update(torch.from_numpy(counts).cuda(), 1e-3, got, ws)
    np.testing.assert_array_equal(got.cpu().numpy(), routing.bias_update(counts, 1e-3, bias))


def test_bias_update_of_even_and_of_huge_loads():
    got = torch.zeros(4, device="cuda")
    moe.router_bias_update(torch.full((4,), 5, dtype=torch.int32, device="cuda"), 0.5, got)
    assert got.tolist() == [0.0] * 4
    counts = torch.full((200, 4), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    counts[0, 2] -= 1
    ws = torch.empty(moe.router_bias_update_workspace_bytes(200, 4), dtype=torch.uint8, device="cuda")
    moe.router_bias_update(counts, 0.5, got, ws)
    assert got.tolist() == [-0.5, -0.5, 0.5, -0.5]


# ---- as a program uses them ----
def test_a_step_in_a_graph_and_on_another_stream():
    """Selection, its gradient, loads and the bias's step, captured and replayed with new logits, against the plain calls."""
    T, E, K = 700, 64, 8
    kw = dict(n_groups=8, topk_groups=4)
    bias0 = torch.randn(E, device="cuda") * 0.1

    def buffers():
        return dict(logits=torch.empty((T, E), device="cuda"), idx=torch.empty((T, K), dtype=torch.int32, device="cuda"),
                    gate=torch.empty((T, K), device="cuda"), dgate=torch.ones((T, K), device="cuda"), d=torch.empty((T, E), device="cuda"),
                    counts=torch.empty((1, E), dtype=torch.int32, device="cuda"), sums=torch.empty((1, E), device="cuda"),
                    n=torch.empty(2, dtype=torch.int32, device="cuda"), losses=torch.empty(2, device="cuda"), bias=bias0.clone(),
                    ws=torch.empty(moe.balance_loss_workspace_bytes(T, E), dtype=torch.uint8, device="cuda"))

    def step(b):
        moe.router_select(None, None, None, b["logits"], K, b["idx"], b["gate"], select_bias=b["bias"], **kw)
        b["dgate"].copy_(b["gate"] - 0.3)
        moe.router_select_backward(None, None, b["logits"], b["idx"], b["dgate"], b["d"], None, None, None, None)
        moe.balance_loss(b["logits"], b["idx"], 0.0, 0.0, b["counts"], b["sums"], b["n"], b["losses"], b["ws"])
        moe.router_bias_update(b["counts"], 0.01, b["bias"])

    batches = [torch.randn((T, E), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i in range(4)]
    a, b = buffers(), buffers()
    b["logits"].copy_(batches[0])
    step(b)                                   # loads the kernels before the capture
    b["bias"].copy_(bias0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    stream = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        step(b)
    b["bias"].copy_(bias0)
    other = torch.cuda.Stream()
    for x in batches:
        a["logits"].copy_(x)
        b["logits"].copy_(x)
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            step(a)
        graph.replay()
        torch.cuda.synchronize()
        for k in ("idx", "gate", "d", "counts", "bias"):
            assert torch.equal(a[k], b[k]), k


def test_binding_refuses_other_types_and_sizes():
    x = torch.zeros((4, 8), device="cuda")
    idx, gate = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    with pytest.raises(TypeError):
        moe.router_select(None, None, None, x.double(), 2, idx, gate)
    with pytest.raises(TypeError):
        moe.router_select(None, None, None, x, 2, idx.long(), gate)
    with pytest.raises(ValueError):
        moe.router_select(None, None, None, x, 3, idx, gate)
    with pytest.raises(ValueError):
        moe.router_select(None, None, None, x, 2, idx, gate, select_bias=torch.zeros(7, device="cuda"))
    with pytest.raises(ValueError):
        moe.router_select(None, None, None, torch.zeros((8, 4), device="cuda").t(), 2, idx, gate)
    with pytest.raises(TypeError):
        moe.router_bias_update(torch.zeros(8, dtype=torch.int64, device="cuda"), 0.1, torch.zeros(8, device="cuda"))
    with pytest.raises(ValueError):
        moe.router_bias_update(torch.zeros(9, dtype=torch.int32, device="cuda"), 0.1, torch.zeros(8, device="cuda"))
    with pytest.raises(ValueError):
        moe.router_bias_update(torch.zeros(8, dtype=torch.int32), 0.1, torch.zeros(8, device="cuda"))
