"""The routing oracle against hand-made cases and against differences of itself (CPU only), and the refusals of the calls."""
import ctypes as C

import numpy as np
import pytest

import paper_2504_14960_amd as moe
from oracle import routing


def test_bias_chooses_but_has_no_part_in_the_gates():
    logits = np.array([[0.0, 1.0, 2.0, -1.0]], dtype=np.float32)
    s = 1 / (1 + np.exp(-logits[0].astype(np.float64)))
    idx, gate = routing.select(logits, 2, routing.SIGMOID, bias=[0, 0, -1, 1], renormalize=False, scale=2.5)
    assert idx.tolist() == [[3, 1]]
    np.testing.assert_allclose(gate[0], 2.5 * s[[3, 1]])


def test_equal_keys_and_equal_groups_take_the_lower_index():
    idx, _ = routing.select(np.zeros((1, 8), dtype=np.float32), 3, routing.SOFTMAX)
    assert idx.tolist() == [[0, 1, 2]]
    idx, _ = routing.select(np.zeros((1, 8), dtype=np.float32), 3, routing.SIGMOID, groups=4, topk_groups=2)
    assert idx.tolist() == [[0, 1, 2]]


def test_groups_by_their_two_best():
    #                     group 0: one large    group 1: two middling
    logits = np.array([[3.0, -9.0, -9.0, 1.0, 1.0, -9.0]], dtype=np.float32)
    one, _ = routing.select(logits, 2, routing.SIGMOID, groups=2, topk_groups=1, group_best=1)
    two, _ = routing.select(logits, 2, routing.SIGMOID, groups=2, topk_groups=1, group_best=2)
    assert one.tolist() == [[0, 1]] and two.tolist() == [[3, 4]]


def test_experts_that_are_not_open_leave_slots_empty():
    logits = np.array([[-np.inf, 0.5, np.nan, -np.inf], [-np.inf] * 4], dtype=np.float32)
    for score in (routing.SOFTMAX, routing.SIGMOID):
        idx, gate = routing.select(logits, 3, score)
        assert idx.tolist() == [[1, -1, -1], [-1, -1, -1]]
        np.testing.assert_allclose(gate, [[1, 0, 0], [0, 0, 0]])


@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
@pytest.mark.parametrize("renormalize", [False, True])
def test_gradient_is_the_difference_of_the_gates(score, renormalize):
    rng = np.random.default_rng(3)
    logits = rng.normal(size=(3, 7)).astype(np.float32)
    logits[1, 2] = -np.inf
    idx, _ = routing.select(logits, 3, score, renormalize=renormalize)
    dgate = rng.normal(size=(3, 3)).astype(np.float32)
    d, size = routing.select_backward(logits, idx, dgate, score, renormalize, 1.5)

    def value(x):
        s, _ = routing.scores(x, score)
        g = np.take_along_axis(s, idx.astype(np.int64), 1)
        return 1.5 * (dgate * (g / g.sum(1, keepdims=True) if renormalize else g)).sum()
    step = 1e-5
    for t in range(3):
        for e in range(7):
            if logits[t, e] == -np.inf:
                assert d[t, e] == 0
                continue
            up, down = logits.astype(np.float64), logits.astype(np.float64)
            up[t, e] += step
            down[t, e] -= step
            # central difference: third derivatives times step^2 (about 1e-10) and rounding over the step (about 1e-11)
            assert abs((value(up) - value(down)) / (2 * step) - d[t, e]) < 1e-8
    assert (abs(d) <= size + 1e-15).all()


def test_bias_steps_towards_the_mean_load():
    b = routing.bias_update([[4, 1, 1], [2, 1, 3]], 0.5, np.zeros(3, dtype=np.float32))      # 6, 2, 4: the mean is 4
    assert b.tolist() == [-0.5, 0.5, 0.0]


# ---- refusals: nothing is launched ----
def _select(**kw):
    a = dict(x=None, w=None, lb=None, logits=4096, sb=None, T=4, H=8, E=8, K=2, score=1, groups=1, topk_groups=1, best=2, renorm=1,
             scale=1.0, dt=1, idx=4096, gate=4096)
    a.update(kw)
    return moe.lib().moe_router_select(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(E=0), 1), (dict(K=0), 1), (dict(K=9), 1), (dict(T=-1), 1), (dict(score=2), 1), (dict(dt=7), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(groups=3), 1), (dict(groups=0), 1), (dict(groups=16), 1), (dict(groups=4, topk_groups=0), 1),
    (dict(groups=4, topk_groups=5), 1), (dict(best=0), 1), (dict(best=3), 1), (dict(groups=4, topk_groups=1, K=3), 1),
    (dict(E=257, K=1), 2), (dict(E=128, K=65), 2), (dict(T=1 << 30, K=2), 2), (dict(T=(1 << 27) + 1, K=1), 2), (dict(logits=None), 1),
    (dict(logits=4100), 1), (dict(idx=None), 1), (dict(gate=None), 1), (dict(sb=4097), 1), (dict(x=4096), 1), (dict(x=4096, w=4096, H=12), 2),
])
def test_select_refusals(kw, status):
    assert _select(**kw) == status
    assert moe.lib().moe_last_error()


def test_no_tokens_is_no_error():
    assert _select(T=0, logits=None, idx=None, gate=None) == 0


def _backward(**kw):
    a = dict(x=None, w=None, logits=4096, idx=4096, dgate=4096, addend=None, T=4, H=8, E=8, K=2, score=1, renorm=1, scale=1.0, dt=1,
             dlogits=8192, dx=None, dw=None, db=None, ws=None, n=0)
    a.update(kw)
    return moe.lib().moe_router_select_backward(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=(1 << 27) + 1, K=1), 2), (dict(score=3), 1), (dict(scale=float("nan")), 1), (dict(K=9), 1), (dict(E=300, K=1), 2), (dict(logits=None), 1),
    (dict(idx=None), 1), (dict(dgate=None), 1), (dict(dlogits=None), 1), (dict(addend=8192), 1), (dict(addend=8200), 1),
    (dict(dx=4096), 1), (dict(dw=4096), 1), (dict(dw=4096, x=4096), 3), (dict(dw=4096, x=4096, ws=4096, n=8), 3),
    (dict(dx=4096, w=4096, H=12), 2), (dict(db=4097), 1),
])
def test_select_backward_refusals(kw, status):
    assert _backward(**kw) == status


@pytest.mark.parametrize("args,status", [
    ((4096, -1, 8, 0.1, 4096, None, 0), 1), ((4096, 1, 0, 0.1, 4096, None, 0), 1), ((4096, 1, 257, 0.1, 4096, None, 0), 2),
    ((4096, (1 << 20) + 1, 8, 0.1, 4096, None, 0), 2), ((4096, 1, 8, float("nan"), 4096, None, 0), 1),
    ((None, 1, 8, 0.1, 4096, None, 0), 1), ((4096, 1, 8, 0.1, None, None, 0), 1), ((4096, 1, 8, 0.1, 4098, None, 0), 1),
    ((4096, 4096, 8, 0.1, 4096, None, 0), 3), ((4096, 4096, 8, 0.1, 4096, 4096, 8), 3), ((4096, 0, 8, 0.1, None, None, 0), 0),
])
def test_bias_update_refusals(args, status):
    assert moe.lib().moe_router_bias_update(*args, None) == status


def test_bias_update_workspace():
    size = moe.router_bias_update_workspace_bytes
    assert size(1, 64) == 0 and size(4096, 256) > 0
    assert size(-1, 8) == size(1 << 21, 8) == size(4096, 0) == size(4096, 257) == 0
    assert all(size(n, 256) <= size(n + 37, 256) for n in range(0, 5000, 37))
    assert isinstance(C.c_size_t(size(4096, 256)).value, int)
