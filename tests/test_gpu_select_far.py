"""Routing by scores where scores are far from 1: gradients of selected experts whose scores are small against fp32's range, or
against the largest of their row, and gates whose softmax adds up many small terms; against the oracle in 64 bits."""
import numpy as np
import pytest

from oracle import routing
from test_gpu_select import ULP, _backward, _check

pytestmark = pytest.mark.gpu

# logits of the two to four selected experts: both sides of where fp32's normal numbers end (87.3), of where its denormal ones do
# (103.3), and far from both, to where 64 bits end (709.78)
FAR = [(-85.0, -90.0), (-90.0, -90.0), (-87.3, -87.4, -88.8), (-100.0, -101.0), (-103.0, -104.5, -103.5), (-50.0, -90.0), (0.0, -80.0),
       (3.0, -70.0), (-150.0, -152.0), (-300.0, -301.5, -303.0, -300.25), (-700.0, -701.0), (-709.5, -708.0), (88.0, 91.0), (100.0, -95.0)]


def _case(score):
    """Rows of 16 logits; the selected ones are experts 1 to 4.  Softmax: beside an expert of logit 0 (a bias can keep that out)."""
    x = np.full((len(FAR), 16), -np.inf, dtype=np.float32)
    idx = np.full((len(FAR), 4), -1, dtype=np.int32)
    for t, row in enumerate(FAR):
        x[t, 1:1 + len(row)] = row
        idx[t, :len(row)] = 1 + np.arange(len(row))
        if score == routing.SOFTMAX:
            x[t, 0], x[t, 5] = 0.0, -0.5
    dgate = np.random.default_rng(3).normal(size=idx.shape).astype(np.float32)
    return x, idx, dgate


@pytest.mark.parametrize("score", [routing.SOFTMAX, routing.SIGMOID])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("K", [4, 12])
def test_gradient_of_small_scores(score, renormalize, K):
    x, idx, dgate = _case(score)
    idx = np.concatenate([idx, np.full((len(x), K - 4), -1, dtype=np.int32)], 1)
    dgate = np.concatenate([dgate, np.zeros((len(x), K - 4), dtype=np.float32)], 1)
    got = _backward(x, idx, dgate, score, renormalize, 1.0)
    want, size = routing.select_backward(x, idx, dgate, score, renormalize, 1.0)
    # Roundings: the argument of an exponential is a difference of two logits, off by half a step of it, which
    # moves the exponential by that distance (at most 110: beyond it lies 0) times ULP; two of them, and some 24 others.  A result
    # among fp32's denormal numbers: half a step of 2^-149 for each of the exponential, its product with 1 - s, with the gradient
    # (below 3), and of the sum.
    assert (abs(got - want) <= (24 + 2 * 110) * ULP * size + 8 * 2.0 ** -149).all()


def test_gates_of_small_scores_have_a_gradient():
    """Two selected logits of -90: gates of one half each, so the gradient is that of any two equal logits, times 1 - s = 1."""
    x = np.full((1, 4), -np.inf, dtype=np.float32)
    x[0, :2] = -90.0
    got = _backward(x, np.array([[0, 1]], dtype=np.int32), np.array([[1.0, -2.0]], dtype=np.float32), routing.SIGMOID, True, 1.0)
    np.testing.assert_allclose(got, [[0.75, -0.75, 0, 0]], rtol=8 * ULP)


@pytest.mark.parametrize("score,low", [(routing.SIGMOID, -710.0), (routing.SIGMOID, -1e30), (routing.SOFTMAX, -746.0), (routing.SOFTMAX, -1e30)])
def test_tokens_whose_gates_are_zero_get_no_gradient(score, low):
    x = np.zeros((3, 6), dtype=np.float32)
    x[:, 1:3] = low
    idx = np.tile(np.array([1, 2], dtype=np.int32), (3, 1))
    got = _backward(x, idx, np.ones((3, 2), dtype=np.float32), score, True, 1.0)
    assert (got == 0).all()


@pytest.mark.parametrize("E,K", [(256, 1), (256, 8), (160, 4), (64, 2), (256, 12), (255, 3)])
def test_softmax_gates_beside_many_small_terms(E, K):
    """One logit of 0 and all others where their exponentials, one by one, are half a step of 1: together up to 2^-17 of the sum."""
    x = (np.log(2.0 ** -25) - np.tile(np.linspace(0, 0.05, E), (5, 1))).astype(np.float32)
    for t in range(5):
        x[t, (t * 37) % E] = 0.0
    _check(x, K, routing.SOFTMAX, renormalize=False)
