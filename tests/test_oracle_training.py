"""The training-step oracle against things that are not itself: torch's optimizer and autograd, differences, closed forms."""
import numpy as np
import pytest
import torch

from oracle import training as o


def _case(T, E, K, seed=0, S=1, masked=0.0):
    rng = np.random.default_rng(seed)
    logits = rng.standard_normal((T, E)) * 2
    idx = np.argsort(-logits, axis=1)[:, :K].astype(np.int32)
    mask = (rng.random(T) >= masked).astype(np.uint8) if masked else None
    offsets = np.concatenate([[0], np.sort(rng.integers(0, T + 1, S - 1)), [T]]) if S > 1 else None
    return logits, idx, mask, offsets


def test_balance_loss_of_even_routing_is_the_coefficient():
    T, E, K = 24, 6, 2
    idx = np.array([[(2 * t) % E, (2 * t + 1) % E] for t in range(T)])
    counts, sums, n, losses = o.balance_loss(np.zeros((T, E)), idx, 0.5, 2.0)
    assert (counts == T * K // E).all() and np.allclose(sums, T / E) and list(n) == [T, T]
    assert np.isclose(losses[0], 0.5) and np.isclose(losses[1], 2.0 * np.log(E) ** 2)


def test_balance_loss_of_one_expert_that_takes_all():
    """Every token sure of expert 0: E times the coefficient for K = 1."""
    logits = np.full((10, 4), -50.0)
    logits[:, 0] = 50.0
    _, _, _, losses = o.balance_loss(logits, np.zeros((10, 1), dtype=np.int32), 1.0, 0.0)
    assert np.isclose(losses[0], 4.0)


def test_sequences_weigh_by_their_tokens_and_padding_does_not_count():
    logits, idx, _, _ = _case(30, 5, 2)
    parts = [o.balance_loss(logits[a:b], idx[a:b], 1.0, 1.0)[3] for a, b in ((0, 7), (7, 30))]
    both = o.balance_loss(logits, idx, 1.0, 1.0, offsets=[0, 7, 7, 30])[3]
    assert np.allclose(both, (7 * parts[0] + 23 * parts[1]) / 30)
    padded = np.concatenate([logits, np.full((4, 5), np.nan)])
    again = o.balance_loss(padded, np.concatenate([idx, np.zeros((4, 2), int)]), 1.0, 1.0,
                           mask=np.r_[np.ones(30), np.zeros(4)], offsets=[0, 7, 34])[3]
    assert np.allclose(again, both)


@pytest.mark.parametrize("S,masked", [(1, 0.0), (4, 0.3)])
def test_balance_gradient_against_differences(S, masked):
    logits, idx, mask, offsets = _case(12, 5, 2, 3, S, masked)
    counts, _, n, _ = o.balance_loss(logits, idx, 0.7, 0.3, mask, offsets)
    d, size = o.balance_loss_backward(logits, counts, n, (1.5, -0.5), 2, 0.7, 0.3, mask, offsets)
    for t in range(12):
        for e in range(5):
            h = 1e-5
            ends = []
            for sign in (h, -h):
                moved = logits.copy()
                moved[t, e] += sign
                ends.append(np.dot((1.5, -0.5), o.balance_loss(moved, idx, 0.7, 0.3, mask, offsets)[3]))
            assert abs((ends[0] - ends[1]) / (2 * h) - d[t, e]) < 1e-9
    assert (abs(d) <= size + 1e-18).all()


def test_balance_gradient_against_autograd():
    logits, idx, _, _ = _case(40, 7, 3, 5)
    counts, _, n, _ = o.balance_loss(logits, idx, 1.0, 1.0)
    x = torch.tensor(logits, requires_grad=True)
    p = torch.softmax(x, 1)
    f = torch.bincount(torch.tensor(idx).flatten(), minlength=7).double()
    loss = 7 / (3 * 40 * 40) * (f * p.sum(0)).sum() + (torch.logsumexp(x, 1) ** 2).mean()
    loss.backward()
    assert np.allclose(o.balance_loss(logits, idx, 1.0, 1.0)[3].sum(), loss.item())
    assert np.allclose(o.balance_loss_backward(logits, counts, n, (1, 1), 3, 1.0, 1.0)[0], x.grad.numpy(), atol=1e-14)


def test_adamw_against_torch():
    rng = np.random.default_rng(1)
    p = torch.tensor(rng.standard_normal(50), requires_grad=True)
    opt = torch.optim.AdamW([p], lr=3e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    q, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.tensor(g)
        opt.step()
        q, m, v = o.adamw(q, g, m, v, 3e-2, 0.8, 0.95, 1e-6, step, 0.1)
    assert np.allclose(q, p.detach().numpy(), rtol=1e-13)
    assert np.allclose(v, opt.state[p]["exp_avg_sq"].numpy(), rtol=1e-13)


def test_grad_norm_clips_like_torch():
    rng = np.random.default_rng(2)
    g = [rng.standard_normal(n) for n in (3, 100)]
    p = [torch.nn.Parameter(torch.zeros(len(x), dtype=torch.float64)) for x in g]
    for q, x in zip(p, g):
        q.grad = torch.tensor(x)
    total = torch.nn.utils.clip_grad_norm_(p, 1.0)
    norm, scale = o.grad_norm(g, 1.0)
    assert np.isclose(norm, total.item()) and np.allclose(p[1].grad.numpy(), g[1] * scale)
    assert o.grad_norm(g)[1] == 1.0 and np.isnan(o.grad_norm([np.array([np.inf])], 1.0)[1])


def test_e4m3_values_are_torchs():
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(o.e4m3_values(), t)


def test_mxfp8_keeps_what_it_can_hold_and_is_unbiased():
    rng = np.random.default_rng(4)
    codes = rng.integers(0, 127, 320).astype(np.uint8) | (rng.integers(0, 2, 320) << 7).astype(np.uint8)
    codes[::32] = 0x7e                                              # the largest value: the scale is the smallest that fits
    scales = rng.integers(1, 248, 10).astype(np.uint8)
    for u in (0, 65535):
        c, s = o.mxfp8(o.mxfp8_values(codes, scales), np.full(320, u), False)
        np.testing.assert_array_equal(s, scales)
        np.testing.assert_array_equal(o.mxfp8_values(c, s), o.mxfp8_values(codes, scales))
    # over all 16-bit numbers the mean is the value itself, to the width of one of them
    u = np.arange(65536)
    for value in rng.standard_normal(20) * 10.0 ** rng.uniform(-4, 2, 20):
        blocks = np.full((2048, 32), value)
        blocks[:, 31] = 300.0                                       # so that the scale is 1
        codes, scales = o.mxfp8(blocks.flatten(), u, False)
        got = o.mxfp8_values(codes, scales).reshape(2048, 32)[:, :31]
        step = max(abs(value) / 8, 2.0 ** -9)                       # at most: three bits of mantissa
        assert abs(got.mean() - value) <= step * 1e-3


def test_mxfp8_scale_and_edges():
    c, s = o.mxfp8(np.zeros(33), np.zeros(33, int), True)
    assert (c == 0).all() and list(s) == [1, 1]
    c, s = o.mxfp8(np.array([448.0, 449.0]), np.zeros(2, int), False)
    assert s[0] == 128
    c, s = o.mxfp8(np.array([1.0, 1e-30]), np.zeros(2, int), True)
    assert c[1] == 1 and o.mxfp8(np.array([1.0, 1e-30]), np.zeros(2, int), False)[0][1] == 0
    c, s = o.mxfp8(np.array([1.0, np.nan]), np.zeros(2, int), False)
    assert s[0] == 255 and np.isnan(o.mxfp8_values(c, s)).all()


def test_random_bits_are_spread_and_differ_by_seed_tensor_and_high_half():
    j = np.arange(1 << 16)
    a = o.random_bits(7, 0, j)
    assert len(np.unique(a)) == len(j)
    for bit in range(32):
        assert abs(((a >> np.uint32(bit)) & 1).mean() - 0.5) < 0.01       # 5 standard deviations of 65536 draws
    for other in (o.random_bits(8, 0, j), o.random_bits(7, 1, j), o.random_bits(7, 0, j + (1 << 32))):
        assert (a == other).mean() < 1e-3


def test_bf16_stochastic_rounds_to_neighbours_and_keeps_exact_values():
    x = np.array([1.0, -2.5, 1 + 2.0 ** -9, 3.1415926], dtype=np.float32)
    for bits in (np.zeros(4, np.uint32), np.arange(4, dtype=np.uint32) * 0x10000001):
        back = (o.bf16_stochastic(x, bits).astype(np.uint32) << 16).view(np.float32)
        assert back[0] == 1.0 and back[1] == -2.5
        assert (abs(back - x) <= abs(x) * 2.0 ** -7).all()
