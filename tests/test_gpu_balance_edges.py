"""Balance loss and its gradient at the edges of what the interface promises: rows, values and sizes that ordinary calls do not
have.  Tolerances are those of test_gpu_balance, which derives them."""
import numpy as np
import pytest

from oracle import training as o
from test_gpu_balance import EPS, _backward, _dev, _forward, _inputs


def _gradient_holds(got, logits, counts, n, offsets, addend=None):
    d, size = o.balance_loss_backward(logits, counts, n, (1.0, 1.0), 2, np.float32(0.01), np.float32(0.001), None, offsets)
    if addend is not None:
        d, size = d + addend, size + abs(addend)
    assert (abs(got - d) <= 64 * EPS * size + 1e-37).all()


@pytest.mark.gpu
@pytest.mark.parametrize("E", [3, 4, 8, 16, 32, 60, 64, 128, 200, 256])
@pytest.mark.parametrize("T,offsets", [(400, [100, 300]), (5000, [2100, 2100, 3300, 4800]), (70000, [66000, 68000, 69990])])
def test_rows_outside_every_sequence_are_left_untouched(E, T, offsets):
    """Before the first sequence and behind the last one, whatever multiple of a chunk they start at, in place too."""
    import torch
    import paper_2504_14960_amd as moe
    offsets = np.array(offsets, np.int32)
    logits, idx, _, _ = _inputs(T, E, 2)
    counts, sums, n, losses = _forward(logits, idx, None, offsets)
    inside = slice(offsets[0], offsets[-1])
    want = o.balance_loss(logits[inside], idx[inside], np.float32(0.01), np.float32(0.001), None, offsets - offsets[0])
    np.testing.assert_array_equal(counts.cpu().numpy(), want[0])
    np.testing.assert_array_equal(n.cpu().numpy(), want[2])
    np.testing.assert_allclose(sums.cpu().numpy(), want[1], rtol=340 * EPS, atol=1e-30)
    np.testing.assert_allclose(losses.cpu().numpy(), want[3], rtol=400 * EPS, atol=1e-30)

    addend = np.random.default_rng(1).standard_normal((T, E)).astype(np.float32) * np.float32(1e-4)
    out = _dev(addend)
    moe.balance_loss_backward(_dev(logits), counts, n, None, 2, 0.01, 0.001, out, addend=out, seq_offsets=_dev(offsets))
    plain = _backward(logits, 2, counts, n, None, offsets, None)
    torch.cuda.synchronize()
    for got, add, outside in ((out.cpu().numpy(), addend[inside], addend), (plain.cpu().numpy(), None, np.full((T, E), -7.0, np.float32))):
        np.testing.assert_array_equal(got[:offsets[0]], outside[:offsets[0]])
        np.testing.assert_array_equal(got[offsets[-1]:], outside[offsets[-1]:])
        _gradient_holds(got[inside], logits[inside], want[0], want[2], offsets - offsets[0], add)


def test_a_workspace_for_the_largest_call_serves_every_smaller_one():
    """The bytes asked for never fall as tokens, experts or sequences grow."""
    import paper_2504_14960_amd as moe
    need = moe.balance_loss_workspace_bytes
    tokens = sorted({max(0, t + d) for t in (0, 64, 128, 512, 4096, 16384, 32768, 65536, 131072, 262144, 1 << 20, 1 << 24, 1 << 30)
                     for d in (-64, -1, 0, 1, 63, 64, 65, 2000) if t + d <= 1 << 30})
    experts, sequences = (1, 2, 4, 16, 17, 60, 64, 65, 128, 129, 255, 256), (1, 2, 3, 4, 5, 15, 16, 17, 33, 256, 1000, 4096, 65536)
    for E in experts:
        for S in sequences:
            sizes = [need(T, E, S) for T in tokens]
            assert sizes == sorted(sizes), (E, S)
    for T in tokens:
        for S in sequences:
            sizes = [need(T, E, S) for E in experts]
            assert sizes == sorted(sizes), (T, S)
        for E in experts:
            sizes = [need(T, E, S) for S in sequences]
            assert sizes == sorted(sizes), (T, E)


def test_a_workspace_of_several_gigabytes_is_asked_for_whole():
    """Packed sequences leave a sum and a count of every expert for 256 tokens or fewer: more bytes than 32 bits count."""
    import paper_2504_14960_amd as moe
    for T, E, S in ((1 << 28, 256, 1), (1 << 28, 256, 65536), (1 << 29, 129, 3), (1 << 30, 64, 1), (1 << 30, 256, 1)):
        assert moe.balance_loss_workspace_bytes(T, E, S) >= (T // 256 + S) * E * 8, (T, E, S)


def test_sizes_that_a_call_refuses_need_no_workspace():
    import paper_2504_14960_amd as moe
    need = moe.balance_loss_workspace_bytes
    assert need(1 << 30, 256, 65536) > 0
    for T, E, S in (((1 << 30) + 1, 8, 1), (100, 257, 1), (100, 8, 65537), ((1 << 31) - 1, 8, (1 << 31) - 1)):
        assert need(T, E, S) == 0, (T, E, S)


@pytest.mark.gpu
@pytest.mark.parametrize("up", [np.inf, -np.inf, np.nan, 3e38])
@pytest.mark.parametrize("E", [3, 8, 16, 60, 64, 200, 256])
def test_rows_that_do_not_count_whatever_the_upstream_gradient(E, up):
    """Masked rows and rows of -inf are 0 (+ addend) where the gradient of the others is not finite."""
    logits, idx, _, offsets = _inputs(500, E, 2, 3)
    mask = (np.arange(500) % 3 != 0).astype(np.uint8)
    logits[mask == 0] = np.nan
    logits[1::9] = -np.inf
    nothing = (mask == 0) | (logits[:, 0] == -np.inf)
    counts, _, n, _ = _forward(logits, idx, mask, offsets)
    addend = np.random.default_rng(2).standard_normal((500, E)).astype(np.float32)
    ups = np.array([up, up], np.float32)
    for add in (None, addend):
        got = _backward(logits, 2, counts, n, mask, offsets, ups, add, cb=3e38, cz=1.0).cpu().numpy()
        np.testing.assert_array_equal(got[nothing], 0.0 if add is None else add[nothing])
        assert not np.isfinite(got[~nothing]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,S", [(40, 1), (3000, 1), (3000, 4)])
def test_logits_of_the_lowest_value(T, S):
    """Rows whose mask leaves nothing, as the type's lowest value: uniform, with a log-sum-exp whose square passes fp32.  A z
    loss that is switched off is 0 then, and one that is tiny is what the formula gives."""
    import torch
    import paper_2504_14960_amd as moe
    E = 16
    logits, idx, _, offsets = _inputs(T, E, 2, S)
    logits[5] = np.finfo(np.float32).min
    logits[6] = np.float32(1e20)
    for cz in (0.0, 2e-38):
        counts, sums, n, losses = _forward(logits, idx, None, offsets, cz=cz)
        want = o.balance_loss(logits, idx, np.float32(0.01), np.float32(cz), None, offsets)
        np.testing.assert_allclose(sums.cpu().numpy(), want[1], rtol=340 * EPS, atol=1e-30)
        with np.errstate(over="ignore"):
            np.testing.assert_allclose(losses.cpu().numpy(), want[3].astype(np.float32), rtol=400 * EPS, atol=1e-30)
    logits[5] = logits[6]
    losses = _forward(logits, idx, None, offsets, cz=1e-30)[3]
    want = o.balance_loss(logits, idx, np.float32(0.01), np.float32(1e-30), None, offsets)[3]
    assert 1e5 < want[1] < 1e10
    np.testing.assert_allclose(losses.cpu().numpy(), want, rtol=400 * EPS)
    out = torch.empty((T, E), device="cuda")
    moe.balance_loss_backward(_dev(logits), counts, n, None, 2, 0.01, 0.0, out, seq_offsets=_dev(offsets))
    assert torch.isfinite(out).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,S,masked", [(9000, 64, 2, 0.0), (9000, 64, 2, 0.2), (6000, 65, 1, 0.1), (70000, 64, 2, 0.1), (5000, 256, 1, 0.0)])
def test_many_chunks_a_sequence(T, E, S, masked):
    """More than 64 chunks of every sequence, which are added up by several workgroups."""
    rng = np.random.default_rng(T + E)
    logits, idx, mask, _ = _inputs(T, E, 2, 1, masked)
    middle = [T // 2 + int(rng.integers(-9, 9))] if S == 2 else []
    offsets = np.array([0] + middle + [T], np.int32)
    counts, sums, n, losses = _forward(logits, idx, mask, offsets)
    want = o.balance_loss(logits, idx, np.float32(0.01), np.float32(0.001), mask, offsets)
    np.testing.assert_array_equal(counts.cpu().numpy(), want[0])
    np.testing.assert_array_equal(n.cpu().numpy(), want[2])
    np.testing.assert_allclose(sums.cpu().numpy(), want[1], rtol=340 * EPS, atol=1e-30)
    np.testing.assert_allclose(losses.cpu().numpy(), want[3], rtol=400 * EPS, atol=1e-30)


@pytest.mark.gpu
def test_gradient_of_more_tokens_than_one_row_of_a_grid():
    """2^28 and some tokens of 129 experts: 2^24 workgroups of 256 threads, 2^32 threads.  All rows but the last thousand are alike."""
    import torch
    import paper_2504_14960_amd as moe
    T, E, tail = (1 << 28) + 777, 129, 1000
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 8 * T * E + (6 << 30):
        pytest.skip("needs 260 GiB of free device memory")
    logits, out = torch.zeros((T, E), device="cuda"), torch.full((T, E), -7.0, device="cuda")
    last = _inputs(tail, E, 2)[0]
    logits[T - tail:] = _dev(last)
    rng = np.random.default_rng(4)
    counts, n = rng.integers(0, 2 * T // E, (1, E)).astype(np.int32), np.array([T, T], np.int32)
    moe.balance_loss_backward(logits, _dev(counts), _dev(n), _dev(np.array([1e9, 1e9], np.float32)), 2, 0.01, 0.001, out)
    torch.cuda.synchronize()
    few = np.concatenate([np.zeros((1, E), np.float32), last])
    d, size = o.balance_loss_backward(few, counts.astype(np.int64), n.astype(np.int64), (1e9, 1e9), 2, np.float32(0.01), np.float32(0.001))
    got = torch.cat([out[:1], out[T - tail:]]).cpu().numpy()
    assert (abs(got - d) <= 64 * EPS * size + 1e-37).all()
    row = out[0].clone()
    for a in range(0, T - tail, 1 << 22):
        assert bool((out[a:min(a + (1 << 22), T - tail)] == row).all()), a
    del logits, out
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("T,E,K", [(8192, 1, 1), (8193, 1, 1), (8192, 2, 2), (8193, 2, 2), (16384, 2, 2), (10922, 3, 2), (8192, 4, 4), (8193, 4, 1)])
def test_few_experts_around_the_line_between_one_chunk_and_many(T, E, K):
    logits, idx, _, _ = _inputs(T, E, K)
    counts, sums, n, losses = _forward(logits, idx, None, None)
    want = o.balance_loss(logits, idx, np.float32(0.01), np.float32(0.001))
    np.testing.assert_array_equal(counts.cpu().numpy(), want[0])
    np.testing.assert_array_equal(n.cpu().numpy(), want[2])
    np.testing.assert_allclose(sums.cpu().numpy(), want[1], rtol=340 * EPS, atol=1e-30)
    np.testing.assert_allclose(losses.cpu().numpy(), want[3], rtol=400 * EPS, atol=1e-30)
