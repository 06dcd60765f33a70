"""The training step as a whole: the layer's backward with the balance gradient, the gradient against differences of the
loss, and the example that trains a layer."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.gpu
@pytest.mark.parametrize("S", [1, 6])
def test_gradient_against_differences_of_the_loss(S):
    """Central differences of the fp32 losses along the signs of the gradient, h = 0.05: the derivative is the sum of the
    gradient's magnitudes, of the order of the losses.  Rounding of the losses (400 * 2^-24 each, see test_gpu_balance) over h
    is 0.05 %, the third-order term h^2 / 6 of a softmax 0.04 %: 2 % is far above both."""
    import torch
    import paper_2504_14960_amd as moe
    T, E, K = 600, 24, 3
    gen = torch.Generator().manual_seed(S)
    logits = (torch.randn((T, E), generator=gen) * 1.5 + torch.randn(E, generator=gen)).cuda()
    idx = logits.topk(K, 1).indices.int()                          # held fixed, as the gradient does
    mask = (torch.rand(T, generator=gen) > 0.2).cuda()
    offsets = None
    if S > 1:
        ends = torch.sort(torch.randint(0, T + 1, (S - 1,), generator=gen)).values
        offsets = torch.cat([torch.zeros(1), ends, torch.full((1,), T)]).int().cuda()
    counts, sums = torch.zeros((S, E), dtype=torch.int32, device="cuda"), torch.zeros((S, E), device="cuda")
    n, losses = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    ws = torch.empty(moe.balance_loss_workspace_bytes(T, E, S), dtype=torch.uint8, device="cuda")

    def loss(x, which):
        moe.balance_loss(x, idx, 1.0, 1.0, counts, sums, n, losses, ws, token_mask=mask, seq_offsets=offsets)
        return float(losses[which])

    for which in (0, 1):
        loss(logits, which)
        up = torch.zeros(2, device="cuda")
        up[which] = 1.0
        d = torch.empty_like(logits)
        moe.balance_loss_backward(logits, counts, n, up, K, 1.0, 1.0, d, token_mask=mask, seq_offsets=offsets)
        way = torch.sign(d)
        got = (loss(logits + 0.05 * way, which) - loss(logits - 0.05 * way, which)) / 0.1
        assert got == pytest.approx(float(d.double().abs().sum()), rel=0.02)
        assert got > 0.1 * loss(logits, which)


@pytest.mark.gpu
def test_layer_backward_takes_the_gradient_along():
    """Every output is, bit for bit, that of the stage calls with moe.router_backward taking the addend; what the addend changes
    in the router's gradients is its product with x, to the rounding of fp32 sums (300 * 2^-24)."""
    import torch
    import paper_2504_14960_amd as moe
    T, H, E, K, F = 200, 128, 8, 2, 128
    gen = torch.Generator().manual_seed(0)

    def normal(*shape, std=0.1):
        return (torch.randn(shape, generator=gen) * std).bfloat16().cuda()

    x, dy, router = normal(T, H, std=1.0), normal(T, H, std=1.0), normal(E, H)
    gate, up, down = normal(E, F, H), normal(E, F, H), normal(E, H, F)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    y, gu = torch.empty((T, H), **bf16), torch.empty((T * K, 2 * F), **bf16)
    ws = torch.empty(moe.layer_workspace_bytes(T, H, E, K, F, 0, 0, moe.MOE_BF16), dtype=torch.uint8, device="cuda")
    bws = torch.empty(moe.layer_backward_workspace_bytes(T, H, E, K, F, 0), dtype=torch.uint8, device="cuda")
    wgu_t, wd_t = torch.empty((E, H, 2 * F), **bf16), torch.empty((E, F, H), **bf16)
    moe.expert_weights_transpose(gate, up, down, wgu_t, wd_t)
    moe.layer_forward_train(x, router, None, gate, up, down, K, True, 0, y, gu, ws)
    addend = (torch.randn((T, E), generator=gen) * 0.3).cuda()

    def backward(addend):
        out = dict(dx=torch.empty((T, H), **bf16), dw=torch.empty((E, H), device="cuda"), db=torch.empty(E, device="cuda"),
                   dg=torch.empty_like(gate), du=torch.empty_like(up), dd=torch.empty_like(down))
        moe.layer_backward(x, router, gate, up, wgu_t, wd_t, dy, K, True, 0, ws, gu, out["dx"], out["dw"], out["db"], out["dg"],
                           out["du"], out["dd"], bws, dlogits_addend=addend)
        return out

    plain, zero, added = backward(None), backward(torch.zeros_like(addend)), backward(addend)
    for k in plain:
        assert torch.equal(plain[k], zero[k]), k
        if k in ("dg", "du", "dd"):
            assert torch.equal(plain[k], added[k]), k
    a, eps = addend.double(), 300 * 2.0 ** -24
    for k, more, size in (("dw", a.T @ x.double(), a.abs().T @ x.double().abs()), ("db", a.sum(0), a.abs().sum(0))):
        want = plain[k].double() + more
        assert ((added[k].double() - want).abs() <= eps * (size + plain[k].double().abs() + want.abs() + 1.0)).all(), k
        assert not torch.equal(added[k], plain[k])

    # the same from the stage calls
    lay = moe.layer_workspace_layout(T, H, E, K, F, 0, 0, moe.MOE_BF16)

    def kept(name, dtype, *shape):
        size = torch.empty(0, dtype=dtype).element_size() * int(np.prod(shape))
        return ws[lay[name]:lay[name] + size].view(dtype).view(shape)

    rows, f32 = T * K, dict(dtype=torch.float32, device="cuda")
    roa = kept("row_of_assign", torch.int32, rows)
    dy_perm, dx_perm, dgate = torch.empty((rows, H), **bf16), torch.empty((rows, H), **bf16), torch.empty((T, K), **f32)
    moe.unpermute_combine_backward(dy, kept("y_perm", torch.bfloat16, rows, H), roa, kept("topk_gate", torch.float32, T, K),
                                   dy_perm, dgate)
    ews = torch.empty(moe.expert_backward_workspace_bytes(rows, H, F, E), dtype=torch.uint8, device="cuda")
    dg, du, dd = torch.empty_like(gate), torch.empty_like(up), torch.empty_like(down)
    moe.grouped_gemm_swiglu_backward(kept("x_perm", torch.bfloat16, rows, H), kept("h", torch.bfloat16, rows, F), gu, dy_perm,
                                     kept("expert_offsets", torch.int32, E + 1), gate, up, wgu_t, wd_t, dx_perm, dg, du, dd, ews)
    dl, dx_router, dx = torch.empty((T, E), **f32), torch.empty((T, H), **bf16), torch.empty((T, H), **bf16)
    dw, db = torch.empty((E, H), **f32), torch.empty(E, **f32)
    rws = torch.empty(moe.router_backward_workspace_bytes(T, H, E), dtype=torch.uint8, device="cuda")
    moe.router_backward(x, router, kept("logits", torch.float32, T, E), kept("topk_idx", torch.int32, T, K), dgate, True, dl,
                        dx_router, dw, db, rws, dlogits_addend=addend)
    moe.permute_backward(dx_perm, roa, dx_router, dx, K)
    for k, t in dict(dx=dx, dw=dw, db=db, dg=dg, du=du, dd=dd).items():
        assert torch.equal(added[k], t), k
    assert not torch.equal(added["dx"], plain["dx"])


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["8bit", "f32"])
def test_example_learns_and_keeps_its_experts_busy(states):
    import train_step
    losses, shares = train_step.train(120, 0.1, states)
    assert np.mean(losses[-10:]) < 0.1 * losses[0]
    assert shares[0] > 0.9 and shares[-1] < 0.6


@pytest.mark.gpu
def test_example_without_the_balance_loss_uses_two_experts():
    import train_step
    _, shares = train_step.train(60, 0.0)
    assert shares[-1] > 0.9
