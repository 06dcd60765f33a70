"""A whole training step of one MoE layer: forward, balance loss, backward, gradient clipping, AdamW.

    python examples/train_step.py [--steps 200] [--balance 0.1] [--states 8bit|f32]

A layer of 8 experts learns to imitate a fixed random layer on tokens of a vocabulary of 512.  Its router starts with a bias
towards two of the experts; the balance loss evens them out (try --balance 0).  The experts' weights are bf16 with fp32
masters or, with --states 8bit, bf16 alone with 8-bit moments: 6 bytes an element instead of 16 with their gradient.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2504_14960_amd as moe  # noqa: E402

T, H, E, K, F = 2048, 256, 8, 2, 256


class Layer:
    """Weights, gradients and optimizer states of one layer, and what its calls need."""

    def __init__(self, states: str, seed: int = 0) -> None:
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, generator=gen, device="cuda") * 0.05

        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        f32 = dict(dtype=torch.float32, device="cuda")
        # the router's weight is read in bf16 and stepped in fp32; its bias is fp32
        masters = [normal(E, H), normal(E, F, H), normal(E, F, H), normal(E, H, F)]
        self.router, self.gate, self.up, self.down = (m.bfloat16() for m in masters)
        self.bias = torch.zeros(E, **f32)
        self.bias[:2] = 3.0
        self.d_router, self.d_bias = torch.empty((E, H), **f32), torch.empty(E, **f32)
        self.d_gate, self.d_up, self.d_down = (torch.empty_like(w) for w in (self.gate, self.up, self.down))
        self.gate_up_t, self.down_t = torch.empty((E, H, 2 * F), **bf16), torch.empty((E, F, H), **bf16)

        params = [self.router, self.bias, self.gate, self.up, self.down]
        grads = [self.d_router, self.d_bias, self.d_gate, self.d_up, self.d_down]
        small = [True, True, False, False, False] if states == "8bit" else [True] * 5
        m, v = ([torch.zeros(p.shape, dtype=torch.float32 if s else torch.uint8, device="cuda") for p, s in zip(params, small)]
                for _ in range(2))
        scales = [[None if s else torch.zeros((p.numel() + 31) // 32, dtype=torch.uint8, device="cuda")
                   for p, s in zip(params, small)] for _ in range(2)]
        kept = [masters[0], None] + (masters[1:] if states == "f32" else [None] * 3)
        self.tensors = moe.AdamWTensors(params, grads, m, v, masters=kept, exp_avg_scales=scales[0], exp_avg_sq_scales=scales[1],
                                        weight_decays=[0.0, 0.0, 0.01, 0.01, 0.01])

        self.y, self.dx = torch.empty((T, H), **bf16), torch.empty((T, H), **bf16)
        self.gu = torch.empty((moe.max_rows(T, K, E, 0), 2 * F), **bf16)
        self.ws = torch.empty(moe.layer_workspace_bytes(T, H, E, K, F, 0, 0, moe.MOE_BF16), dtype=torch.uint8, device="cuda")
        self.backward_ws = torch.empty(moe.layer_backward_workspace_bytes(T, H, E, K, F, 0), dtype=torch.uint8, device="cuda")
        layout = moe.layer_workspace_layout(T, H, E, K, F, 0, 0, moe.MOE_BF16)
        self.logits = self.ws[layout["logits"]:][:4 * T * E].view(torch.float32).view(T, E)
        self.topk_idx = self.ws[layout["topk_idx"]:][:4 * T * K].view(torch.int32).view(T, K)

        self.counts, self.prob_sums = torch.empty((1, E), dtype=torch.int32, device="cuda"), torch.empty((1, E), **f32)
        self.tokens, self.losses = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, **f32)
        self.balance_ws = torch.empty(moe.balance_loss_workspace_bytes(T, E), dtype=torch.uint8, device="cuda")
        self.dlogits = torch.empty((T, E), **f32)
        self.norm = torch.empty(2, **f32)                      # the norm, and the factor the step multiplies gradients with
        self.norm_ws = torch.empty(moe.grad_norm_workspace_bytes(len(params)), dtype=torch.uint8, device="cuda")

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        moe.layer_forward_train(x, self.router, self.bias, self.gate, self.up, self.down, K, True, 0, self.y, self.gu, self.ws)
        return self.y

    def step(self, x, dy, step, balance_coef, z_coef, lr) -> None:
        """Everything after the forward of x: dy is the gradient of the task's loss in y."""
        moe.balance_loss(self.logits, self.topk_idx, balance_coef, z_coef, self.counts, self.prob_sums, self.tokens, self.losses,
                         self.balance_ws)
        moe.balance_loss_backward(self.logits, self.counts, self.tokens, None, K, balance_coef, z_coef, self.dlogits)
        moe.expert_weights_transpose(self.gate, self.up, self.down, self.gate_up_t, self.down_t)
        moe.layer_backward(x, self.router, self.gate, self.up, self.gate_up_t, self.down_t, dy, K, True, 0, self.ws, self.gu,
                           self.dx, self.d_router, self.d_bias, self.d_gate, self.d_up, self.d_down, self.backward_ws,
                           dlogits_addend=self.dlogits)
        moe.grad_norm(self.tensors, self.norm, self.norm_ws, max_norm=1.0)
        moe.adamw_step(self.tensors, lr, 0.9, 0.99, 1e-8, step, seed=step, grad_scale=self.norm[1:])


def train(steps: int, balance_coef: float = 0.1, states: str = "8bit", report=None):
    """The task's loss and the share of assignments that the two busiest experts take, step by step."""
    layer, target = Layer(states, seed=1), Layer(states, seed=2)
    target.bias.zero_()
    gen = torch.Generator(device="cuda").manual_seed(3)
    vocabulary = torch.randn((512, H), generator=gen, device="cuda").bfloat16()
    history = []
    for step in range(1, steps + 1):
        x = vocabulary[torch.randint(512, (T,), generator=gen, device="cuda")]
        want = target.forward(x).float()
        y = layer.forward(x).float()
        scale = want.square().mean()
        loss = (y - want).square().mean() / scale
        dy = ((y - want) * (2.0 / (y.numel() * scale))).bfloat16()
        layer.step(x, dy, step, balance_coef, 1e-4, lr=3e-3)
        history.append((loss, layer.counts.float().topk(2).values.sum() / (T * K), layer.losses.clone(), layer.norm[0].clone()))
        if report and step % report == 0:
            loss, share, extra, norm = history[-1]
            print(f"step {step:4d}  loss {float(loss):.4f}  balance {float(extra[0]):.4f}  z {float(extra[1]):.5f}  "
                  f"gradient norm {float(norm):.3f}  two busiest experts {float(share):.3f}", flush=True)
    return [float(h[0]) for h in history], [float(h[1]) for h in history]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--balance", type=float, default=0.1)
    ap.add_argument("--states", choices=("8bit", "f32"), default="8bit")
    args = ap.parse_args()
    train(args.steps, args.balance, args.states, report=max(1, args.steps // 10))
