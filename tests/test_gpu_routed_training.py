"""Training steps of a layer that is routed by scores with a balancing bias and whose experts run on block-scaled E4M3: every stage against
64 bits on what the stage before it left, and steps captured into a graph against plain ones on another stream."""
import numpy as np
import pytest
import torch

import paper_2504_14960_amd as moe
from oracle import combine, combine_backward, permute_backward
from oracle import fp8_block as fb
from oracle import routing

pytestmark = pytest.mark.gpu
BF16 = 2.0 ** -8      # half a step, relative
F32 = 2.0 ** -24
RATE = 0.01


def _np(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


class Layer:
    def __init__(self, T, H, F, E, K, groups, topk_groups, capacity, seed):
        gen = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=gen)
        self.sizes, self.seed = (T, H, F, E, K, capacity), seed
        self.how = dict(n_groups=groups, topk_groups=topk_groups, gate_scale=2.5)
        R = moe.max_rows(T, K, E, capacity)
        dev, f32, i32 = "cuda", torch.float32, torch.int32
        self.w = [(normal(*s) / s[2] ** 0.5).to(dev) for s in ((E, F, H), (E, F, H), (E, H, F))]
        self.w_router = (normal(E, H) / H ** 0.5).bfloat16().to(dev)
        self.closed = torch.zeros(E)
        self.closed[2] = -float("inf")        # an expert that takes no tokens: where its group is the only one, K are not to be had
        self.closed, self.bias = self.closed.to(dev), torch.zeros(E, device=dev)
        self.x, self.dy = (torch.empty((T, H), dtype=torch.bfloat16, device=dev) for _ in range(2))
        b = lambda *s: torch.full(s, 0xa5, dtype=torch.uint8, device=dev)
        h = lambda *s: torch.full(s, 7.0, dtype=torch.bfloat16, device=dev)
        st = moe.fp8_block_scale_stride
        self.q = []
        for n, c in ((F, H), (F, H), (H, F), (H, 2 * F), (F, H)):
            self.q += [b(E, n, c), b(E, n // 128, st(c))]
        self.logits, self.dlogits = (torch.empty((T, E), dtype=f32, device=dev) for _ in range(2))
        self.idx, self.gate, self.dgate = (torch.empty((T, K), dtype=t, device=dev) for t in (i32, f32, f32))
        self.xc, self.xs, self.hc, self.hs = b(R, H), b(R, st(H)), b(R, F), b(R, st(F))
        self.gu, self.yp, self.dyp, self.dxp = h(R, 2 * F), h(R, H), h(R, H), h(R, H)
        self.y, self.dx_router, self.dx = h(T, H), h(T, H), h(T, H)
        self.counts, self.offsets, self.roa, self.aor = (torch.empty(n, dtype=i32, device=dev) for n in (E, E + 1, T * K, R))
        self.dw = [h(*t.shape) for t in self.w]
        self.dw_router = torch.empty((E, H), device=dev)
        self.ws = [b(n) for n in (moe.permute_workspace_bytes(T, K, E), moe.expert_backward_fp8_block_workspace_bytes(R, H, F, E),
                                  moe.router_backward_workspace_bytes(T, H, E))]

    def tokens(self, n):
        gen = torch.Generator().manual_seed(1000 * self.seed + n)
        for t in (self.x, self.dy):
            t.copy_(torch.randn(t.shape, generator=gen).bfloat16())

    def step(self):
        T, H, F, E, K, capacity = self.sizes
        q = self.q
        moe.expert_weights_fp8_block(*self.w, *q)
        moe.router_select(self.x, self.w_router, self.closed, self.logits, K, self.idx, self.gate, select_bias=self.bias, **self.how)
        moe.permute_fp8_block(self.x, self.idx, E, capacity, self.xc, self.xs, self.counts, self.offsets, self.roa, self.aor, self.ws[0])
        moe.grouped_gemm_swiglu_fp8_block(self.xc, self.xs, self.offsets, *q[:6], self.hc, self.hs, self.gu, self.yp)
        moe.unpermute_combine(self.yp, self.roa, self.gate, None, self.y)
        moe.unpermute_combine_backward(self.dy, self.yp, self.roa, self.gate, self.dyp, self.dgate)
        moe.grouped_gemm_swiglu_fp8_block_backward(self.xc, self.xs, self.hc, self.hs, self.gu, self.dyp, self.offsets, *q[6:], self.dxp,
                                                   *self.dw, self.ws[1])
        moe.router_select_backward(self.x, self.w_router, self.logits, self.idx, self.dgate, self.dlogits, self.dx_router,
                                   self.dw_router, None, self.ws[2], gate_scale=self.how["gate_scale"])
        moe.permute_backward(self.dxp, self.roa, self.dx_router, self.dx, K)
        moe.router_bias_update(self.counts, RATE, self.bias)

    def results(self):
        return dict(idx=self.idx, gate=self.gate, y=self.y, dx=self.dx, dgate=self.dgate, dlogits=self.dlogits, bias=self.bias,
                    dw_router=self.dw_router, **{"dw%d" % i: t for i, t in enumerate(self.dw)})

    def learn(self):
        for w, d in zip(self.w, self.dw):
            w.sub_(d, alpha=0.01)


SIZES = [
    dict(T=97, H=256, F=384, E=16, K=4, groups=4, topk_groups=1, capacity=0),      # groups of four: three are left of the closed one's
    dict(T=300, H=512, F=128, E=8, K=2, groups=1, topk_groups=1, capacity=60),     # rows are dropped
    dict(T=1, H=128, F=128, E=4, K=1, groups=2, topk_groups=1, capacity=0),
]


@pytest.mark.parametrize("size", SIZES)
def test_every_stage(size):
    a = Layer(seed=1, **size)
    T, H, F, E, K, capacity = a.sizes
    a.bias.copy_(torch.linspace(-0.1, 0.1, E))
    a.tokens(0)
    before = _np(a.bias).astype(np.float32)
    a.step()
    torch.cuda.synchronize()
    logits, idx, gate, roa = a.logits.cpu().numpy(), _np(a.idx), _np(a.gate), _np(a.roa)
    lv = _np(a.x) @ _np(a.w_router).T
    assert (abs(logits - lv)[:, np.arange(E) != 2] <= ((H + 2) * F32 * (abs(_np(a.x)) @ abs(_np(a.w_router)).T))[:, np.arange(E) != 2]).all()
    want, g = routing.select(logits, K, routing.SIGMOID, before, a.how["n_groups"], a.how["topk_groups"], 2, True, 2.5)
    np.testing.assert_array_equal(idx, want)
    assert (idx != 2).all() and (size["groups"] != 4 or (idx == -1).any())
    assert (abs(gate - g) <= 8 * F32 * g).all()
    rows = [(t, k) for t in range(T) for k in range(K) if roa[t * K + k] >= 0]
    assert all(idx[t, k] >= 0 for t, k in rows) and len(rows) == _np(a.offsets)[E]
    assert capacity == 0 or len(rows) < T * K
    codes, scales = fb.quantize_rows(_np(a.x))
    for t, k in rows:
        r = roa[t * K + k]
        np.testing.assert_array_equal(_np(a.xc[r]), codes[t])
        np.testing.assert_array_equal(_np(a.xs[r, :H // 128]), scales[t])
    # y: K products added up in fp32, one rounding
    yp = _np(a.yp)
    y, size_y = combine(yp, roa, gate), combine(abs(yp), roa, abs(gate))
    assert (abs(_np(a.y) - y) <= BF16 * abs(y) + (K + 1) * F32 * 2 * size_y).all()
    dyp, dgate = combine_backward(_np(a.dy), yp, roa, gate)
    at = [roa[t * K + k] for t, k in rows]
    assert (abs(_np(a.dyp)[at] - dyp[at]) <= (BF16 + 2 * F32) * abs(dyp[at])).all()
    dsize = combine_backward(abs(_np(a.dy)), abs(yp), roa, gate)[1]
    assert (abs(_np(a.dgate) - dgate) <= (H + 2) * F32 * 2 * dsize).all()
    # exponentials, the sum of K of them, quotients and the product: some 40 roundings of what is added up
    dl, dl_size = routing.select_backward(logits, idx, _np(a.dgate), routing.SIGMOID, True, 2.5)
    assert (abs(_np(a.dlogits) - dl) <= 64 * F32 * dl_size + 2.0 ** -140).all()
    # in the routing's products the operands are the logits' gradient as it stands
    d, w, x = _np(a.dlogits), _np(a.w_router), _np(a.x)
    assert (abs(_np(a.dx_router) - d @ w) <= BF16 * abs(d @ w) + (E + 2) * F32 * 2 * (abs(d) @ abs(w))).all()
    assert (abs(_np(a.dw_router) - d.T @ x) <= (T + 2) * F32 * 2 * (abs(d).T @ abs(x))).all()
    dx, dx_size = (permute_backward(f(_np(a.dxp)), roa, T, K, f(_np(a.dx_router))) for f in (lambda v: v, abs))
    assert (abs(_np(a.dx) - dx) <= BF16 * abs(dx) + (K + 2) * F32 * 2 * dx_size).all()
    np.testing.assert_array_equal(a.bias.cpu().numpy(), routing.bias_update(_np(a.counts), RATE, before))


def test_steps_in_a_graph_and_on_another_stream():
    a, b = (Layer(seed=2, **SIZES[0]) for _ in range(2))
    for t in (a, b):
        t.tokens(0)
        t.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    other = torch.cuda.Stream()
    last = None
    for n in range(1, 5):
        for t in (a, b):
            t.learn()
            t.tokens(n)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            a.step()
        graph.replay()
        torch.cuda.synchronize()
        got = b.results()
        for k, v in a.results().items():
            assert torch.equal(v, got[k]), k
        assert last is None or not torch.equal(last, a.bias)
        last = a.bias.clone()
