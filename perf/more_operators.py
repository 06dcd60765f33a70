"""Routing by scores with groups and a balancing bias, and the expert FFN in 8 bits with a scale for every block of 128, as a
set of measurable cases.

A case is a dict of plain values.  ``kind`` names the entry point a pass goes through:

* ``route``         moe.router_select: experts and gates of every token from its logits;
* ``route_backward``  moe.router_select_backward: the gradient of the gates in the logits;
* ``bias_update``   moe.router_bias_update: one step of the balancing bias from the experts' loads;
* ``weights``       moe.expert_weights_fp8_block: a layer's weights to E4M3 with a scale for every 128 x 128 of them, in the
                    layouts of the forward and of the backward;
* ``ffn``           moe.permute_fp8_block, moe.grouped_gemm_swiglu_fp8_block: tokens gathered by expert and quantised, and
                    the experts' FFN on them;
* ``ffn_backward``  moe.grouped_gemm_swiglu_fp8_block_backward: its gradients in the rows and in the weights.

Where ``own`` is false the same results come from elementary torch operations in 32 bits (scores, which decide what is
selected, in 64); ``exact`` has them in 64 bits.  Layer shapes are those of moe_inputs.configs, or generic.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
RATE = 1e-3
SOFTMAX, SIGMOID = "softmax", "sigmoid"


def _route(name, kind, T, E, K, **kw):
    return dict(name=name, kind=kind, **{**dict(T=T, E=E, K=K, score=SIGMOID, groups=1, topk_groups=1, group_best=2, bias=True,
                                                renormalize=True, scale=2.5, masked=0.0), **kw})


def _layer(name, kind, **kw):
    return dict(name=name, kind=kind, **kw)


def listed():
    return [
        # a batch of sequences being decoded: latency of a small call
        _route("route_32", "route", 32, 64, 8, groups=8, topk_groups=4),
        # a long-context batch on the most experts a layer may have, in groups (the nodes they live on)
        _route("route_262144", "route", 262144, 256, 8, groups=8, topk_groups=4),
        # packed tokens with padding and experts that some tokens may not take, in odd numbers, softmax scores
        _route("route_back_7777", "route_backward", 7777, 60, 4, score=SOFTMAX, scale=1.0, masked=0.1),
        # the gradient of the largest call
        _route("route_back_262144", "route_backward", 262144, 256, 8, groups=8, topk_groups=4),
        # the step of a router's balancing bias after one micro-batch
        dict(name="bias_1x64", kind="bias_update", rows=1, E=64),
        # the same after a global batch whose loads were kept per sequence
        dict(name="bias_4096x256", kind="bias_update", rows=4096, E=256),
        # fp32 masters of a small layer with sizes that are no powers of two
        _layer("weights_small_f32", "weights", E=12, H=1024, F=1408, dtype="f32"),
        # the token-drop configuration's bf16 weights after an optimizer step
        _layer("weights_tokendrop", "weights", E=64, H=4096, F=1408, dtype="bf16"),
        # a batch of sequences being decoded by a fine-grained layer: nearly every expert has a few rows
        _layer("ffn_decode_32_qwen2", "ffn", T=32, E=64, K=8, H=3584, F=2560, skew=0.0, save=False),
        # the benchmark's layer: long prompts, or the forward of a training step, which keeps what the backward needs
        _layer("ffn_8192_8x22b", "ffn", T=8192, E=8, K=2, H=6144, F=16384, skew=1.0, save=True),
        # a small micro-batch, tokens and experts in odd numbers
        _layer("ffn_back_777", "ffn_backward", T=777, E=12, K=3, H=1024, F=1408, skew=1.0),
        # a micro-batch of the fine-grained layer
        _layer("ffn_back_2048_g8t8", "ffn_backward", T=2048, E=64, K=8, H=6144, F=2048, skew=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["flops"] / 1e15, w["bytes"] / 4e12)


def draw(rng):
    """One more case of the same ranges: kinds in turn, tokens and sizes over their logarithm, odd ones too."""
    while True:
        kind = rng.choice(["route", "route", "route_backward", "bias_update", "weights", "ffn", "ffn", "ffn_backward"])
        if kind.startswith("route"):
            E, groups = rng.choice([(4, 1), (8, 2), (16, 4), (60, 1), (64, 1), (64, 8), (72, 6), (128, 4), (160, 8), (256, 8),
                                    (rng.randint(2, 256), 1)])
            topk_groups = rng.randint(1, groups)
            K = rng.randint(1, min(topk_groups * (E // groups), 12))
            # (one expert with its gate divided by itself: the gradient is 0, and relative errors say nothing)
            return dict(kind=kind, T=_log_int(rng, 1, 262144), E=E, K=K, score=rng.choice([SOFTMAX, SIGMOID]), groups=groups,
                        topk_groups=topk_groups, group_best=rng.choice([1, 2]), bias=rng.random() < 0.6,
                        renormalize=K > 1 and rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),
                        masked=rng.choice([0.0, 0.0, 0.1, 0.5]))
        if kind == "bias_update":
            return dict(kind=kind, rows=_log_int(rng, 1, 4096), E=rng.choice([8, 64, 256, rng.randint(2, 256)]))
        E, K = rng.choice([(4, 1), (8, 2), (12, 3), (16, 2), (32, 4), (60, 4), (64, 6), (64, 8), (128, 8)])
        case = dict(kind=kind, E=E, H=128 * rng.randint(2, 48), F=128 * _log_int(rng, 2, 96 if E <= 16 else 20))
        if kind == "weights":
            case["dtype"] = rng.choice(["bf16", "f32"])
        else:
            case.update(K=K, T=_log_int(rng, 1, 8192), skew=rng.choice([0.0, 0.5, 1.0]))
            if kind == "ffn":
                case["save"] = rng.random() < 0.4
        if E * case["H"] * case["F"] <= 6e8 and _cost(case) <= max(_cost(c) for c in listed()):
            return case


def work(case):
    """Bytes and operations a pass cannot do without."""
    kind = case["kind"]
    if kind == "route":
        T, E, K = (case[k] for k in ("T", "E", "K"))
        return {"bytes": 4 * T * E + 8 * T * K + (4 * E if case["bias"] else 0), "flops": 12 * T * E}
    if kind == "route_backward":
        T, E, K = (case[k] for k in ("T", "E", "K"))
        # sigmoid scores: the selected experts' logits are all that is looked at
        return {"bytes": 4 * T * (2 * E if case["score"] == SOFTMAX else E + K) + 8 * T * K, "flops": 8 * T * E}
    if kind == "bias_update":
        return {"bytes": 4 * case["rows"] * case["E"] + 8 * case["E"], "flops": case["rows"] * case["E"]}
    E, H, F = (case[k] for k in ("E", "H", "F"))
    n = 3 * E * H * F
    if kind == "weights":
        return {"bytes": n * ((2 if case["dtype"] == "bf16" else 4) + 2) + 2 * n / BLOCK ** 2, "flops": 4 * n}
    R = case["T"] * case["K"]
    # weights of experts that no token takes are not needed: as many as tokens that choose evenly are expected to reach
    taken = E * (1 - (1 - case["K"] / E) ** case["T"])
    weights = taken * 3 * H * F
    scales = (2 * H + 2 * F) / BLOCK
    if kind == "ffn":
        return {"bytes": weights + R * (2 * H / case["K"] + H + F + 2 * H + scales / 2 + (4 * F if case["save"] else 0)),
                "flops": 6 * R * H * F}
    return {"bytes": weights + R * (H + F + 4 * F + 2 * H + 2 * H + scales / 2) + 6 * E * H * F, "flops": 12 * R * H * F}


# ---------------------------------------------------------------------------------------------------------------
# inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["kind"].startswith("route"):
        return _prepare_route(case, gen)
    if case["kind"] == "bias_update":
        # loads of experts that are not balanced yet
        mean = torch.exp(torch.randn(case["E"], generator=gen, device="cuda")) * 64
        counts = torch.poisson(mean.expand(case["rows"], -1).contiguous(), generator=gen).to(torch.int32)
        st = dict(case=case, counts=counts, bias=torch.randn(case["E"], generator=gen, device="cuda") * 0.01)
        if own:
            import paper_2504_14960_amd as moe
            st["ws"] = torch.empty(moe.router_bias_update_workspace_bytes(case["rows"], case["E"]), dtype=torch.uint8,
                                   device="cuda")
        return st
    if case["kind"] == "weights":
        return _prepare_weights(case, gen)
    return _prepare_ffn(case, gen)


def _prepare_route(case, gen):
    T, E, K = (case[k] for k in ("T", "E", "K"))
    # logits of normalised tokens and the usual initialisation, and what tells the experts apart
    logits = torch.randn((T, E), generator=gen, device="cuda") * 1.5 + torch.randn(E, generator=gen, device="cuda") * 0.5
    if case["masked"]:
        logits[torch.rand((T, E), generator=gen, device="cuda") < 0.05] = -math.inf     # experts a token may not take
        pad = torch.rand(T, generator=gen, device="cuda") < case["masked"]              # padding takes none
        logits[pad] = -math.inf
    st = dict(case=case, logits=logits, bias=None)
    if case["bias"]:
        st["bias"] = torch.randn(E, generator=gen, device="cuda") * 0.05
    st["idx"] = torch.empty((T, K), dtype=torch.int32, device="cuda")
    st["gate"] = torch.empty((T, K), dtype=torch.float32, device="cuda")
    if case["kind"] == "route_backward":
        _plain_route(st)
        st["dgate"] = torch.randn((T, K), generator=gen, device="cuda") * 1e-2
        st["dlogits"] = torch.empty((T, E), dtype=torch.float32, device="cuda")
    return st


def _stride(C):
    """Bytes of a row of scales: whole words of four."""
    return (C // BLOCK + 3) // 4 * 4


def _codes(*shape):
    return torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")


def _scales(*shape):
    return torch.zeros(shape[:-1] + (_stride(shape[-1]),), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)


def _weight(case, gen, E, N, K, dtype):
    """Rows of a weight differ in size, as they do once trained."""
    w = torch.empty((E, N, K), dtype=dtype, device="cuda").normal_(0.0, 0.02, generator=gen)
    return w.mul_(torch.exp(0.5 * torch.randn((E, N, 1), generator=gen, device="cuda")).to(dtype))


def _prepare_weights(case, gen):
    E, H, F = (case[k] for k in ("E", "H", "F"))
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    st = dict(case=case, w_gate=_weight(case, gen, E, F, H, dtype), w_up=_weight(case, gen, E, F, H, dtype),
              w_down=_weight(case, gen, E, H, F, dtype))
    st["out"] = dict(gate=_codes(E, F, H), gate_scales=_scales(E, F // BLOCK, H), up=_codes(E, F, H),
                     up_scales=_scales(E, F // BLOCK, H), down=_codes(E, H, F), down_scales=_scales(E, H // BLOCK, F),
                     gate_up_t=_codes(E, H, 2 * F), gate_up_t_scales=_scales(E, H // BLOCK, 2 * F), down_t=_codes(E, F, H),
                     down_t_scales=_scales(E, F // BLOCK, H))
    return st


def _prepare_ffn(case, gen):
    T, E, K, H, F = (case[k] for k in ("T", "E", "K", "H", "F"))
    R = T * K
    x = torch.randn((T, H), generator=gen, device="cuda").to(torch.bfloat16)
    x[:, torch.randint(0, H, (max(1, H // 256),), generator=gen, device="cuda")] *= 20     # channels that stand out
    pull = torch.randn((T, E), generator=gen, device="cuda") + case["skew"] * torch.randn(E, generator=gen, device="cuda")
    idx = pull.topk(K, dim=1).indices.to(torch.int32)
    order = torch.sort(idx.flatten().long(), stable=True).indices
    counts = torch.bincount(idx.flatten().long(), minlength=E)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    st = dict(case=case, x=x, idx=idx, order=order, rows=counts.tolist())     # rows: for the plain form's loop over experts

    def weight(*shape):
        codes, scales = _codes(*shape), _scales(shape[0], shape[1] // BLOCK, shape[2])
        for e in range(E):
            _quantize_square(_weight(case, gen, 1, shape[1], shape[2], torch.bfloat16), codes[e:e + 1], scales[e:e + 1])
        return codes, scales

    if case["kind"] == "ffn":
        st["w_gate"], st["w_up"], st["w_down"] = weight(E, F, H), weight(E, F, H), weight(E, H, F)
        st["out"] = dict(x=_codes(R, H), x_scales=_scales(R, H), h=_codes(R, F), h_scales=_scales(R, F),
                         y=torch.empty((R, H), dtype=torch.bfloat16, device="cuda"))
        if case["save"]:
            st["out"]["gu"] = torch.empty((R, 2 * F), dtype=torch.bfloat16, device="cuda")
        if own:
            import paper_2504_14960_amd as moe
            st["maps"] = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (E, E + 1, R, R)]
            st["ws"] = torch.empty(moe.permute_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
        return st
    st["offsets"] = offsets
    st["wgu_t"], st["wd_t"] = weight(E, H, 2 * F), weight(E, F, H)
    st["xq"], st["hq"] = (_codes(R, H), _scales(R, H)), (_codes(R, F), _scales(R, F))
    gu = torch.randn((R, 2 * F), generator=gen, device="cuda")
    st["gu"] = gu.to(torch.bfloat16)
    _quantize_rows(x.float()[order // K], *st["xq"])
    _quantize_rows(_silu(gu[:, :F]) * gu[:, F:], *st["hq"])
    st["dy"] = (torch.randn((R, H), generator=gen, device="cuda") * 1e-3
                * torch.rand((R, 1), generator=gen, device="cuda")).to(torch.bfloat16)            # gates differ from row to row
    st["out"] = dict(dx=torch.empty((R, H), dtype=torch.bfloat16, device="cuda"),
                     dw_gate=torch.empty((E, F, H), dtype=torch.bfloat16, device="cuda"),
                     dw_up=torch.empty((E, F, H), dtype=torch.bfloat16, device="cuda"),
                     dw_down=torch.empty((E, H, F), dtype=torch.bfloat16, device="cuda"))
    if own:
        import paper_2504_14960_amd as moe
        st["ws"] = torch.empty(moe.expert_backward_fp8_block_workspace_bytes(R, H, F, E), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------------
# one pass

def run(st):
    return _RUN[st["case"]["kind"]](st)


def _run_route(st):
    c = st["case"]
    if own:
        import paper_2504_14960_amd as moe
        moe.router_select(None, None, None, st["logits"], c["K"], st["idx"], st["gate"],
                          score=moe.MOE_SCORE_SIGMOID if c["score"] == SIGMOID else moe.MOE_SCORE_SOFTMAX,
                          select_bias=st["bias"], n_groups=c["groups"], topk_groups=c["topk_groups"],
                          group_best=c["group_best"], renormalize=c["renormalize"], gate_scale=c["scale"])
    else:
        _plain_route(st)
    return {"idx": st["idx"], "gate": st["gate"]}


def _run_route_backward(st):
    c = st["case"]
    if own:
        import paper_2504_14960_amd as moe
        moe.router_select_backward(None, None, st["logits"], st["idx"], st["dgate"], st["dlogits"], None, None, None, None,
                                   score=moe.MOE_SCORE_SIGMOID if c["score"] == SIGMOID else moe.MOE_SCORE_SOFTMAX,
                                   renormalize=c["renormalize"], gate_scale=c["scale"])
    else:
        _plain_route_backward(st)
    return st["dlogits"]


def _run_bias_update(st):
    if own:
        import paper_2504_14960_amd as moe
        moe.router_bias_update(st["counts"], RATE, st["bias"], st["ws"])
    else:
        n = st["counts"].sum(0)
        st["bias"] += RATE * torch.sign(n.sum() - n * len(n)).float()
    return st["bias"]


def _run_weights(st):
    o = st["out"]
    if own:
        import paper_2504_14960_amd as moe
        moe.expert_weights_fp8_block(st["w_gate"], st["w_up"], st["w_down"], o["gate"], o["gate_scales"], o["up"],
                                     o["up_scales"], o["down"], o["down_scales"], o["gate_up_t"], o["gate_up_t_scales"],
                                     o["down_t"], o["down_t_scales"])
    else:
        F = st["case"]["F"]
        for name in ("gate", "up", "down"):
            _quantize_square(st["w_" + name], o[name], o[name + "_scales"])
        o["gate_up_t"][:, :, :F], o["gate_up_t"][:, :, F:] = o["gate"].transpose(1, 2), o["up"].transpose(1, 2)
        o["down_t"].copy_(o["down"].transpose(1, 2))
        n = F // BLOCK
        for to, a, name in ((0, n, "gate"), (n, n, "up")):
            _bytes(o["gate_up_t_scales"])[:, :, to:to + a] = _bytes(o[name + "_scales"])[:, :, :st["case"]["H"] // BLOCK].transpose(1, 2)
        _bytes(o["down_t_scales"])[:, :, :st["case"]["H"] // BLOCK] = _bytes(o["down_scales"])[:, :, :n].transpose(1, 2)
    return o


def _run_ffn(st):
    o, c = st["out"], st["case"]
    if own:
        import paper_2504_14960_amd as moe
        counts, offsets, row_of_assign, assign_of_row = st["maps"]
        moe.permute_fp8_block(st["x"], st["idx"], c["E"], 0, o["x"], o["x_scales"], counts, offsets, row_of_assign,
                              assign_of_row, st["ws"])
        moe.grouped_gemm_swiglu_fp8_block(o["x"], o["x_scales"], offsets, *st["w_gate"], *st["w_up"], *st["w_down"], o["h"],
                                          o["h_scales"], o.get("gu"), o["y"])
    else:
        _plain_ffn(st)
    return o


def _run_ffn_backward(st):
    o = st["out"]
    if own:
        import paper_2504_14960_amd as moe
        moe.grouped_gemm_swiglu_fp8_block_backward(*st["xq"], *st["hq"], st["gu"], st["dy"], st["offsets"], *st["wgu_t"],
                                                   *st["wd_t"], o["dx"], o["dw_gate"], o["dw_up"], o["dw_down"], st["ws"])
    else:
        _plain_ffn_backward(st)
    return o


_RUN = dict(route=_run_route, route_backward=_run_route_backward, bias_update=_run_bias_update, weights=_run_weights,
            ffn=_run_ffn, ffn_backward=_run_ffn_backward)


# ---------------------------------------------------------------------------------------------------------------
# the plain forms

def _scores(logits, score):
    """Scores of the experts a token may take, 0 for the others, in 64 bits: rounding decides what comes first."""
    x = logits.double()
    open_ = x > -math.inf                                  # neither -inf nor NaN
    if score == SIGMOID:
        p = 1 / (1 + torch.exp(-x))
    else:
        p = torch.exp(x - torch.where(open_, x, -math.inf).amax(1, keepdim=True).clamp(min=-1e30))
        p = p / torch.where(open_, p, 0).sum(1, keepdim=True).clamp(min=1e-300)
    return torch.where(open_, p, 0), open_


def _first(keys, n):
    """The n largest keys of every row and where they are, the lowest place first among equal ones."""
    v, i = torch.sort(keys, dim=1, descending=True, stable=True)
    return v[:, :n], i[:, :n]


def _choose(score32, open_, bias, c):
    """Selected experts of every token, -1 where none is left."""
    T, E = score32.shape
    key = score32 if bias is None else score32 + bias
    key = torch.where(open_, key, -math.inf)
    if c["groups"] > 1:
        g = key.view(T, c["groups"], -1)
        best = torch.sort(g, dim=2, descending=True).values[:, :, :min(c["group_best"], g.shape[2])]
        total = torch.where(best > -math.inf, best, 0).sum(2)
        total = torch.where(best[:, :, 0] > -math.inf, total, -math.inf)
        keep = torch.zeros_like(total, dtype=torch.bool).scatter_(1, _first(total, c["topk_groups"])[1], True)
        key = torch.where(keep[:, :, None], g, -math.inf).view(T, E)
    v, i = _first(key, c["K"])
    return torch.where(v > -math.inf, i, -1)


def _plain_route(st):
    c = st["case"]
    s, open_ = _scores(st["logits"], c["score"])
    s = s.float()
    i = _choose(s, open_, st["bias"], c)
    st["idx"].copy_(i)
    g = torch.where(i >= 0, s.gather(1, i.clamp(min=0)), 0)
    if c["renormalize"]:
        g = g / g.sum(1, keepdim=True).clamp(min=2.0 ** -149)
    st["gate"].copy_(g * c["scale"])


def _plain_route_backward(st):
    c = st["case"]
    p, _ = _scores(st["logits"], c["score"])
    p = p.float()
    i, has = st["idx"].long().clamp(min=0), st["idx"] >= 0
    s = torch.where(has, p.gather(1, i), 0)
    d = torch.where(has, st["dgate"], 0) * c["scale"]
    if c["renormalize"]:
        total = s.sum(1, keepdim=True)
        d = torch.where(has & (total > 0), (d - (d * s).sum(1, keepdim=True) / total) / total, 0)
    out = st["dlogits"].zero_()
    if c["score"] == SIGMOID:
        rest = 1 / (1 + torch.exp(st["logits"].gather(1, i)))
        out.scatter_add_(1, i, torch.where(has, d * s * rest, 0))
    else:
        out.scatter_add_(1, i, d * s).sub_(p * (d * s).sum(1, keepdim=True))


def _bytes(t):
    return t.view(torch.uint8)


def _scale_bytes(top):
    """The smallest power of two, from 2^-126, that leaves at most 448 of these largest values, as E8M0."""
    return torch.clamp(((top.view(torch.int32) + 0x1fffff) >> 23) - 8, min=1)


def _power(b, inverse=False):
    return ((254 - b if inverse else b).to(torch.int32) << 23).view(torch.float32)


def _quantize_rows(x, codes, scales):
    """Blocks of 128 along the rows of x, in 32 bits."""
    R, C = x.shape
    v = x.float().view(R, -1, BLOCK)
    b = _scale_bytes(v.abs().amax(2))
    codes.copy_((v * _power(b, True)[:, :, None]).view(R, C))
    _bytes(scales)[:, :C // BLOCK] = b.to(torch.uint8)


def _quantize_square(w, codes, scales):
    """Blocks of 128 x 128 of every expert's w."""
    E, N, K = w.shape
    v = w.float().view(E, N // BLOCK, BLOCK, K // BLOCK, BLOCK)
    b = _scale_bytes(v.abs().amax((2, 4)))
    codes.copy_((v * _power(b, True)[:, :, None, :, None]).view(E, N, K))
    _bytes(scales)[:, :, :K // BLOCK] = b.to(torch.uint8)


def _rows(codes, scales):
    R, C = codes.shape
    b = _bytes(scales)[:, :C // BLOCK]
    return (codes.float().view(R, -1, BLOCK) * _power(b)[:, :, None]).view(R, C)


def _square(codes, scales):
    N, K = codes.shape
    b = _bytes(scales)[:, :K // BLOCK]
    return (codes.float().view(N // BLOCK, BLOCK, K // BLOCK, BLOCK) * _power(b)[:, None, :, None]).view(N, K)


def _silu(g):
    return g / (1 + torch.exp(-g))


def _experts(st):
    """The experts with rows, as (expert, their rows)."""
    at = 0
    for e, n in enumerate(st["rows"]):
        if n:
            yield e, slice(at, at + n)
        at += n


def _plain_ffn(st):
    o, c = st["out"], st["case"]
    _quantize_rows(st["x"][st["order"] // c["K"]], o["x"], o["x_scales"])
    for e, r in _experts(st):
        x = _rows(o["x"][r], o["x_scales"][r])
        g, u = (x @ _square(w[0][e], w[1][e]).T for w in (st["w_gate"], st["w_up"]))
        if c["save"]:
            o["gu"][r] = torch.cat([g, u], 1).to(torch.bfloat16)
        _quantize_rows(_silu(g) * u, o["h"][r], o["h_scales"][r])
        o["y"][r] = (_rows(o["h"][r], o["h_scales"][r]) @ _square(st["w_down"][0][e], st["w_down"][1][e]).T).to(torch.bfloat16)


def _quantized(x):
    """x as its codes and scales have it."""
    codes, scales = _codes(*x.shape), _scales(*x.shape)
    _quantize_rows(x, codes, scales)
    return _rows(codes, scales)


def _plain_ffn_backward(st):
    o, F = st["out"], st["case"]["F"]
    for name in ("dw_gate", "dw_up", "dw_down"):
        o[name].zero_()
    for e, r in _experts(st):
        dy, x, h = st["dy"][r].float(), _rows(*(t[r] for t in st["xq"])), _rows(*(t[r] for t in st["hq"]))
        g, u = st["gu"][r, :F].float(), st["gu"][r, F:].float()
        dh = _quantized(dy) @ _square(st["wd_t"][0][e], st["wd_t"][1][e]).T
        s = 1 / (1 + torch.exp(-g))
        d = torch.cat([dh * u * s * (1 + g * (1 - s)), dh * g * s], 1)
        o["dx"][r] = (_quantized(d) @ _square(st["wgu_t"][0][e], st["wgu_t"][1][e]).T).to(torch.bfloat16)
        o["dw_down"][e] = (dy.T @ h).to(torch.bfloat16)
        dw = (d.T @ x).to(torch.bfloat16)
        o["dw_gate"][e], o["dw_up"][e] = dw[:F], dw[F:]


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"route": _exact_route, "route_backward": _exact_route_backward, "bias_update": _exact_bias,
            "weights": _exact_weights, "ffn": _exact_ffn, "ffn_backward": _exact_ffn_backward}[case["kind"]](st)


def _exact_scores(st):
    x = torch.nan_to_num(st["logits"].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    p = torch.sigmoid(x) if st["case"]["score"] == SIGMOID else torch.nan_to_num(torch.softmax(x, 1), nan=0.0)
    return p, x


def _exact_route(st):
    c = st["case"]
    p, x = _exact_scores(st)
    i = _choose(p.float(), x > -math.inf, st["bias"], c)
    g = p.gather(1, i.clamp(min=0)) * (i >= 0)
    if c["renormalize"]:
        g = torch.nan_to_num(g / g.sum(1, keepdim=True), nan=0.0)
    return {"idx": None, "gate": g * c["scale"]}


def _exact_route_backward(st):
    """By torch's own derivative of the gates."""
    c = st["case"]
    has = st["idx"] >= 0
    rows = has.any(1).nonzero()[:, 0]
    out = torch.zeros(st["logits"].shape, dtype=torch.float64, device="cuda")
    with torch.enable_grad():
        x = st["logits"][rows].double().requires_grad_()
        p = torch.sigmoid(x) if c["score"] == SIGMOID else torch.softmax(x, 1)
        g = p.gather(1, st["idx"][rows].long().clamp(min=0)) * has[rows]
        if c["renormalize"]:
            g = g / g.sum(1, keepdim=True)
        (g * c["scale"] * has[rows] * st["dgate"][rows].double()).sum().backward()
    out[rows] = x.grad
    return out


def _exact_bias(st):
    n = st["counts"].sum(0).double()
    return st["bias"].double() + RATE * torch.sign(n.mean() - n)


def _exact_power(top):
    return torch.exp2(torch.ceil(torch.log2(top.double().clamp(min=2.0 ** -126) / 448)).clamp(min=-126))


def _exact_to_8bit(v, scale):
    """The nearest of E4M3's values: four significant bits down to 2^-6, steps of 2^-9 below."""
    y = v / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_rows(x):
    """Codes' values, the scales with their padding, and the product of the two."""
    R, C = x.shape
    v = x.double().view(R, -1, BLOCK)
    scale = _exact_power(v.abs().amax(2))
    codes = _exact_to_8bit(v, scale[:, :, None])
    full = torch.full((R, _stride(C)), 2.0 ** -127, dtype=torch.float64, device="cuda")
    full[:, :C // BLOCK] = scale
    return codes.view(R, C), full, (codes * scale[:, :, None]).view(R, C)


def _exact_weights(st):
    out = {}
    for name in ("gate", "up", "down"):
        w = st["w_" + name].double()
        E, N, K = w.shape
        v = w.view(E, N // BLOCK, BLOCK, K // BLOCK, BLOCK)
        scale = _exact_power(v.abs().amax((2, 4)))
        out[name] = _exact_to_8bit(v, scale[:, :, None, :, None]).view(E, N, K)
        out[name + "_scale"] = scale

    def padded(s):
        full = torch.full(s.shape[:2] + (_stride(s.shape[2] * BLOCK),), 2.0 ** -127, dtype=torch.float64, device="cuda")
        full[:, :, :s.shape[2]] = s
        return full

    def t(name):
        return out[name].transpose(1, 2)
    return {"gate": out["gate"], "up": out["up"], "down": out["down"], "gate_up_t": torch.cat([t("gate"), t("up")], 2),
            "down_t": t("down").contiguous(), "gate_scales": padded(out["gate_scale"]), "up_scales": padded(out["up_scale"]),
            "down_scales": padded(out["down_scale"]), "down_t_scales": padded(t("down_scale")),
            "gate_up_t_scales": padded(torch.cat([t("gate_scale"), t("up_scale")], 2))}


def _exact_square(w, e):
    codes, scales = w[0][e], w[1][e]
    N, K = codes.shape
    s = scales.double()[:, :K // BLOCK]
    return codes.double() * s.repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)


def _exact_ffn(st):
    c = st["case"]
    token = st["order"] // c["K"]
    codes, scales, x = _exact_rows(st["x"][token])
    out = {"x": codes, "x_scales": scales, "h": torch.zeros(st["out"]["h"].shape, dtype=torch.float64, device="cuda"),
           "h_scales": torch.zeros(st["out"]["h_scales"].shape, dtype=torch.float64, device="cuda"),
           "y": torch.zeros(st["out"]["y"].shape, dtype=torch.float64, device="cuda")}
    if c["save"]:
        out["gu"] = torch.zeros(st["out"]["gu"].shape, dtype=torch.float64, device="cuda")
    for e, r in _experts(st):
        g, u = x[r] @ _exact_square(st["w_gate"], e).T, x[r] @ _exact_square(st["w_up"], e).T
        if c["save"]:
            out["gu"][r] = torch.cat([g, u], 1)
        out["h"][r], out["h_scales"][r], h = _exact_rows(g * torch.sigmoid(g) * u)
        out["y"][r] = h @ _exact_square(st["w_down"], e).T
    return out


def _exact_ffn_backward(st):
    F = st["case"]["F"]
    out = {k: torch.zeros(v.shape, dtype=torch.float64, device="cuda") for k, v in st["out"].items()}

    def values(q, r):
        return q[0][r].double() * q[1][r].double()[:, :q[0].shape[1] // BLOCK].repeat_interleave(BLOCK, 1)
    for e, r in _experts(st):
        dy, g, u = st["dy"][r].double(), st["gu"][r, :F].double(), st["gu"][r, F:].double()
        dh = _exact_rows(dy)[2] @ _exact_square(st["wd_t"], e).T
        with torch.enable_grad():
            g.requires_grad_(), u.requires_grad_()
            (g * torch.sigmoid(g) * u).backward(dh)
        d = torch.cat([g.grad, u.grad], 1)
        out["dx"][r] = _exact_rows(d)[2] @ _exact_square(st["wgu_t"], e).T
        out["dw_down"][e] = dy.T @ values(st["hq"], r)
        dw = d.T @ values(st["xq"], r)
        out["dw_gate"][e], out["dw_up"][e] = dw[:F], dw[F:]
    return out
