"""What follows the layer's gradients in a training step, as a set of measurable cases: the router's balance loss with its
gradient, the norm of all gradients, and the AdamW step.

A case is a dict of plain values.  ``kind`` names the entry point a pass goes through:

* ``balance``   moe.balance_loss: per-expert counts, sums of probabilities, balance and z loss of a batch;
* ``balance_backward``  moe.balance_loss_backward: their gradient in the router's logits;
* ``norm``      moe.grad_norm: the norm of a list of gradients and the factor that clips it;
* ``adamw``     moe.adamw_step: one step over a list of tensors, with states in 32 bits or in 8.

Where ``own`` is false the same results come from elementary torch operations in 32 bits; ``exact`` has them in 64 bits.
Layer shapes are those of moe_inputs.configs, or generic.
"""
from __future__ import annotations

import math

import torch

own = False

BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 3e-4, 0.1
BALANCE_COEF, Z_COEF = 1e-2, 1e-3
BLOCK = 32           # elements of an 8-bit state that share one scale


def _balance(name, kind, T, E, K, **kw):
    return dict(name=name, kind=kind, **{**dict(T=T, E=E, K=K, sequences=1, masked=0.0, bias="none", add=False), **kw})


def _tensors(name, kind, layer, **kw):
    return dict(name=name, kind=kind, layer=layer, **{**dict(grad="bf16", count=0, numel=0), **kw})


def listed():
    return [
        # the parity configuration's router: latency of a small call
        _balance("balance_256", "balance", 256, 8, 2),
        # packed sequences of uneven lengths with padding, experts and tokens in odd numbers, the loss kept per sequence
        _balance("balance_packed_7777", "balance", 7777, 60, 4, sequences=23, masked=0.1, bias="normal"),
        # the token-drop configuration's micro-batch: many tokens on 64 experts, strongly skewed
        _balance("balance_32768", "balance", 32768, 64, 6, bias="zipf1.2"),
        # a long-context batch on the most experts a layer may have
        _balance("balance_262144", "balance", 262144, 256, 8, bias="normal"),
        # the gradients of the same: packed sequences added to the gates' gradient, the largest batch
        _balance("balance_back_packed_7777", "balance_backward", 7777, 60, 4, sequences=23, masked=0.1, bias="normal",
                 add=True),
        _balance("balance_back_262144", "balance_backward", 262144, 256, 8, bias="normal"),
        # gradients of many small tensors: routers, biases and norms of a model
        _tensors("norm_small", "norm", "small", grad="f32", count=60, numel=400_000),
        # the expert and router gradients of the token-drop configuration
        _tensors("norm_tokendrop", "norm", "tokendrop"),
        # fp32 weights with fp32 states in many odd sizes
        _tensors("adamw_small", "adamw", "small", grad="f32", count=60, numel=400_000, param="f32", state="f32"),
        # bf16 weights with fp32 masters and 8-bit states, a short list of odd sizes
        _tensors("adamw8_small", "adamw", "small", count=9, numel=3_000_001, param="master", state="8bit"),
        # bf16 weights with fp32 masters and states, one layer
        _tensors("adamw_tokendrop", "adamw", "tokendrop", param="master", state="f32"),
        # bf16 weights without masters and 8-bit states, the largest layer whose three copies leave room
        _tensors("adamw8_8x7b", "adamw", "mixtral8x7b", param="bf16", state="8bit"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: kinds in turn, tokens, elements and tensors over their logarithm, odd ones too."""
    kind = rng.choice(["balance", "balance_backward", "norm", "adamw", "adamw"])
    if kind.startswith("balance"):
        T = _log_int(rng, 1, 262144)
        E = rng.choice([4, 8, 16, 64, 128, 256, rng.randint(2, 256)])
        sequences = 1 if rng.random() < 0.5 else _log_int(rng, 1, min(T, 1024))
        return dict(kind=kind, T=T, E=E, K=rng.randint(1, min(E, 8)), sequences=sequences,
                    masked=rng.choice([0.0, 0.0, 0.1, 0.5]), bias=rng.choice(["none", "normal", "zipf1.2"]),
                    add=kind == "balance_backward" and rng.random() < 0.5)
    numel = _log_int(rng, 1000, 500_000_000)
    case = dict(kind=kind, layer="small", grad=rng.choice(["f32", "bf16"]), numel=numel,
                count=_log_int(rng, 1, min(400, numel // 250)))
    if kind == "adamw":
        case.update(param=rng.choice(["f32", "master", "bf16"]), state=rng.choice(["f32", "8bit"]))
    return case


# ---------------------------------------------------------------------------------------------------------------
# sizes

def _sizes(case):
    """Elements of every tensor of the list: a layer's (router, its bias, gate, up, down), or uneven ones."""
    if case["layer"] != "small":
        from moe_inputs import get_config
        c = get_config(case["layer"])
        return [c.E * c.H, c.E] + 3 * [c.E * c.H * c.F]
    n, total = case["count"], case["numel"]
    # uneven and odd, the same for every seed; about a tenth of them are vectors of a few hundred elements
    weight = [0.05 + ((37 * i + 11) % 101) / 101 if i % 10 else 0.0 for i in range(n)]
    if n == 1:
        return [total]
    return [max(1, int(total * w / sum(weight))) if w else 129 + 2 * i for i, w in enumerate(weight)]


def _starts(sizes):
    """Where the tensors start in one flat buffer: multiples of 64 elements, so that every piece is aligned."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += (n + 63) // 64 * 64
    return starts, at


def work(case):
    """Bytes and operations a pass cannot do without."""
    if case["kind"].startswith("balance"):
        T, E, K, S = (case[k] for k in ("T", "E", "K", "sequences"))
        mask = T if case["masked"] else 0
        if case["kind"] == "balance":
            return {"bytes": 4 * T * E + 4 * T * K + mask + 8 * S * E + 4 * S + 8, "flops": 6 * T * E}
        return {"bytes": (12 if case["add"] else 8) * T * E + mask + 4 * S * E + 4 * S, "flops": 10 * T * E}
    n = sum(_sizes(case))
    grad = 4 if case["grad"] == "f32" else 2
    if case["kind"] == "norm":
        return {"bytes": grad * n + 8, "flops": 2 * n}
    param = {"f32": 8, "master": 2 + 8, "bf16": 4}[case["param"]]
    state = 16 if case["state"] == "f32" else 4 + 4 / BLOCK
    return {"bytes": (grad + param + state) * n, "flops": 15 * n}


# ---------------------------------------------------------------------------------------------------------------
# inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["kind"].startswith("balance"):
        return _prepare_balance(case, gen)
    return _prepare_tensors(case, gen)


def _prepare_balance(case, gen):
    T, E, K, S = (case[k] for k in ("T", "E", "K", "sequences"))
    # logits of normalised tokens and the usual initialisation, and what tells the experts apart
    logits = torch.randn((T, E), generator=gen, device="cuda") * 1.5
    if case["bias"] == "normal":
        logits += torch.randn(E, generator=gen, device="cuda")
    elif case["bias"] == "zipf1.2":
        logits -= 1.2 * torch.log(torch.randperm(E, generator=gen, device="cuda") + 1.0)
    st = dict(case=case, logits=logits, idx=logits.topk(K, dim=1).indices.to(torch.int32), mask=None, offsets=None)
    if case["masked"]:
        keep = torch.rand(T, generator=gen, device="cuda") >= case["masked"]
        st["mask"] = keep.to(torch.uint8)
        logits[~keep] = float("nan")                     # padding holds whatever was there
    if S > 1:
        # the ends of sequences packed into one batch; some meet, which leaves a sequence without tokens
        ends = torch.sort(torch.randint(0, T + 1, (S - 1,), generator=gen, device="cuda")).values
        st["offsets"] = torch.cat([ends.new_zeros(1), ends, ends.new_full((1,), T)]).to(torch.int32)
    st["counts"] = torch.empty((S, E), dtype=torch.int32, device="cuda")
    st["prob_sums"] = torch.empty((S, E), dtype=torch.float32, device="cuda")
    st["seq_tokens"] = torch.empty((S + 1,), dtype=torch.int32, device="cuda")
    st["losses"] = torch.empty((2,), dtype=torch.float32, device="cuda")
    if case["kind"] == "balance_backward":
        st["counts"], st["seq_tokens"] = (t.to(torch.int32) for t in _count(st))
        st["dlosses"] = torch.rand(2, generator=gen, device="cuda") + 0.5
        # the gates' gradient, which the result is added to
        st["gates"] = torch.randn((T, E), generator=gen, device="cuda") * (1e-2 / T) if case["add"] else None
        st["dlogits"] = torch.empty((T, E), dtype=torch.float32, device="cuda")
    if own and case["kind"] == "balance":
        import paper_2504_14960_amd as moe
        st["ws"] = torch.empty(moe.balance_loss_workspace_bytes(T, E, S), dtype=torch.uint8, device="cuda")
    return st


def _prepare_tensors(case, gen):
    sizes = _sizes(case)
    starts, total = _starts(sizes)
    grad = torch.float32 if case["grad"] == "f32" else torch.bfloat16

    def normal(dtype, std):
        return torch.empty(total, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    # a gradient whose size differs from one run of 1024 elements to the next, as rows of a weight do
    rows = torch.exp(torch.randn((total + 1023) // 1024, generator=gen, device="cuda"))
    rows = rows.repeat_interleave(1024)[:total]
    st = dict(case=case, sizes=sizes, starts=starts, step=1000, seed=int(torch.randint(1 << 31, (1,), generator=gen, device="cuda")),
              grad=normal(grad, 1e-3).mul_(rows.to(grad)))
    if case["kind"] == "norm":
        st["out"] = torch.empty(2, dtype=torch.float32, device="cuda")
    else:
        st["scale"] = torch.rand(1, generator=gen, device="cuda") * 0.5 + 0.5
        st["param"] = normal(torch.float32, 0.02)
        st["master"] = None
        if case["param"] != "f32":
            if case["param"] == "master":
                st["master"] = st["param"]
            st["param"] = st["param"].to(torch.bfloat16)
        m, v = normal(torch.float32, 3e-4).mul_(rows), normal(torch.float32, 1e-3).mul_(rows).square_()
        st["scales"] = None
        if case["state"] == "8bit":
            sm, sv = (torch.full(((total + BLOCK - 1) // BLOCK,), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
            cm, cv = (torch.zeros(total, dtype=torch.uint8, device="cuda") for _ in range(2))
            for i, (n, a) in enumerate(zip(sizes, starts)):
                bits = _random_bits(n, st["seed"] ^ 0x5bd1, i)
                for src, code, scale, shift in ((m, cm, sm, 0), (v, cv, sv, 16)):
                    code[a:a + n], s = _to_8bit(src[a:a + n], (bits >> shift) & 0xffff, shift == 16)
                    scale[a // BLOCK:a // BLOCK + len(s)] = s
            m, v, st["scales"] = cm, cv, (sm, sv)
        st["m"], st["v"] = m, v
    del rows
    if own:
        import paper_2504_14960_amd as moe
        cut = [slice(a, a + n) for n, a in zip(sizes, starts)]
        blocks = [slice(a // BLOCK, a // BLOCK + (n + BLOCK - 1) // BLOCK) for n, a in zip(sizes, starts)]

        def pieces(t, at=cut):
            return None if t is None else [t[c] for c in at]

        if case["kind"] == "norm":
            st["list"] = moe.GradTensors(pieces(st["grad"]))
            st["ws"] = torch.empty(moe.grad_norm_workspace_bytes(len(sizes)), dtype=torch.uint8, device="cuda")
        else:
            sm, sv = st["scales"] or (None, None)
            st["list"] = moe.AdamWTensors(pieces(st["param"]), pieces(st["grad"]), pieces(st["m"]), pieces(st["v"]),
                                          masters=pieces(st["master"]), exp_avg_scales=pieces(sm, blocks),
                                          exp_avg_sq_scales=pieces(sv, blocks), weight_decays=_decays(sizes))
    return st


def _decays(sizes):
    """Small vectors (biases) are not decayed."""
    return [0.0 if n < 1024 else DECAY for n in sizes]


# ---------------------------------------------------------------------------------------------------------------
# one pass

def run(st):
    return _RUN[st["case"]["kind"]](st)


def _run_balance(st):
    if own:
        import paper_2504_14960_amd as moe
        moe.balance_loss(st["logits"], st["idx"], BALANCE_COEF, Z_COEF, st["counts"], st["prob_sums"], st["seq_tokens"],
                         st["losses"], st["ws"], token_mask=st["mask"], seq_offsets=st["offsets"])
    else:
        _plain_balance(st)
    return {k: st[k] for k in ("counts", "prob_sums", "seq_tokens", "losses")}


def _run_balance_backward(st):
    if own:
        import paper_2504_14960_amd as moe
        moe.balance_loss_backward(st["logits"], st["counts"], st["seq_tokens"], st["dlosses"], st["case"]["K"],
                                  BALANCE_COEF, Z_COEF, st["dlogits"], addend=st["gates"], token_mask=st["mask"],
                                  seq_offsets=st["offsets"])
    else:
        _plain_balance_backward(st)
    return st["dlogits"]


def _run_norm(st):
    if own:
        import paper_2504_14960_amd as moe
        moe.grad_norm(st["list"], st["out"], st["ws"], max_norm=1.0, multiplier=0.5)
    else:
        _plain_norm(st)
    return st["out"]


def _run_adamw(st):
    st["step"] += 1
    if own:
        import paper_2504_14960_amd as moe
        moe.adamw_step(st["list"], LR, BETA1, BETA2, EPS, st["step"], seed=st["seed"] + st["step"], grad_scale=st["scale"])
    else:
        _plain_adamw(st)
    out = {k: st[k] for k in ("param", "m", "v")}
    if st["master"] is not None:
        out["master"] = st["master"]
    if st["scales"] is not None:                         # 8 bits: as the values they stand for
        out["m"], out["v"] = (out[k].view(torch.float8_e4m3fn) for k in "mv")
        out["m_scale"], out["v_scale"] = (s.view(torch.float8_e8m0fnu) for s in st["scales"])
    return out


_RUN = dict(balance=_run_balance, balance_backward=_run_balance_backward, norm=_run_norm, adamw=_run_adamw)


# ---------------------------------------------------------------------------------------------------------------
# the plain forms, in 32 bits

def _sequence_of_token(st):
    if st["offsets"] is None:
        return torch.zeros(st["case"]["T"], dtype=torch.int64, device="cuda")
    at = torch.arange(st["case"]["T"], device="cuda")
    return torch.searchsorted(st["offsets"].long(), at, right=True) - 1


def _count(st):
    """Assignments of every sequence to every expert, and valid tokens of every sequence and of all."""
    c, seq = st["case"], _sequence_of_token(st)
    valid = torch.ones_like(seq) if st["mask"] is None else st["mask"].long()
    cell = (seq[:, None] * c["E"] + st["idx"]).flatten()
    counts = torch.zeros(c["sequences"] * c["E"], dtype=torch.int64, device="cuda")
    counts.index_add_(0, cell, valid[:, None].expand(-1, c["K"]).flatten())
    n = torch.zeros(c["sequences"], dtype=torch.int64, device="cuda").index_add_(0, seq, valid)
    return counts.view(c["sequences"], c["E"]), torch.cat([n, n.sum()[None]])


def _softmax(st):
    """Probabilities and log-sum-exp of every token; zeros for masked ones, whatever their logits hold."""
    x = st["logits"]
    if st["mask"] is not None:
        keep = st["mask"].bool()[:, None]
        x = torch.where(keep, x, torch.zeros_like(x))
    top = x.amax(1, keepdim=True)
    p = torch.exp(x - top)
    z = p.sum(1, keepdim=True)
    p = p / z
    lse = top + torch.log(z)
    if st["mask"] is not None:
        p, lse = p * keep, lse * keep
    return p, lse


def _plain_balance(st):
    c = st["case"]
    p, lse = _softmax(st)
    counts, n = _count(st)
    if st["offsets"] is None:
        sums = p.sum(0, keepdim=True)
    else:
        sums = torch.zeros((c["sequences"], c["E"]), device="cuda").index_add_(0, _sequence_of_token(st), p)
    all_tokens = n[-1].clamp(min=1).float()
    per_sequence = (counts.float() * sums).sum(1) / n[:-1].clamp(min=1).float()
    st["counts"].copy_(counts)
    st["prob_sums"].copy_(sums)
    st["seq_tokens"].copy_(n)
    st["losses"][0] = per_sequence.sum() * (BALANCE_COEF * c["E"] / c["K"]) / all_tokens
    st["losses"][1] = (lse * lse).sum() * Z_COEF / all_tokens


def _plain_balance_backward(st):
    c = st["case"]
    p, lse = _softmax(st)
    n = st["seq_tokens"]
    all_tokens = n[-1].clamp(min=1).float()
    g = st["counts"].float() / n[:-1, None].clamp(min=1).float() * (BALANCE_COEF * c["E"] / c["K"]) / all_tokens
    g = (g * st["dlosses"][0])[_sequence_of_token(st)]
    d = p * (g - (p * g).sum(1, keepdim=True)) + p * lse * (2 * Z_COEF / all_tokens * st["dlosses"][1])
    if st["gates"] is not None:
        d = d + st["gates"]
    st["dlogits"].copy_(d)


def _plain_norm(st):
    parts = [st["grad"][a:a + n].float().square().sum() for n, a in zip(st["sizes"], st["starts"])]
    norm = 0.5 * torch.sqrt(torch.stack(parts).sum())
    st["out"][0] = norm
    st["out"][1] = torch.where(torch.isfinite(norm), 0.5 * torch.clamp(1.0 / (norm + 1e-6), max=1.0), norm * float("nan"))


def _mix(x):
    """Two rounds of multiply and shift on 32-bit numbers held in 64."""
    x = x ^ (x >> 16)
    x = (x * 0x7feb352d) & 0xffffffff
    x = x ^ (x >> 15)
    x = (x * 0x846ca68b) & 0xffffffff
    return x ^ (x >> 16)


def _key(seed, tensor, high):
    x = (seed + 0x9e3779b9 * (tensor + 1) + 0x85ebca6b * high) & 0xffffffff
    return _mix(x)


def _random_bits(n, seed, tensor):
    """32 bits for every element of a tensor, from the seed, the tensor's place in the list and the element's in it."""
    assert n < 1 << 32
    return _mix(torch.arange(n, device="cuda") ^ _key(seed, tensor, 0))


def _by_block(x):
    n = len(x)
    pad = -n % BLOCK
    return (torch.cat([x, x.new_zeros(pad)]) if pad else x).view(-1, BLOCK)


def _to_8bit(x, bits16, keep_positive):
    """E4M3 codes and E8M0 scales of x, rounded up with the probability of the part cut off; ``keep_positive``: what is
    above zero stays there."""
    blocks = _by_block(x)
    top = blocks.abs().amax(1).view(torch.int32)
    scale = torch.clamp(((top + 0x1fffff) >> 23) - 8, min=1)      # the smallest power of two that leaves at most 448
    inverse = ((254 - scale) << 23).view(torch.float32)
    y = (blocks * inverse[:, None]).flatten()[:len(x)]
    a = y.abs()
    r = (bits16.to(torch.int32) << 4) | 8                         # 20 bits, in the middle of their step
    normal = ((a.view(torch.int32) + r) >> 20) - (120 << 3)
    small = ((a * 2.0 ** 29).to(torch.int32) + r) >> 20           # below 2^-6: steps of 2^-9
    code = torch.where(a >= 2.0 ** -6, normal, torch.where(a < 2.0 ** -6, small, 0x7f))
    if keep_positive:
        code = torch.where((code == 0) & (x > 0), 1, code)
    else:
        code = code | torch.where(torch.signbit(y), 0x80, 0)
    return code.to(torch.uint8), scale.to(torch.uint8)


def _from_8bit(code, scale):
    return code.view(torch.float8_e4m3fn).float() * scale.view(torch.float8_e8m0fnu).float().repeat_interleave(BLOCK)[:len(code)]


def _plain_adamw(st):
    decays = _decays(st["sizes"])
    for i, (n, a) in enumerate(zip(st["sizes"], st["starts"])):
        _plain_adamw_tensor(st, i, slice(a, a + n), slice(a // BLOCK, a // BLOCK + (n + BLOCK - 1) // BLOCK), decays[i])


def _plain_adamw_tensor(st, i, at, blocks, decay):
    t, case = st["step"], st["case"]
    g = st["grad"][at].float() * st["scale"]
    p = (st["param"] if st["master"] is None else st["master"])[at].float()
    m, v = st["m"][at], st["v"][at]
    bits = None
    if case["state"] == "8bit":
        m, v = _from_8bit(m, st["scales"][0][blocks]), _from_8bit(v, st["scales"][1][blocks])
    if case["state"] == "8bit" or case["param"] == "bf16":
        bits = _random_bits(at.stop - at.start, st["seed"] + t, i)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    denom = torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** t)) + EPS
    p = p * (1 - LR * decay) - (m / denom) * (LR / (1 - BETA1 ** t))
    if case["state"] == "8bit":
        st["m"][at], st["scales"][0][blocks] = _to_8bit(m, bits & 0xffff, False)
        st["v"][at], st["scales"][1][blocks] = _to_8bit(v, bits >> 16, True)
    else:
        st["m"][at], st["v"][at] = m, v
    if case["param"] == "bf16":                          # rounded up with the probability of the part cut off
        extra = ((bits * 0x9e3779b1) & 0xffffffff) >> 16
        st["param"][at] = ((p.view(torch.int32) + extra.to(torch.int32)) & -65536).view(torch.float32).to(torch.bfloat16)
    else:
        if st["master"] is not None:
            st["master"][at] = p
        st["param"][at] = p.to(st["param"].dtype)


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"balance": _exact_balance, "balance_backward": _exact_balance_backward, "norm": _exact_norm,
            "adamw": _exact_adamw}[case["kind"]](st)


def _exact_tokens(st):
    """Log-probabilities, lse and the sequence of the tokens that count, as (rows, logp, lse, sequence)."""
    rows = torch.arange(st["case"]["T"], device="cuda") if st["mask"] is None else st["mask"].nonzero()[:, 0]
    x = st["logits"][rows].double()
    lse = torch.logsumexp(x, dim=1)
    if st["offsets"] is None:
        seq = torch.zeros_like(rows)
    else:
        seq = (rows[:, None] >= st["offsets"][None, 1:-1]).sum(1) if len(rows) * len(st["offsets"]) < 1 << 28 else \
            torch.bucketize(rows, st["offsets"][1:-1].long(), right=True)
    return rows, x - lse[:, None], lse, seq


def _exact_counts(st, rows, seq):
    S, E = st["case"]["sequences"], st["case"]["E"]
    counts = torch.bincount((seq[:, None] * E + st["idx"][rows].long()).flatten(), minlength=S * E).view(S, E)
    return counts, torch.bincount(seq, minlength=S)


def _exact_balance(st):
    c = st["case"]
    rows, logp, lse, seq = _exact_tokens(st)
    counts, n = _exact_counts(st, rows, seq)
    order = torch.cumsum(n, 0)
    total = torch.cat([logp.new_zeros(1, c["E"]), torch.cumsum(torch.exp(logp), 0)])   # tokens lie in order of their sequence
    sums = total[order] - total[order - n]
    losses = logp.new_zeros(2)
    if len(rows):
        has = n > 0
        losses[0] = BALANCE_COEF * c["E"] / (c["K"] * len(rows)) * ((counts[has] * sums[has]).sum(1) / n[has]).sum()
        losses[1] = Z_COEF * (lse ** 2).mean()
    return {"counts": None, "prob_sums": sums, "seq_tokens": None, "losses": losses}


def _exact_balance_backward(st):
    c = st["case"]
    rows, logp, lse, seq = _exact_tokens(st)
    counts, n = _exact_counts(st, rows, seq)
    d = torch.zeros((c["T"], c["E"]), dtype=torch.float64, device="cuda")
    if len(rows):
        db, dz = st["dlosses"].double()
        p = torch.exp(logp)
        g = (db * BALANCE_COEF * c["E"] / (c["K"] * len(rows)) * counts / n.clamp(min=1)[:, None])[seq]
        d[rows] = p * (g - (p * g).sum(1, keepdim=True) + (dz * 2 * Z_COEF / len(rows) * lse)[:, None])
    return d if st["gates"] is None else d + st["gates"].double()


def _exact_norm(st):
    sq = sum(st["grad"][a:a + n].double().pow(2).sum() for n, a in zip(st["sizes"], st["starts"]))
    norm = 0.5 * sq.sqrt()
    return torch.stack([norm, 0.5 * torch.clamp(1 / (norm + 1e-6), max=1)])


def _exact_8bit(x, uniform, floor):
    """Values of codes and of scales for x, from the format's definition: four significant bits down to 2^-6, steps of
    2^-9 below, a scale 2^k with the largest of a block at most 448 * 2^k."""
    pad = torch.cat([x, x.new_zeros(-len(x) % BLOCK)]).view(-1, BLOCK)
    k = torch.ceil(torch.log2(pad.abs().amax(1).clamp(min=2.0 ** -126) / 448)).clamp(min=-126)
    y = (pad / torch.exp2(k)[:, None]).flatten()[:len(x)]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    q = torch.floor(y.abs() / step + uniform) * step
    if floor:
        q = torch.where((q == 0) & (x > 0), 2.0 ** -9, q)
    return torch.copysign(q, y), torch.exp2(k)


def _exact_adamw(st):
    t, case = st["step"] + 1, st["case"]
    out = {k: st[k].double() if st[k].is_floating_point() else st[k].view(torch.float8_e4m3fn).double()
           for k in ("param", "m", "v")}
    if st["master"] is not None:
        out["master"] = st["master"].double()
    if st["scales"] is not None:
        out["m_scale"], out["v_scale"] = (s.view(torch.float8_e8m0fnu).double() for s in st["scales"])
    for i, (n, a) in enumerate(zip(st["sizes"], st["starts"])):
        at, blocks = slice(a, a + n), slice(a // BLOCK, a // BLOCK + (n + BLOCK - 1) // BLOCK)
        g = st["grad"][at].double() * st["scale"].double()
        m, v = out["m"][at], out["v"][at]
        if st["scales"] is not None:
            m = m * out["m_scale"][blocks].repeat_interleave(BLOCK)[:n]
            v = v * out["v_scale"][blocks].repeat_interleave(BLOCK)[:n]
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
        p = out["master" if st["master"] is not None else "param"][at]
        p = p * (1 - LR * _decays(st["sizes"])[i]) - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
        if st["scales"] is not None:
            bits = _random_bits(n, st["seed"] + t, i)
            for name, x, shift in (("m", m, 0), ("v", v, 16)):
                u = (((bits >> shift) & 0xffff).double() + 0.5) / 65536
                out[name][at], out[name + "_scale"][blocks] = _exact_8bit(x, u, name == "v")
        else:
            out["m"][at], out["v"][at] = m, v
        if st["master"] is not None:
            out["master"][at] = p
        out["param"][at] = p
    return out
