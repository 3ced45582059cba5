"""Performance cases of the operators of a served layer: 8-bit integer products and routed experts.

Operators
  int8      Y = X W^T with W in 8-bit integers (a scale for each output channel) and X quantised by token in the call
  grouped   the experts' products: rows sorted by expert, each group times its expert's matrix, bf16 or 8-bit integers
  route     logits to chosen experts, weights, and the rows sorted by expert
  combine   the experts' outputs back to their tokens, weighted and summed

"gated": W holds the rows of a gate and then those of an up projection, and the result is silu(gate) * up.
Widths that are summed over (d_in) are multiples of 16, as those of models are; rows, outputs and experts are any number.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
INF = math.inf
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # generating one token: an attention projection of a 7B model, where latency counts
        {"name": "int8_one_token", "op": "int8", "m": 1, "d_out": 4096, "d_in": 4096, "gated": False, "x": "bf16", "y": "bf16", "smooth": False},
        # a handful of sequences through a small model's down projection, fp32 activations whose channels were smoothed
        {"name": "int8_few_tokens", "op": "int8", "m": 13, "d_out": 2048, "d_in": 5632, "gated": False, "x": "f32", "y": "f32", "smooth": True},
        # an odd chunk of a prompt through a 13B model's down projection
        {"name": "int8_chunk", "op": "int8", "m": 509, "d_out": 5120, "d_in": 13824, "gated": False, "x": "bf16", "y": "bf16", "smooth": True},
        # a long prompt through a 7B model's gate and up projections: the largest product
        {"name": "int8_prompt_gated", "op": "int8", "m": 8192, "d_out": 11008, "d_in": 4096, "gated": True, "x": "bf16", "y": "bf16", "smooth": False},
        # generating for 5 sequences, 2 of 8 experts each, 8-bit gate and up projections: most experts have one row or none
        {"name": "grouped_decode_int8", "op": "grouped", "tokens": 5, "k": 2, "experts": 8, "d_out": 5632, "d_in": 2048, "gated": True, "x": "int8", "y": "bf16"},
        # generating for 48 sequences, 6 of 64 small experts each, decoded bf16 weights
        {"name": "grouped_decode_bf16", "op": "grouped", "tokens": 48, "k": 6, "experts": 64, "d_out": 1408, "d_in": 2048, "gated": False, "x": "bf16", "y": "f32"},
        # a prompt over 8 large experts in 8 bits: groups of a few hundred to a few thousand rows
        {"name": "grouped_prompt_int8", "op": "grouped", "tokens": 4001, "k": 2, "experts": 8, "d_out": 11008, "d_in": 4096, "gated": True, "x": "int8", "y": "bf16"},
        # several prompts over 64 experts in bf16: uneven groups of about five hundred rows
        {"name": "grouped_prompt_bf16", "op": "grouped", "tokens": 4096, "k": 8, "experts": 64, "d_out": 2816, "d_in": 2048, "gated": True, "x": "bf16", "y": "bf16"},
        # the router while generating for 5 sequences: the smallest call of all
        {"name": "route_decode", "op": "route", "m": 5, "experts": 8, "k": 2, "x": "f32", "renormalise": True},
        # the router over long prompts and many experts, some experts closed and some tokens padding
        {"name": "route_prompt", "op": "route", "m": 16384, "experts": 256, "k": 8, "x": "bf16", "renormalise": False},
        # the end of a routed layer while generating
        {"name": "combine_decode", "op": "combine", "m": 5, "k": 2, "d": 4096, "x": "bf16"},
        # and over long prompts
        {"name": "combine_prompt", "op": "combine", "m": 8192, "k": 8, "d": 4096, "x": "bf16"},
    ]


_MOST_FLOPS, _MOST_WEIGHTS, _MOST_BYTES = 1.4e12, 700e6, 600e6


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, most):
    """The width of a layer: one of the models that the codec is measured on, or an odd multiple of 16."""
    return rng.choice([w for w in (2048, 4096, 5120, 5632, 11008, 13824) if w <= most]) if rng.random() < 0.5 else 16 * (2 * _log_int(rng, 16, most // 32) - 1)


def _outs(rng, most):
    return _width(rng, most) if rng.random() < 0.4 else _log_int(rng, 48, most) | 1


def draw(rng):
    op = rng.choice(["int8", "int8", "int8", "grouped", "grouped", "grouped", "route", "combine"])
    while True:
        if op == "route":
            experts = _log_int(rng, 4, 512)
            c = {"op": op, "m": _log_int(rng, 1, 32768), "experts": experts, "k": rng.randint(1, min(8, experts)),
                 "x": rng.choice(["bf16", "f32"]), "renormalise": rng.random() < 0.5}
            fits = work(c)["bytes"] <= 20e6
        elif op == "combine":
            c = {"op": op, "m": _log_int(rng, 1, 16384), "k": rng.randint(1, 8), "d": _outs(rng, 8192), "x": rng.choice(["bf16", "f32"])}
            fits = work(c)["bytes"] <= _MOST_BYTES
        elif op == "int8":
            c = {"op": op, "m": _log_int(rng, 1, 8192), "d_out": _outs(rng, 13824), "d_in": _width(rng, 13824),
                 "gated": rng.random() < 0.3, "x": rng.choice(["bf16", "bf16", "f32"]), "y": rng.choice(["bf16", "bf16", "f32"]),
                 "smooth": rng.random() < 0.4}
            fits = work(c)["flops"] <= _MOST_FLOPS
        else:
            experts = _log_int(rng, 2, 128)
            c = {"op": op, "tokens": _log_int(rng, 1, 8192), "k": rng.randint(1, min(8, experts)), "experts": experts,
                 "d_out": _outs(rng, 11008), "d_in": _width(rng, 8192), "gated": rng.random() < 0.4,
                 "x": rng.choice(["int8", "bf16"]), "y": rng.choice(["bf16", "bf16", "f32"])}
            size = experts * (2 if c["gated"] else 1) * c["d_out"] * c["d_in"] * (2 if c["x"] == "bf16" else 1)
            fits = size <= _MOST_WEIGHTS and work(c)["flops"] <= _MOST_FLOPS and work(c)["bytes"] <= _MOST_BYTES
        if fits:
            return c


def work(case):
    op, wide = case["op"], {"bf16": 2, "f32": 4, "int8": 1}
    if op == "route":
        m, k, n = case["m"], case["k"], case["experts"]
        return {"bytes": m * n * wide[case["x"]] + 16 * m * k + 4 * (n + 1), "flops": 0}
    if op == "combine":
        m, k, d = case["m"], case["k"], case["d"]
        return {"bytes": m * (k + 1) * d * wide[case["x"]] + 8 * m * k, "flops": 2 * m * k * d}
    outs = case["d_out"] * (2 if case["gated"] else 1)
    if op == "int8":
        m, d_in = case["m"], case["d_in"]
        return {"bytes": m * d_in * wide[case["x"]] + outs * (d_in + 4) + m * case["d_out"] * wide[case["y"]], "flops": 2 * m * outs * d_in}
    rows, d_in, w = case["tokens"] * case["k"], case["d_in"], wide[case["x"]]
    used = case["experts"] * (1 - (1 - case["k"] / case["experts"]) ** case["tokens"])   # experts with a row, were all alike
    return {"bytes": int(used * outs * d_in * w + case["tokens"] * d_in * w + rows * case["d_out"] * wide[case["y"]] + 4 * rows),
            "flops": 2 * rows * outs * d_in}


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _activations(gen, m, d, dtype):
    """Rows of different sizes, with a few channels that are far larger than the others."""
    x = torch.randn(m, d, generator=gen, device=DEV)
    gains = torch.exp(0.3 * torch.randn(d, generator=gen, device=DEV))
    gains = torch.where(torch.rand(d, generator=gen, device=DEV) < 0.01, 8 * gains, gains)
    sizes = torch.exp(0.5 * torch.randn(m, 1, generator=gen, device=DEV))
    return (x * gains * sizes).to(dtype), gains


def _codes(gen, *shape):
    return (torch.randn(*shape, generator=gen, device=DEV, dtype=torch.bfloat16) * 32).round().clamp(-127, 127).to(torch.int8)


def _logits(gen, m, n, dtype):
    """Some experts are liked more than others; of many, one in 32 is closed; of many tokens, one in 64 is padding."""
    x = torch.randn(m, n, generator=gen, device=DEV) + 0.7 * torch.randn(n, generator=gen, device=DEV)
    if n >= 64:
        x[:, 7::32] = -INF
    if m >= 64:
        x[5::64] = -INF
    return x.to(dtype)


def _sorted_by_expert(gen, tokens, n, k):
    """Offsets and rows of a routed batch, most liked experts first in number of rows."""
    liked = torch.randn(tokens, n, generator=gen, device=DEV) + 0.7 * torch.randn(n, generator=gen, device=DEV)
    chosen = liked.topk(k, dim=1).indices.reshape(-1)
    order = torch.argsort(chosen, stable=True)
    counts = torch.zeros(n, dtype=torch.int64, device=DEV).index_add_(0, chosen, torch.ones_like(chosen))
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return offsets.to(torch.int32), (order // k).to(torch.int32), offsets.tolist()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, s = case["op"], dict(case)
    if op == "route":
        s["logits"] = _logits(gen, case["m"], case["experts"], _TYPES[case["x"]])
    elif op == "combine":
        m, k = case["m"], case["k"]
        s["Y"] = torch.randn(m * k, case["d"], generator=gen, device=DEV).to(_TYPES[case["x"]])
        places = torch.randperm(m * k, generator=gen, device=DEV).to(torch.int32)
        if m >= 64:
            places.view(m, k)[5::64] = -1          # padding
        s["positions"] = places.view(m, k)
        s["weights"] = torch.softmax(torch.randn(m, k, generator=gen, device=DEV), dim=1)
    else:
        outs, d_in = case["d_out"] * (2 if case["gated"] else 1), case["d_in"]
        if op == "int8":
            s["X"], gains = _activations(gen, case["m"], d_in, _TYPES[case["x"]])
            s["col_scale"] = gains.rsqrt() if case["smooth"] else None
            s["W"] = _codes(gen, outs, d_in)
            s["w_scales"] = torch.exp(0.2 * torch.randn(outs, generator=gen, device=DEV)) / (32 * math.sqrt(d_in))
        else:
            n = case["experts"]
            s["offsets"], s["rows"], s["bounds"] = _sorted_by_expert(gen, case["tokens"], n, case["k"])
            if case["x"] == "int8":
                s["X"], s["W"] = _codes(gen, case["tokens"], d_in), _codes(gen, n, outs, d_in)
                s["x_scales"] = torch.exp(0.5 * torch.randn(case["tokens"], generator=gen, device=DEV)) / 32
                s["w_scales"] = torch.exp(0.2 * torch.randn(n, outs, generator=gen, device=DEV)) / (32 * math.sqrt(d_in))
            else:
                s["X"], _ = _activations(gen, case["tokens"], d_in, torch.bfloat16)
                s["W"] = torch.randn(n, outs, d_in, generator=gen, device=DEV, dtype=torch.bfloat16).mul_(1 / math.sqrt(d_in))
                s["x_scales"] = s["w_scales"] = None
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------


def _gate(y, gated):
    if not gated:
        return y
    g, u = y.chunk(2, dim=1)
    return g / (1 + torch.exp(-g)) * u


def _plain_int8(s):
    x = s["X"].float()
    if s["col_scale"] is not None:
        x = x * s["col_scale"]
    most = x.abs().amax(dim=1, keepdim=True)
    codes = torch.where(most > 0, torch.round(x * (torch.full_like(most, 127) / most)), 0)
    y = codes @ s["W"].float().T * (most / 127) * s["w_scales"]
    return _gate(y, s["gated"]).to(_TYPES[s["y"]])


def _plain_grouped(s):
    """One product for each expert that has rows: padded to one batch, uneven groups would cost many times their rows."""
    out = torch.empty(s["tokens"] * s["k"], s["d_out"], dtype=_TYPES[s["y"]], device=DEV)
    for e in range(s["experts"]):
        a, b = s["bounds"][e], s["bounds"][e + 1]
        if a == b:
            continue
        rows = s["rows"][a:b]
        y = s["X"][rows].float() @ s["W"][e].float().T
        if s["x_scales"] is not None:
            y = y * s["x_scales"][rows][:, None] * s["w_scales"][e]
        out[a:b] = _gate(y, s["gated"])
    return out


def _plain_route(s):
    k, n = s["k"], s["experts"]
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -INF, x)
    values, chosen = torch.sort(x, dim=1, descending=True, stable=True)
    p = torch.where(values > -INF, torch.exp(torch.where(values == values[:, :1], 0, values - values[:, :1])), 0)
    total = (p[:, :k] if s["renormalise"] else p).sum(dim=1, keepdim=True)
    valid = values[:, :k] > -INF
    experts = torch.where(valid, chosen[:, :k], -1)
    weights = torch.where(valid, p[:, :k] / total, 0)
    key = torch.where(valid, chosen[:, :k], n).reshape(-1)
    counts = torch.zeros(n + 1, dtype=torch.int64, device=key.device).index_add_(0, key, torch.ones_like(key))
    ends = counts.cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends[:n]])
    order = torch.argsort(key, stable=True)
    place = torch.arange(key.numel(), device=key.device)
    rows = torch.where(place < offsets[n], order // k, -1)
    positions = torch.empty_like(place).index_copy_(0, order, place).view_as(experts)
    return {"experts": experts.to(torch.int32), "weights": weights, "offsets": offsets.to(torch.int32), "rows": rows.to(torch.int32),
            "positions": torch.where(valid, positions, -1).to(torch.int32)}


def _plain_combine(s):
    at = s["positions"]
    y = s["Y"][at.clamp(min=0)].float() * s["weights"][:, :, None]
    return torch.where(at[:, :, None] >= 0, y, 0).sum(dim=1).to(_TYPES[s["x"]])


def _own(s):
    from paper_2605_26339_amd import qamw

    op = s["op"]
    if op == "int8":
        return qamw.int8_matmul(s["X"], s["W"], s["w_scales"], col_scale=s["col_scale"], gated=s["gated"], out_dtype=_TYPES[s["y"]])
    if op == "grouped":
        return qamw.grouped_matmul(s["X"], s["W"], s["offsets"], rows=s["rows"], x_scales=s["x_scales"], w_scales=s["w_scales"],
                                   gated=s["gated"], out_dtype=_TYPES[s["y"]])
    if op == "route":
        r = qamw.route(s["logits"], s["k"], renormalise=s["renormalise"])
        return {"experts": r.experts, "weights": r.weights, "offsets": r.offsets, "rows": r.rows, "positions": r.positions}
    return qamw.combine(s["Y"], s["positions"], s["weights"], out_dtype=_TYPES[s["x"]])


_PLAIN = {"int8": _plain_int8, "grouped": _plain_grouped, "route": _plain_route, "combine": _plain_combine}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------


def _scaled_sum(x, w, row_scale, out_scale, gated):
    """sum_j x_ij w_nj times both scales, gate and up apart, in 64 bits."""
    halves = []
    for part, scale in zip(w.chunk(2) if gated else (w,), out_scale.chunk(2) if gated else (out_scale,)):
        halves.append(torch.mm(x.double(), part.double().t().contiguous()) * torch.outer(row_scale.double(), scale.double()))
    return halves[0] * torch.sigmoid(halves[0]) * halves[1] if gated else halves[0]


def _exact_route(s):
    x, k, n, m = s["logits"].double().cpu(), s["k"], s["experts"], s["m"]
    logits = x.tolist()
    total = torch.exp(x - x.amax(dim=1, keepdim=True)).nan_to_num(0.0).sum(dim=1).tolist()
    weights = torch.zeros(m, k, dtype=torch.float64)
    for t, row in enumerate(logits):
        best = sorted((e for e in range(n) if row[e] > -INF), key=lambda e: (-row[e], e))[:k]
        if best:
            w = [math.exp(row[e] - row[best[0]]) for e in best]
            whole = math.fsum(w) if s["renormalise"] else total[t]
            weights[t, :len(best)] = torch.tensor([v / whole for v in w], dtype=torch.float64)
    return {"experts": None, "weights": weights, "offsets": None, "rows": None, "positions": None}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        return _exact_route(s)
    if op == "combine":
        out = torch.zeros(case["m"], case["d"], dtype=torch.float64, device=DEV)
        for j in range(case["k"]):
            at = s["positions"][:, j].long()
            has = (at >= 0).nonzero()[:, 0]
            out[has] += s["Y"].double()[at[has]] * s["weights"][has, j].double()[:, None]
        return out
    if op == "int8":
        v = s["X"].double() * (1.0 if s["col_scale"] is None else s["col_scale"].double())
        step = v.abs().amax(dim=1) / 127
        return _scaled_sum(torch.round(v / step[:, None]), s["W"], step, s["w_scales"], case["gated"])
    out = torch.empty(case["tokens"] * case["k"], case["d_out"], dtype=torch.float64, device=DEV)
    ones = torch.ones(s["W"].shape[1], device=DEV)
    for e, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if b > a:
            rows = s["rows"][a:b].long()
            scale = s["x_scales"][rows] if s["x_scales"] is not None else torch.ones(b - a, device=DEV)
            out[a:b] = _scaled_sum(s["X"][rows], s["W"][e], scale, ones if s["w_scales"] is None else s["w_scales"][e], case["gated"])
    return out
