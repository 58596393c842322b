"""The operators of rows that choose their weights, as measurable cases.

A token of a mixture of experts goes through k of E feed-forward weights, a row of a batch that many users share through the
low-rank adapter of its user.  The operators:

  route    router logits [tokens, experts]: the k experts of each token, their weights, and the entries (a token and one of its
           experts) laid out by expert: `order` holds the entries expert after expert, each expert's in their order, `offsets`
           where each expert begins, `place` where each entry went.  `count` < tokens: a padded batch, whose last tokens choose none
  experts  products of the entries' rows with the quantised weights of their experts, in that layout.  `gated`: the first product of a
           feed-forward block, which gathers the tokens' rows and ends in silu(gate) * up; else the last one, whose rows lie in order
  combine  the weighted sum of the k rows of each token, added to the token's residual
  adapt    out = base + factor * (x A^T) B^T with each row's own A and B; rows without an adapter keep their base
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16, "float32": torch.float32}
# members of the number format's family: the type of rows and parameters, bits of a code, fraction bits of the type, its range of scales
FORMATS = {"e0m4": (torch.float16, 4, 10, 2.0 ** -14, 65504.0), "e0m8": (torch.float16, 8, 10, 2.0 ** -14, 65504.0),
           "bf16": (torch.bfloat16, 4, 7, 2.0 ** -126, 3.3895313892515355e38)}


def route(name, tokens, experts, k, dtype="float16", scoring="softmax", renormalise=True, count=None):
    return {"name": name, "op": "route", "tokens": tokens, "experts": experts, "k": k, "dtype": dtype, "scoring": scoring,
            "renormalise": renormalise, "count": tokens if count is None else count}


def experts(name, tokens, experts, k, N, K, group=128, gated=True, format="e0m4"):
    return {"name": name, "op": "experts", "tokens": tokens, "experts": experts, "k": k, "N": N, "K": K, "group": group, "gated": gated,
            "format": format}


def combine(name, tokens, experts, k, N, dtype="float16"):
    return {"name": name, "op": "combine", "tokens": tokens, "experts": experts, "k": k, "N": N, "dtype": dtype}


def adapt(name, rows, adapters, rank, N, K, dtype="float16", requests=0):
    return {"name": name, "op": "adapt", "rows": rows, "adapters": adapters, "rank": rank, "N": N, "K": K, "dtype": dtype, "requests": requests}


def listed():
    return [
        # a single user's next token: latency counts
        route("route one token", 1, 64, 6),
        # a prompt's part through a router of many experts
        route("route 4096 tokens of 128", 4096, 128, 8, dtype="bfloat16"),
        # a single user's next token through many small experts
        experts("gate/up one token 128 small", 1, 128, 8, 1536, 2048),
        # a serving batch of 32 single tokens: most experts are read, for a row or two each; the finer groups
        experts("down b32 128 small g64", 32, 128, 8, 2048, 768, group=64, gated=False),
        # a serving batch on few experts of the 6B model's feed-forward size, in 8 bits, an odd number of tokens
        experts("gate/up b13 8 of 6B 8-bit", 13, 8, 2, 27392, 4096, format="e0m8"),
        # a bfloat16 prompt of ordinary, odd length
        experts("gate/up prompt 1001 bf16", 1001, 64, 6, 2816, 2048, format="bf16"),
        # a long prompt through many small experts
        experts("gate/up prompt 4096 128 small", 4096, 128, 8, 1536, 2048),
        # the same through few large ones, with the 6B model's feed-forward size
        experts("down prompt 4096 8 of 6B", 4096, 8, 2, 4096, 13696, gated=False),
        # the end of the block for a few users and for a prompt
        combine("combine b4", 4, 128, 8, 2048),
        combine("combine 4096 bf16", 4096, 128, 8, 2048, dtype="bfloat16"),
        # a serving batch: 64 users, 40 adapters, on the 6B model's qkv projection
        adapt("adapt b64 of 40", 64, 40, 16, 4608, 4096),
        # prompts of five users of different, odd lengths on the output projection
        adapt("adapt prompts 3001 bf16", 3001, 12, 64, 4096, 4096, dtype="bfloat16", requests=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    op = rng.choice(["route", "experts", "experts", "experts", "combine", "adapt", "adapt"])
    while True:
        tokens, k = _log_int(rng, 1, 8192), rng.choice([1, 2, 2, 4, 6, 8, 8])
        number = rng.choice([8, 8, 16, 60, 64, 128, 256])
        dtype = rng.choice(["float16", "bfloat16"])
        if op == "route":
            case = route("", 2 * tokens, number, k, rng.choice(["float16", "bfloat16", "float32"]), rng.choice(["softmax", "softmax", "sigmoid"]),
                         rng.random() < 0.7, rng.choice([None, rng.randint(0, 2 * tokens)]))
        elif op == "experts":
            format = rng.choice(["e0m4", "e0m4", "e0m4", "bf16", "e0m8"])
            group = rng.choice([64, 128, 128] if format == "e0m8" else [32, 64, 128, 128])
            gated = rng.random() < 0.5
            step = max(group, 64)
            K = step * _log_int(rng, 512 // step, 14336 // step)
            N = 64 * _log_int(rng, 8, 428) if gated else 8 * _log_int(rng, 64, 1800)
            case = experts("", tokens, number, k, N, K, group, gated, format)
            if number * N * K > 1.0e9:
                continue
        elif op == "combine":
            case = combine("", tokens, number, k, rng.choice([8, 8, 1]) * _log_int(rng, 64, 1000), dtype)
        else:
            rows = rng.choice([_log_int(rng, 1, 256), _log_int(rng, 257, 8192)])
            case = adapt("", rows, _log_int(rng, 1, 100), 8 * rng.choice([1, 2, 2, 3, 4, 8, 16]), 8 * _log_int(rng, 64, 3500), 8 * _log_int(rng, 64, 1800),
                         dtype, 0 if rows <= 256 else rng.randint(1, 12))
            if rows * case["N"] > 1.0e8:
                continue
        del case["name"]
        if _cost(case) <= most:
            return case


def _active(case):
    """Experts that at least one token chooses, on average, if all are equally liked."""
    return case["experts"] * (1.0 - (1.0 - case["k"] / case["experts"]) ** case["tokens"])


def work(case):
    op = case["op"]
    if op == "route":
        size = 4 if case["dtype"] == "float32" else 2
        n = case["tokens"] * case["k"]
        return {"bytes": case["tokens"] * case["experts"] * size + n * 8 + n * 8 + 4 * (case["experts"] + 1), "flops": 4 * case["tokens"] * case["experts"]}
    if op == "combine":
        n = case["tokens"] * case["k"]
        return {"bytes": 2 * case["N"] * (n + 2 * case["tokens"]) + 8 * n, "flops": 2 * n * case["N"]}
    if op == "adapt":
        rows, N, K, rank = case["rows"], case["N"], case["K"], case["rank"]
        used = case["requests"] or case["adapters"] * (1.0 - (1.0 - 1.0 / case["adapters"]) ** rows)
        return {"bytes": int(2 * rows * (K + 2 * N) + 2 * min(used, case["adapters"]) * rank * (N + K) + 4 * rows), "flops": 2 * rows * rank * (N + K)}
    n, N, K = case["tokens"] * case["k"], case["N"], case["K"]
    bits = FORMATS[case["format"]][1]
    weights = _active(case) * (N * K * bits // 8 + 4 * N * K // case["group"])
    return {"bytes": int(weights + 2 * (case["tokens"] if case["gated"] else n) * K + 2 * n * (N // 2 if case["gated"] else N) + 4 * n), "flops": 2 * n * N * K}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) + 29)
    return gen


def _logits(case, gen):
    """Some experts are liked more than others, by all tokens."""
    liked = torch.randn(case["experts"], generator=gen, device=DEVICE) * 0.5
    return torch.randn((case["tokens"], case["experts"]), generator=gen, device=DEVICE) * 1.5 + liked


def _choice(case, gen):
    """Each token's experts, int32 [tokens, k]."""
    return torch.topk(_logits(case, gen), case["k"], dim=-1).indices.int()


def _activations(rows, width, dtype, gen):
    """A channel in a hundred is an outlier."""
    x = torch.randn((rows, width), generator=gen, device=DEVICE)
    x[:, torch.randperm(width, generator=gen, device=DEVICE)[:max(1, width // 100)]] *= 10.0
    return x.to(dtype)


def _weights(case, gen):
    """One expert's weights [N, K]; called once for each, in order."""
    w = torch.randn((case["N"], case["K"]), generator=gen, device=DEVICE)
    return w.mul_(torch.rand((case["N"], 1), generator=gen, device=DEVICE).mul_(1.5).add_(0.5).mul_(case["K"] ** -0.5)).to(FORMATS[case["format"]][0])


def _adapters(case, gen):
    """(each row's adapter int32, -1 for none; A; B; factors): a tenth of the rows of a batch, or one request in six, has none."""
    rows, number, rank, dtype = case["rows"], case["adapters"], case["rank"], TYPES[case["dtype"]]
    if case["requests"]:
        ends = torch.rand(case["requests"] - 1, generator=gen, device=DEVICE).mul_(rows).long().sort().values
        request = torch.searchsorted(ends, torch.arange(rows, device=DEVICE), right=True)
        adapter = torch.randint(number, (case["requests"],), generator=gen, device=DEVICE)
        adapter[torch.rand(case["requests"], generator=gen, device=DEVICE) < 1.0 / 6.0] = -1
        index = adapter[request]
    else:
        index = torch.randint(number, (rows,), generator=gen, device=DEVICE)
        index[torch.rand(rows, generator=gen, device=DEVICE) < 0.1] = -1
    A = (torch.randn((number, rank, case["K"]), generator=gen, device=DEVICE) * case["K"] ** -0.5).to(dtype)
    B = (torch.randn((number, case["N"], rank), generator=gen, device=DEVICE) * 0.3).to(dtype)
    return index.int(), A, B, torch.rand(number, generator=gen, device=DEVICE) * 1.5 + 0.5


def _layout(index, number):
    """(offsets, order, place) of entries int32 [...] by their group, those of no group behind the last; integers."""
    flat = index.flatten().long()
    n = flat.numel()
    inside = (flat >= 0) & (flat < number)
    key = torch.where(inside, flat, number)
    order = torch.sort(key, stable=True).indices
    offsets = torch.zeros(number + 1, dtype=torch.int32, device=DEVICE)
    offsets[1:] = torch.cumsum(torch.bincount(key, minlength=number + 1)[:number], 0)
    place = torch.empty(n, dtype=torch.int64, device=DEVICE)
    place[order] = torch.arange(n, device=DEVICE)
    return offsets, order.int(), torch.where(inside, place, -1).int()


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    if own:
        import paper_2403_20041_amd as e0m4
    if case["op"] == "route":
        state["logits"] = _logits(case, gen).to(TYPES[case["dtype"]])
        state["count"] = torch.tensor([case["count"]], dtype=torch.int32, device=DEVICE)
        return state
    if case["op"] == "adapt":
        state["index"], state["A"], state["B"], state["factors"] = _adapters(case, gen)
        state["x"] = _activations(case["rows"], case["K"], TYPES[case["dtype"]], gen)
        state["base"] = torch.randn((case["rows"], case["N"]), generator=gen, device=DEVICE).to(TYPES[case["dtype"]])
        if own:
            state["plan"] = e0m4.e0m4_groups(state["index"], case["adapters"])
        else:
            offsets, state["order"], _ = _layout(state["index"], case["adapters"])
            state["offsets"] = offsets.tolist()
        return state
    chosen = _choice(case, gen)
    n = chosen.numel()
    if own:
        state["plan"] = e0m4.e0m4_groups(chosen, case["experts"])
    else:
        offsets, state["order"], state["place"] = _layout(chosen, case["experts"])
        state["offsets"] = offsets.tolist()
    if case["op"] == "combine":
        state["weights"] = torch.softmax(torch.randn((case["tokens"], case["k"]), generator=gen, device=DEVICE), -1)
        state["rows"] = torch.randn((n, case["N"]), generator=gen, device=DEVICE).to(TYPES[case["dtype"]])
        state["base"] = torch.randn((case["tokens"], case["N"]), generator=gen, device=DEVICE).to(TYPES[case["dtype"]])
        return state
    dtype = FORMATS[case["format"]][0]
    state["x"] = _activations(case["tokens"] if case["gated"] else n, case["K"], dtype, gen)
    if own:
        quantise = {"e0m4": e0m4.e0m4_quantize, "e0m8": e0m4.e0m8_quantize, "bf16": e0m4.e0m4_bf16_quantize}[case["format"]]
        state["codes"] = torch.stack([quantise(_weights(case, gen), case["group"])[0] for _ in range(case["experts"])])
    else:
        state["weights"] = [_quantised(_weights(case, gen), case["group"], case["format"]) for _ in range(case["experts"])]
    return state


# ---- plain form -----------------------------------------------------------------------------------------------------


def _quantised(w, group, format):
    """Codes [N, K] with scale and bias [N, K / group]; the format's own steps are in 32 bits, each rounded once (computed in 64)."""
    dtype, bits, fraction, least, largest = FORMATS[format]
    high = 4.0 - 2.0 ** (1 - fraction)
    w = w.double().unflatten(-1, (-1, group))
    low, top = w.amin(-1).clamp(max=0.0), w.amax(-1).clamp(min=0.0)
    scale = ((top - low).float().double() / (high - 2.0)).float().clamp(least, largest).to(dtype)
    bias = (2.0 - (low / scale.double()).float().double()).float().clamp(2.0, high).to(dtype)
    bias = (bias.view(torch.int16) & -(1 << (fraction - bits))).view(dtype)
    w = w.div_(scale.double().unsqueeze(-1)).float().add_(bias.float().unsqueeze(-1)).clamp_(2.0, high).to(dtype)
    y = (w.view(torch.int16) & ((1 << fraction) - 1)) >> (fraction - bits - 1)          # the code's bits, and the one below
    return ((y + 1) >> 1).clamp_(max=(1 << bits) - 1).to(torch.uint8).flatten(-2), scale, bias


def _values(codes, scale, bias, format):
    """What the codes stand for, in 16 bits: that is the format's definition."""
    dtype, bits = FORMATS[format][:2]
    w = 2.0 + codes.unflatten(-1, (scale.shape[-1], -1)).float() / float(1 << (bits - 1))
    return ((w - bias.float().unsqueeze(-1)) * scale.float().unsqueeze(-1)).to(dtype).flatten(-2)


def _plain_route(s):
    case = s["case"]
    logits = s["logits"].float()
    best = torch.sort(logits, dim=-1, descending=True, stable=True)
    chosen, top = best.indices[:, :case["k"]], best.values[:, :case["k"]]
    if case["scoring"] == "softmax":
        w = (top - best.values[:, :1]).exp()
        total = w.sum(-1, keepdim=True) if case["renormalise"] else (logits - best.values[:, :1]).exp().sum(-1, keepdim=True)
        w = w / total
    else:
        w = 1.0 / (1.0 + (-top).exp())
        if case["renormalise"]:
            w = w / w.sum(-1, keepdim=True)
    there = torch.arange(case["tokens"], device=DEVICE)[:, None] < s["count"]
    chosen = torch.where(there, chosen, -1).int()
    offsets, order, place = _layout(chosen, case["experts"])
    return {"experts": chosen, "weights": torch.where(there, w, 0.0), "offsets": offsets, "order": order, "place": place}


def _plain_experts(s):
    case = s["case"]
    n, N = s["order"].numel(), case["N"]
    out = torch.empty((n, N // 2 if case["gated"] else N), dtype=s["x"].dtype, device=DEVICE)
    for e in range(case["experts"]):
        lo, hi = s["offsets"][e], s["offsets"][e + 1]
        if lo == hi:
            continue
        x = s["x"][s["order"][lo:hi].long() // case["k"]] if case["gated"] else s["x"][lo:hi]
        a = torch.matmul(x.float(), _values(*s["weights"][e], case["format"]).float().t())
        if case["gated"]:
            gate, up = a[:, :N // 2], a[:, N // 2:]
            a = gate / (1.0 + (-gate).exp()) * up
        out[lo:hi] = a.to(out.dtype)
    return {"out": out}


def _plain_combine(s):
    rows = s["rows"][s["place"].long()].view(s["case"]["tokens"], s["case"]["k"], -1).float()
    return {"out": (s["base"].float() + (rows * s["weights"].unsqueeze(-1)).sum(1)).to(s["base"].dtype)}


def _plain_adapt(s):
    out = s["base"].clone()
    for a in range(s["case"]["adapters"]):
        lo, hi = s["offsets"][a], s["offsets"][a + 1]
        if lo == hi:
            continue
        rows = s["order"][lo:hi].long()
        h = torch.matmul(s["x"][rows].float(), s["A"][a].float().t())
        out[rows] = (s["base"][rows].float() + s["factors"][a] * torch.matmul(h, s["B"][a].float().t())).to(out.dtype)
    return {"out": out}


PLAIN = {"route": _plain_route, "experts": _plain_experts, "combine": _plain_combine, "adapt": _plain_adapt}


# ---- the framework's operators --------------------------------------------------------------------------------------


def _own_route(s):
    import paper_2403_20041_amd as e0m4

    case = s["case"]
    chosen, weights, plan = e0m4.e0m4_route(s["logits"], case["k"], scoring=e0m4.E0M4_ROUTE_SIGMOID if case["scoring"] == "sigmoid" else e0m4.E0M4_ROUTE_SOFTMAX,
                                            renormalise=case["renormalise"], count=s["count"])
    return {"experts": chosen, "weights": weights, "offsets": plan.offsets, "order": plan.order, "place": plan.place}


def _own_experts(s):
    import paper_2403_20041_amd as e0m4

    case = s["case"]
    call = {"e0m4": e0m4.e0m4_matmul_grouped, "e0m8": e0m4.e0m8_matmul_grouped, "bf16": e0m4.e0m4_bf16_matmul_grouped}[case["format"]]
    if case["gated"]:
        return {"out": call(s["x"], s["plan"], s["codes"], case["N"], case["K"], case["group"], share=case["k"], epilogue=e0m4.E0M4_EPILOGUE_SWIGLU)}
    return {"out": call(s["x"], s["plan"], s["codes"], case["N"], case["K"], case["group"])}


def _own_combine(s):
    import paper_2403_20041_amd as e0m4

    return {"out": e0m4.e0m4_combine(s["rows"], s["weights"], s["plan"], base=s["base"])}


def _own_adapt(s):
    import paper_2403_20041_amd as e0m4

    return {"out": e0m4.e0m4_lora(s["x"], s["plan"], s["A"], s["B"], factors=s["factors"], base=s["base"])}


OWN = {"route": _own_route, "experts": _own_experts, "combine": _own_combine, "adapt": _own_adapt}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---- 64 bits --------------------------------------------------------------------------------------------------------


def _stands_for(w, group, format):
    """The values in 64 bits that the format has for weights [N, K]: 2^bits levels in [2, 4), the group's range with 0 in it laid over
    them, the bias cut to a level.  What the format itself rounds is rounded here."""
    dtype, bits, fraction, least, largest = FORMATS[format]
    f32 = lambda t: t.to(torch.float32).to(torch.float64)  # noqa: E731
    narrow = lambda t: t.to(torch.float32).to(dtype).to(torch.float64)  # noqa: E731
    shape, levels, span = w.shape, 2.0 ** bits, 2.0 - 2.0 ** (1 - fraction)
    x = w.to(torch.float64).reshape(-1, group)
    bottom = torch.minimum(x.min(1, keepdim=True).values, torch.zeros_like(x[:, :1]))
    ceiling = torch.maximum(x.max(1, keepdim=True).values, torch.zeros_like(x[:, :1]))
    step = narrow(torch.clamp(f32(f32(ceiling - bottom) / span), least, largest))
    zero = narrow(torch.clamp(f32(2.0 - f32(bottom / step)), 2.0, 2.0 + span))
    zero = torch.floor(zero * (levels / 2.0)) / (levels / 2.0)
    image = narrow(torch.clamp(f32(f32(x / step) + zero), 2.0, 2.0 + span))
    level = torch.floor((image - 2.0) * levels)                              # one bit more than the code has, which rounds up
    level = torch.clamp(torch.floor((level + 1.0) / 2.0), max=levels - 1.0)
    return narrow((2.0 + level / (levels / 2.0) - zero) * step).reshape(shape)


def exact(case, seed):
    gen = _generator(seed)
    if case["op"] == "route":
        logits = _logits(case, gen).to(TYPES[case["dtype"]]).double()
        k, count, number = case["k"], case["count"], case["experts"]
        chosen = torch.full((case["tokens"], k), -1, dtype=torch.int32, device=DEVICE)
        weights = torch.zeros((case["tokens"], k), dtype=torch.float64, device=DEVICE)
        z = logits[:count]
        picked = torch.argsort(-z, dim=1, stable=True)[:, :k]
        chosen[:count] = picked.int()
        top = z.gather(1, picked)
        if case["scoring"] == "sigmoid":
            w = torch.sigmoid(top)
            w = w / w.sum(1, keepdim=True) if case["renormalise"] else w
        else:
            w = (top - (top if case["renormalise"] else z).logsumexp(1, keepdim=True)).exp()
        weights[:count] = w
        order, offsets, flat = [], [0], chosen.flatten()
        for e in range(number):
            order.append((flat == e).nonzero().flatten())
            offsets.append(offsets[-1] + order[-1].numel())
        order.append((flat < 0).nonzero().flatten())
        order = torch.cat(order)
        place = torch.full_like(flat, -1)
        place[order[:offsets[-1]]] = torch.arange(offsets[-1], dtype=torch.int32, device=DEVICE)
        return {"experts": chosen, "weights": weights, "offsets": torch.tensor(offsets, dtype=torch.int32, device=DEVICE), "order": order.int(),
                "place": place}
    if case["op"] == "adapt":
        index, A, B, factors = _adapters(case, gen)
        x = _activations(case["rows"], case["K"], TYPES[case["dtype"]], gen).double()
        out = torch.randn((case["rows"], case["N"]), generator=gen, device=DEVICE).to(TYPES[case["dtype"]]).double()
        for a in range(case["adapters"]):
            rows = (index == a).nonzero().flatten()
            if rows.numel():
                out[rows] += factors[a].double() * ((x[rows] @ A[a].double().T) @ B[a].double().T)
        return {"out": out}
    chosen = _choice(case, gen)
    flat = chosen.flatten()
    entries = [(flat == e).nonzero().flatten() for e in range(case["experts"])]
    if case["op"] == "combine":
        w = torch.softmax(torch.randn((case["tokens"], case["k"]), generator=gen, device=DEVICE), -1).double().flatten()
        rows = torch.randn((flat.numel(), case["N"]), generator=gen, device=DEVICE).to(TYPES[case["dtype"]])
        out = torch.randn((case["tokens"], case["N"]), generator=gen, device=DEVICE).to(TYPES[case["dtype"]]).double()
        at = 0
        for mine in entries:
            if mine.numel():
                out.index_add_(0, mine // case["k"], rows[at:at + mine.numel()].double() * w[mine, None])
                at += mine.numel()
        return {"out": out}
    n, N, K = flat.numel(), case["N"], case["K"]
    x = _activations(case["tokens"] if case["gated"] else n, K, FORMATS[case["format"]][0], gen)
    out = torch.empty((n, N // 2 if case["gated"] else N), dtype=torch.float64, device=DEVICE)
    at = 0
    for mine in entries:
        w = _weights(case, gen)
        if mine.numel():
            mine_x = (x[mine // case["k"]] if case["gated"] else x[at:at + mine.numel()]).double()
            a = mine_x @ _stands_for(w, case["group"], case["format"]).T
            if case["gated"]:
                a = torch.nn.functional.silu(a[:, :N // 2]) * a[:, N // 2:]
            out[at:at + mine.numel()] = a
            at += mine.numel()
    return {"out": out}
