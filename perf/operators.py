"""The operators around a key/value cache that is held in 4 bits, as measurable cases.

The cache keeps the keys and values of a decoder's past tokens as E0M4 codes with a scale and a bias for each group of
`group` values along the head dimension.  Three operators work on it:

  append   new rows of keys and values are quantised into the cache (the case returns them read back, as the values that
           their codes stand for)
  attend   attention of the newest tokens' queries over the cache: grouped heads, causal or not, a sliding window, a mask,
           and, where `weights` is set, the sum over queries and heads of the attention that each cached row received,
           added to what it received before
  evict    the rows that received the least attention leave the cache, the newest `recent` ones stay; the remaining rows
           keep their order

`length` is the number of rows of the longest sequence after the append; in a batch the sequences end at different lengths.
`new` is the number of tokens that a sequence adds (its queries); in a batch of prompts they are of different numbers too.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16}
LOW, HIGH = 2.0, 4.0 - 2.0 ** -9        # the binade of the codes' values
MOST = 57344.0                          # larger magnitudes are stored as this one


def append(name, batch, kv_heads, dim, group, new, past, dtype="float16"):
    return {"name": name, "op": "append", "dtype": dtype, "batch": batch, "heads": kv_heads, "kv_heads": kv_heads, "dim": dim,
            "group": group, "new": new, "length": past + new}


def attend(name, batch, heads, kv_heads, dim, group, new, past, dtype="float16", causal=True, window=0, mask=False, weights=False):
    return {"name": name, "op": "attend", "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "group": group, "new": new, "length": past + new, "causal": causal, "window": window, "mask": mask, "weights": weights}


def evict(name, batch, kv_heads, dim, group, length, budget, recent):
    return {"name": name, "op": "evict", "dtype": "float16", "batch": batch, "heads": kv_heads, "kv_heads": kv_heads, "dim": dim,
            "group": group, "new": 0, "length": length, "budget": budget, "recent": recent}


def listed():
    return [
        # the smallest call: the one new token of a single user's chat with the 6B model (32 heads on 2 of keys and values)
        append("append 6B one token", 1, 2, 128, 128, 1, 700),
        # two users' prompts on the 14B model (40 heads of keys and values), the finer groups
        append("append 14B two prompts", 2, 40, 128, 64, 2048, 0),
        # a single user's next token on the 6B model, early in a chat: latency counts
        attend("decode 6B b1 701", 1, 32, 2, 128, 128, 1, 700),
        # a full small batch on the 2B model (8 heads of 256 on a single one of keys and values), bfloat16
        attend("decode 2B b16 4001 bf16", 16, 8, 1, 256, 128, 1, 4000, dtype="bfloat16"),
        # long contexts of a model with a head of keys and values for each query head, tracked for eviction
        attend("decode 14B b4 16000 tracked", 4, 40, 40, 128, 64, 1, 15999, weights=True),
        # a serving batch with four heads to one of keys and values
        attend("decode 32/8 b32 8192", 32, 32, 8, 128, 128, 1, 8191),
        # a tree of drafted tokens verified in one pass
        attend("draft tree 12 6B 5012", 1, 32, 2, 128, 128, 12, 5000, mask=True),
        # two users' prompts of different, odd lengths on the 6B model
        attend("prompts 1001 6B", 2, 32, 2, 128, 128, 1001, 0),
        # a prompt whose attention is tracked, so that the cache can be cut down after it
        attend("prompt 2048 14B bf16 tracked", 1, 40, 40, 128, 64, 2048, 0, dtype="bfloat16", weights=True),
        # the next part of a long document
        attend("part 2048 of 16384 6B", 1, 32, 2, 128, 128, 2048, 14336),
        # chats that outgrew their share of the cache
        evict("evict 6B b4 8000 to 2000", 4, 2, 128, 128, 8000, 2000, 250),
        # long prompts cut down to what decoding will need
        evict("evict 14B b4 16000 to 4096", 4, 40, 128, 64, 16000, 4096, 512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    op = rng.choice(["append", "attend", "attend", "attend", "evict"])
    while True:
        dim = rng.choice([64, 128, 128, 256])
        group = rng.choice([g for g in (32, 64, 128) if g <= dim])
        kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 40])
        batch = _log_int(rng, 1, 32)
        dtype = rng.choice(["float16", "bfloat16"])
        if op == "append":
            case = append("", batch, kv_heads, dim, group, rng.choice([1, _log_int(rng, 2, 4096)]), rng.choice([0, _log_int(rng, 1, 8000)]), dtype)
        elif op == "attend":
            heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8, 16])
            new = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 65, 4096)])
            past = 0 if new > 64 and rng.random() < 0.5 else _log_int(rng, 1, 32000)
            causal = rng.random() < 0.85
            case = attend("", batch, heads, kv_heads, dim, group, new, past, dtype, causal, _log_int(rng, 100, 8000) if causal and rng.random() < 0.2 else 0,
                          new <= 64 and rng.random() < 0.3, rng.random() < 0.3)
            if heads > 64 or batch * heads * new * (past + new) > 1.3e9:
                continue
        else:
            length = _log_int(rng, 300, 32000)
            budget = max(2, int(length * rng.uniform(0.1, 0.9)))
            case = evict("", batch, kv_heads, dim, group, length, budget, int(budget * rng.uniform(0.0, 0.6)))
        del case["name"]
        if batch * kv_heads * dim * case["length"] <= 4.5e8 and _cost(case) <= most:
            return case


def _lengths(case):
    """(rows of each sequence after its append, new tokens of each): the first sequence is the longest, the others are spread."""
    batch, new, past = case["batch"], case["new"], case["length"] - case["new"]
    pasts = [past - (3 * past * b) // (4 * batch) for b in range(batch)]
    news = [new - ((new // 2) * b) // batch for b in range(batch)]
    return [p + n for p, n in zip(pasts, news)], news


def _kept(case):
    return [min(n, case["budget"]) for n in _lengths(case)[0]]


def _pairs(case):
    """Pairs of a query and a row that it looks at, of one head (a mask's holes are not taken off)."""
    total = 0
    for n, m in zip(*_lengths(case)):
        if not case["causal"]:
            total += n * m
        else:
            first, w = n - m + 1, case["window"] or n        # the first query sees `first` rows, the last one n, none more than w
            full = max(0, min(m, w - first + 1))             # queries that the window does not cut
            total += full * first + full * (full - 1) // 2 + (m - full) * w
    return total


def work(case):
    dim, heads, kv = case["dim"], case["heads"], case["kv_heads"]
    row = dim + 8 * dim // case["group"]                     # bytes of a row's key and value codes, scales and biases in the cache
    lengths, news = _lengths(case)
    if case["op"] == "append":
        elems = 2 * sum(news) * kv * dim
        return {"bytes": elems * 2 + sum(news) * kv * row * 2 + elems * 2, "flops": 8 * elems}
    if case["op"] == "evict":
        kept = sum(_kept(case)) * kv
        return {"bytes": 4 * sum(lengths) * kv + 2 * kept * row + 4 * kept * dim + 4 * case["batch"] * case["budget"] * kv * 2, "flops": sum(lengths) * kv}
    rows = sum(min(n, case["window"] + m - 1) if case["window"] else n for n, m in zip(lengths, news))
    wide = 2 * 2 * sum(news) * heads * dim
    return {"bytes": rows * kv * row + wide + (8 * rows * kv if case["weights"] else 0) + (sum(n * m for n, m in zip(lengths, news)) if case["mask"] else 0),
            "flops": 4 * dim * heads * _pairs(case)}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed) + 17)
    return gen


def _rows(case, gen):
    """Keys and values [batch, length, kv_heads, dim]: keys with a few strong channels, tokens of different strength, and the first
    token's values small, as trained models have them."""
    shape = (case["batch"], case["length"], case["kv_heads"], case["dim"])
    token = torch.rand(shape[:3] + (1,), generator=gen, device=DEVICE) * 0.8 + 0.6
    keys = torch.randn(shape, generator=gen, device=DEVICE).mul_(token)
    keys[..., torch.randperm(shape[-1], generator=gen, device=DEVICE)[:shape[-1] // 16]] *= 4.0
    values = torch.randn(shape, generator=gen, device=DEVICE).mul_(token)
    values[:, 0] *= 0.05
    return keys.to(TYPES[case["dtype"]]), values.to(TYPES[case["dtype"]])


def prepare(case, seed):
    gen = _generator(seed)
    batch, heads, kv, dim, group = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "group"))
    lengths, news = _lengths(case)
    state = {"case": case, "lengths": torch.tensor(lengths, dtype=torch.int32, device=DEVICE),
             "news": torch.tensor(news, dtype=torch.int32, device=DEVICE)}
    state["before"] = state["lengths"] - state["news"]
    if case["op"] == "append":
        # the keys and values are columns of one projection's output
        keys, values = _rows(dict(case, length=case["new"]), gen)
        wide = torch.zeros((batch, case["new"], (heads + 2 * kv) * dim), dtype=keys.dtype, device=DEVICE)
        wide[..., heads * dim:(heads + kv) * dim] = keys.flatten(2)
        wide[..., (heads + kv) * dim:] = values.flatten(2)
        state["keys"] = wide[..., heads * dim:(heads + kv) * dim].view(batch, case["new"], kv, dim)
        state["values"] = wide[..., (heads + kv) * dim:].view(batch, case["new"], kv, dim)
    else:
        keys, values = _rows(case, gen)
    if case["op"] == "attend":
        wide = torch.randn((batch, case["new"], (heads + 2 * kv) * dim), generator=gen, device=DEVICE).to(TYPES[case["dtype"]])
        state["queries"] = wide[..., :heads * dim].view(batch, case["new"], heads, dim)
        state["mask"] = None
        if case["mask"]:                # drafted tokens look at some of the drafted tokens before them, and at themselves
            mask = torch.ones((batch, case["new"], case["length"]), dtype=torch.bool, device=DEVICE)
            tree = torch.rand((batch, case["new"], case["new"]), generator=gen, device=DEVICE) < 0.5
            mask[..., case["length"] - case["new"]:] = tree | torch.eye(case["new"], dtype=torch.bool, device=DEVICE)
            state["mask"] = mask
    if case["op"] == "evict" or case.get("weights"):
        w = torch.rand((batch, kv, case["length"]), generator=gen, device=DEVICE)
        w = torch.where(w < 0.2, 0.0, -torch.log(w)) * 0.5               # a fifth of the rows never received any
        inside = torch.arange(case["length"], device=DEVICE) < state["lengths" if case["op"] == "evict" else "before"][:, None, None]
        state["received"] = torch.where(inside, w, 0.0).contiguous()
    if own:
        import paper_2403_20041_amd as e0m4

        state["shape"] = e0m4.E0M4KV4Shape(batch, kv, case["length"], dim, group)
        state["cache"] = e0m4.e0m4_kv4_alloc(state["shape"], DEVICE)
        if case["op"] != "append":
            zeros = torch.zeros_like(state["lengths"])
            e0m4.e0m4_kv4_append(state["cache"], state["shape"], keys, values, zeros, counts=state["lengths"])
        if case["op"] == "evict":
            state["small"] = state["shape"]._replace(capacity=case["budget"])
            state["small cache"] = e0m4.e0m4_kv4_alloc(state["small"], DEVICE)
    elif case["op"] != "append":
        state["key codes"] = _quantised(keys, group)
        state["value codes"] = _quantised(values, group)
    return state


# ---- plain form -----------------------------------------------------------------------------------------------------


def _quantised(rows, group):
    """Codes [..., dim] with scale and bias [..., dim / group] of rows [..., dim]; the format's own steps are in 32 bits, each
    rounded once (computed in 64)."""
    w = torch.nan_to_num(rows.double(), nan=0.0).clamp_(-MOST, MOST).unflatten(-1, (-1, group))
    low, high = w.amin(-1).clamp(max=0.0), w.amax(-1).clamp(min=0.0)
    scale = ((high - low).float().double() / (HIGH - LOW)).float().clamp(2.0 ** -14, 65504.0).half()
    bias = (LOW - (low / scale.double()).float().double()).float().clamp(LOW, HIGH).half()
    bias = (bias.view(torch.int16) & -64).view(torch.float16)
    w = w.div_(scale.double().unsqueeze(-1)).float().add_(bias.float().unsqueeze(-1)).clamp_(LOW, HIGH).half()
    y = (w.view(torch.int16) & 0x3FF) >> 5                               # the four highest fraction bits, and the one below
    return ((y + 1) >> 1).clamp_(max=15).to(torch.uint8).flatten(-2), scale, bias


def _values(codes, scale, bias):
    """What the codes stand for, in 16 bits: that is the format's definition."""
    w = 2.0 + codes.unflatten(-1, (scale.shape[-1], -1)).float() / 8.0
    return ((w - bias.float().unsqueeze(-1)) * scale.float().unsqueeze(-1)).half().flatten(-2)


def _plain_append(s):
    group = s["case"]["group"]
    there = (torch.arange(s["case"]["new"], device=DEVICE) < s["news"][:, None])[..., None, None]
    return {k: torch.where(there, _values(*_quantised(s[k], group)), 0.0) for k in ("keys", "values")}


def _plain_attend(s):
    case, new = s["case"], s["case"]["new"]
    keys, values = (_values(*s[k]).float().permute(0, 2, 1, 3) for k in ("key codes", "value codes"))    # [batch, kv, rows, dim]
    batch, kv, rows, dim = keys.shape
    share = case["heads"] // kv
    q = s["queries"].float().unflatten(2, (kv, share)).permute(0, 2, 3, 1, 4).reshape(batch, kv, share * new, dim)
    scores = torch.matmul(q, keys.transpose(-1, -2)).mul_(1.0 / math.sqrt(dim)).view(batch, kv, share, new, rows)
    j = torch.arange(rows, device=DEVICE)
    i = torch.arange(new, device=DEVICE)[:, None]
    lengths, news = s["lengths"][:, None, None], s["news"][:, None, None]
    seen = (j < lengths) & (i < news)                                    # [batch, new, rows]
    if case["causal"]:
        at = lengths - news + i
        seen &= j <= at
        if case["window"]:
            seen &= j > at - case["window"]
    if s["mask"] is not None:
        seen &= s["mask"]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0.0, 1.0, total))
    out = torch.matmul(p.view(batch, kv, share * new, rows), values).view(batch, kv, share, new, dim)
    out = {"out": out.permute(0, 3, 1, 2, 4).reshape(batch, new, kv * share, dim).to(s["queries"].dtype)}
    if case["weights"]:
        out["received"] = s["received"] + p.sum((2, 3))
    return out


def _plain_evict(s):
    case, lengths = s["case"], s["lengths"][:, None, None]
    j = torch.arange(case["length"], device=DEVICE)
    rank = torch.where(j >= lengths - case["recent"], math.inf, s["received"])
    rank = torch.where(j < lengths, rank, -math.inf)
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :case["budget"]]
    first = torch.sort(torch.where(first < lengths, first, case["length"]), dim=-1).values
    there = first < lengths
    at = torch.where(there, first, 0)
    by_row = at.permute(0, 2, 1)[..., None]
    out = {"kept": torch.where(there, first, -1).int(), "lengths": s["lengths"].clamp(max=case["budget"]),
           "received": torch.where(there, s["received"].gather(-1, at), 0.0)}
    for name, held in (("keys", "key codes"), ("values", "value codes")):
        picked = [t.gather(1, by_row.expand(-1, -1, -1, t.shape[-1])) for t in s[held]]
        out[name] = torch.where(there.permute(0, 2, 1)[..., None], _values(*picked), 0.0)
    return out


PLAIN = {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}


# ---- the framework's operators --------------------------------------------------------------------------------------


def _own_append(s):
    import paper_2403_20041_amd as e0m4

    e0m4.e0m4_kv4_append(s["cache"], s["shape"], s["keys"], s["values"], s["before"], counts=s["news"])
    keys, values = e0m4.e0m4_kv4_read(s["cache"], s["shape"], s["lengths"], s["case"]["new"], first=s["before"])
    return {"keys": keys, "values": values}


def _own_attend(s):
    import paper_2403_20041_amd as e0m4

    case = s["case"]
    received = s["received"].clone() if case["weights"] else None        # (a program adds to its own, pass after pass)
    out = e0m4.e0m4_kv4_attention(s["queries"], s["cache"], s["shape"], s["lengths"], counts=s["news"], causal=case["causal"],
                                  window=case["window"], mask=s["mask"], weights=received)
    return {"out": out, "received": received} if case["weights"] else {"out": out}


def _own_evict(s):
    import paper_2403_20041_amd as e0m4

    case = s["case"]
    kept, lengths, received = e0m4.e0m4_kv4_evict(s["cache"], s["shape"], s["received"], s["lengths"], case["budget"], case["recent"],
                                                  s["small cache"], s["small"])
    keys, values = e0m4.e0m4_kv4_read(s["small cache"], s["small"], lengths, case["budget"])
    return {"kept": kept, "lengths": lengths, "received": received, "keys": keys, "values": values}


OWN = {"append": _own_append, "attend": _own_attend, "evict": _own_evict}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---- 64 bits --------------------------------------------------------------------------------------------------------


def _stands_for(rows, group):
    """The values in 64 bits that the format has for rows [..., dim]: sixteen levels in [2, 4), the group's range with 0 in it laid
    over them, the bias cut to a level.  What the format itself rounds is rounded here."""
    f32 = lambda t: t.to(torch.float32).to(torch.float64)  # noqa: E731
    f16 = lambda t: t.to(torch.float16).to(torch.float64)  # noqa: E731
    shape = rows.shape
    x = rows.to(torch.float64).reshape(-1, group)
    x = torch.clamp(torch.where(torch.isnan(x), 0.0, x), -MOST, MOST)
    bottom = torch.minimum(x.min(1, keepdim=True).values, torch.zeros_like(x[:, :1]))
    ceiling = torch.maximum(x.max(1, keepdim=True).values, torch.zeros_like(x[:, :1]))
    step = f16(torch.clamp(f32(f32(ceiling - bottom) / 1.998046875), 2.0 ** -14, 65504.0))
    zero = f16(torch.clamp(f32(2.0 - f32(bottom / step)), 2.0, 3.998046875))
    zero = torch.floor(zero * 8.0) / 8.0
    image = f16(torch.clamp(f32(f32(x / step) + zero), 2.0, 3.998046875))
    level = torch.clamp(torch.floor((image - 2.0) * 8.0 + 0.5), max=15.0)     # the fifth bit rounds up
    return f16((2.0 + level / 8.0 - zero) * step).reshape(shape)


def exact(case, seed):
    gen = _generator(seed)
    batch, heads, kv, dim, group, new = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "group", "new"))
    lengths, news = _lengths(case)
    if case["op"] == "append":
        keys, values = (_stands_for(t, group) for t in _rows(dict(case, length=new), gen))
        for b in range(batch):
            keys[b, news[b]:] = 0.0
            values[b, news[b]:] = 0.0
        return {"keys": keys, "values": values}
    keys, values = _rows(case, gen)
    if case["op"] == "evict":
        w = torch.rand((batch, kv, case["length"]), generator=gen, device=DEVICE)
        w = torch.where(w < 0.2, 0.0, -torch.log(w)) * 0.5
        budget, recent = case["budget"], case["recent"]
        out = {"kept": torch.full((batch, kv, budget), -1, dtype=torch.int32, device=DEVICE),
               "lengths": torch.tensor([min(n, budget) for n in lengths], dtype=torch.int32, device=DEVICE),
               "received": torch.zeros((batch, kv, budget), dtype=torch.float64, device=DEVICE),
               "keys": torch.zeros((batch, budget, kv, dim), dtype=torch.float64, device=DEVICE),
               "values": torch.zeros((batch, budget, kv, dim), dtype=torch.float64, device=DEVICE)}
        for b in range(batch):
            n = lengths[b]
            for h in range(kv):
                if n <= budget:
                    stay = torch.arange(n, device=DEVICE)
                else:
                    old = w[b, h, :n - recent]
                    order = torch.argsort(-old.double(), stable=True)[:budget - recent]     # largest first, ties to the lowest index
                    stay = torch.cat([torch.sort(order).values, torch.arange(n - recent, n, device=DEVICE)])
                m = stay.numel()
                out["kept"][b, h, :m] = stay.int()
                out["received"][b, h, :m] = w[b, h, stay].double()
                out["keys"][b, :m, h] = _stands_for(keys[b, stay, h], group)
                out["values"][b, :m, h] = _stands_for(values[b, stay, h], group)
        return out
    wide = torch.randn((batch, new, (heads + 2 * kv) * dim), generator=gen, device=DEVICE).to(TYPES[case["dtype"]])
    tree = None
    if case["mask"]:
        tree = torch.rand((batch, new, new), generator=gen, device=DEVICE) < 0.5
        tree |= torch.eye(new, dtype=torch.bool, device=DEVICE)
    if case["weights"]:
        w = torch.rand((batch, kv, case["length"]), generator=gen, device=DEVICE)
        w = (torch.where(w < 0.2, 0.0, -torch.log(w)) * 0.5).double()
    out = torch.zeros((batch, new, heads, dim), dtype=torch.float64, device=DEVICE)
    received = torch.zeros((batch, kv, case["length"]), dtype=torch.float64, device=DEVICE)
    share = heads // kv
    for b in range(batch):
        n, m = lengths[b], news[b]
        row, col = torch.arange(n - m, n, device=DEVICE)[:, None], torch.arange(n, device=DEVICE)[None]
        hidden = torch.zeros((m, n), dtype=torch.bool, device=DEVICE)
        if case["causal"]:
            hidden |= col > row
            if case["window"]:
                hidden |= col <= row - case["window"]
        if tree is not None:
            start = case["length"] - new
            if n > start:
                hidden[:, start:] |= ~tree[b, :m, :n - start]
        for h in range(kv):
            K, V = _stands_for(keys[b, :n, h], group), _stands_for(values[b, :n, h], group)
            if case["weights"]:
                received[b, h, :n - m] = w[b, h, :n - m]
            for r in range(h * share, (h + 1) * share):
                z = wide[b, :m, r * dim:(r + 1) * dim].double() @ K.T / math.sqrt(dim)
                z[hidden] = -math.inf
                a = torch.exp(z - z.logsumexp(1, keepdim=True))
                a[hidden.all(1)] = 0.0
                out[b, :m, r] = a @ V
                if case["weights"]:
                    received[b, h, :n] += a.sum(0)
    return {"out": out, "received": received} if case["weights"] else {"out": out}
