"""Plain forms of the operators of rows that choose their weights, in 64 bits, on the CPU, and bounds of the kernels' errors."""
import torch

U = 2.0 ** -24                          # half a step of fp32


def layout(index, groups):
    """(offsets, order, place) int32 of entries by their group."""
    flat = index.flatten().tolist()
    members = [[i for i, g in enumerate(flat) if g == e] for e in range(groups)]
    rest = [i for i, g in enumerate(flat) if not 0 <= g < groups]
    offsets = [0]
    for m in members:
        offsets.append(offsets[-1] + len(m))
    order = [i for m in members for i in m] + rest
    place = [-1] * len(flat)
    for at, i in enumerate(order[:offsets[-1]]):
        place[i] = at
    return tuple(torch.tensor(v, dtype=torch.int32) for v in (offsets, order, place))


def route(logits, k, sigmoid=False, renormalise=True, factor=1.0, count=None):
    """(chosen, weights in 64 bits)."""
    big = torch.finfo(torch.float32).max
    z = torch.nan_to_num(logits.double(), nan=-big, posinf=big, neginf=-big)
    chosen = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    top = z.gather(1, chosen)
    if sigmoid:
        w = torch.sigmoid(top)
        if renormalise:
            w = torch.softmax(torch.nn.functional.logsigmoid(top), 1)
    else:
        # (differences from the largest: beside 3e38 a logarithm of a sum has no digits left)
        w = (top - top[:, :1]).exp() / ((top if renormalise else z) - top[:, :1]).exp().sum(1, keepdim=True)
    chosen, w = chosen.int(), w * factor
    if count is not None:
        there = torch.arange(logits.shape[0])[:, None] < count
        chosen, w = torch.where(there, chosen, -1), torch.where(there, w, 0.0)
    return chosen, w


def half_step(y, dtype):
    """Half a step of the type at y (of its smallest normal number below that)."""
    return y.abs().clamp(min=torch.finfo(dtype).smallest_normal) * torch.finfo(dtype).eps / 2


def products(X, rows, groups_of, W, scales, group, gated):
    """rows[p] is the row of X and groups_of[p] the weights of position p; W [groups, N, K] as dequantised, scales [groups, N, K / group].
    (y, bound of |kernel - y|): weights may be rounded to their type or not (half a step of each), a group's sum of x (2 + c/8 - bias) has
    terms up to 4 |x| scale, sums are in fp32."""
    x, w, s = X[rows].double(), W.double(), scales.double()
    K = x.shape[1]
    out, bound = [], []
    for p in range(len(rows)):
        g = groups_of[p]
        a = w[g] @ x[p]
        size = w[g].abs() @ x[p].abs()
        reach = s[g] @ x[p].abs().view(-1, group).sum(1) * 4.0
        e = size * (torch.finfo(W.dtype).eps / 2 + (K + 16) * U) + reach * (2 * group + 16) * U
        if gated:
            h = a.shape[0] // 2
            gate, up, eg, eu = a[:h], a[h:], e[:h], e[h:]
            silu = gate * torch.sigmoid(gate)
            # (the slope of silu is at most 1.1; its exponential and quotient are good to 2^-20)
            a = silu * up
            e = 1.1 * eg * up.abs() + silu.abs() * eu + 1.1 * eg * eu + a.abs() * 2.0 ** -20
        out.append(a)
        bound.append(e)
    y, e = torch.stack(out), torch.stack(bound)
    return y, half_step(y.abs() + e, W.dtype) + e


def combine(Y, weights, place, base):
    tokens, k = weights.shape
    out = base.double().clone() if base is not None else torch.zeros((tokens, Y.shape[1]), dtype=torch.float64)
    size = out.abs()
    for t in range(tokens):
        for j in range(k):
            at = int(place[t * k + j])
            if at >= 0:
                out[t] += weights[t, j].double() * Y[at].double()
                size[t] += (weights[t, j].double() * Y[at].double()).abs()
    return out, half_step(out, Y.dtype) * (1 + 2.0 ** -7) + size * (k + 2) * U


def lora(X, index, A, B, factors, base):
    """(out, bound): A x in fp32 over K, its two parts leave 2^-22 of it and 2^-23 of its row's largest (bf16: 2^-16 of it), the rank's sum in fp32."""
    rows, N = X.shape[0], B.shape[1]
    rank, K = A.shape[1:]
    out = base.double().clone() if base is not None else torch.zeros((rows, N), dtype=torch.float64)
    e = torch.zeros((rows, N), dtype=torch.float64)
    part = 2.0 ** -22 if X.dtype == torch.float16 else 2.0 ** -16
    for m in range(rows):
        a = int(index[m])
        if not 0 <= a < A.shape[0]:
            continue
        f = float(factors[a]) if factors is not None else 1.0
        x, b = X[m].double(), B[a].double()
        h = A[a].double() @ x
        eh = (A[a].double().abs() @ x.abs()) * (K + 8) * U + h.abs() * part + h.abs().max() * 2.0 ** -23
        delta = f * (b @ h)
        e[m] = abs(f) * (b.abs() @ (eh + (2 * rank + 8) * U * h.abs())) + (out[m].abs() + delta.abs()) * 4 * U
        out[m] += delta
    return out, half_step(out.abs() + e, X.dtype) + e
