"""Plain forms of the operators around the key/value cache in E0M4 codes, in 64 bits, on the CPU."""
import math

import numpy as np
import torch

MOST = 57344.0


def stored(rows, group, oracle):
    """What a cache holds after rows [..., dim] (fp16, or bf16 within fp16's normal range): the oracle's codes' values, fp16."""
    x = torch.nan_to_num(rows.float(), nan=0.0).clamp(-MOST, MOST).to(torch.float16)
    flat = x.reshape(-1, x.shape[-1]).numpy()
    codes, scales, bias = oracle.quantize(np.ascontiguousarray(flat), group)
    return torch.from_numpy(oracle.dequant(codes, scales, bias, group).reshape(x.shape).copy())


def seen(lengths, counts, n, rows, causal, window, mask):
    """[batch, n, rows] of truth values."""
    j = torch.arange(rows)[None, None]
    i = torch.arange(n)[None, :, None]
    length, count = lengths.long()[:, None, None], counts.long()[:, None, None]
    out = (j < length) & (i < count)
    at = length - count + i
    if causal:
        out &= j <= at
        if window:
            out &= j > at - window
    if mask is not None:
        cut = torch.zeros(out.shape, dtype=torch.bool)
        m = mask.expand(out.shape[0], out.shape[1], mask.shape[2])[..., :rows]
        cut[..., :m.shape[2]] = m
        out &= cut
    return out


def attention(q, keys, values, look):
    """q [batch, n, heads, dim], keys and values [batch, rows, kv, dim], look [batch, n, rows] -> out, received [batch, kv, rows], and
    per output the sum of p |v| and per query row the largest sum of |q| |k| (what error bounds go by)."""
    batch, n, heads, dim = q.shape
    rows, kv = keys.shape[1:3]
    share = heads // kv
    qd = q.double().view(batch, n, kv, share, dim).permute(0, 2, 3, 1, 4)           # [batch, kv, share, n, dim]
    k, v = (t.double().permute(0, 2, 3, 1) for t in (keys, values))                 # [batch, kv, dim, rows]
    s = qd @ k[:, :, None] / math.sqrt(dim)
    s = s.masked_fill(~look[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True) if rows else torch.zeros(s.shape[:-1] + (1,), dtype=s.dtype)
    p = (s - torch.where(top == -math.inf, 0.0, top)).exp()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    order = lambda t: t.permute(0, 3, 1, 2, 4).reshape(batch, n, heads, -1)  # noqa: E731
    out = order(p @ v[:, :, None].transpose(-1, -2))
    size = order(p @ v[:, :, None].abs().transpose(-1, -2))
    reach = qd.abs() @ k[:, :, None].abs() / math.sqrt(dim)
    reach = order(reach.amax(-1, keepdim=True) if rows else torch.zeros(reach.shape[:-1] + (1,)))
    return out, p.sum((2, 3)), size, reach


def attention_bounds(out, size, reach, dim, rows, dtype):
    """Bound of the error of each output: its rounding (half a step, of the smallest normal number below that); P's rounding to half a step of fp16; scores in fp32 (dim products and sums, the
    product with the factor and with exp2's argument, whose size the score bounds; twice, for the weight and for the sum); exp2 and
    sums over the rows in fp32."""
    u = 2.0 ** -24
    score = (dim + 8) * u * reach + 2.0 ** -22
    inner = size * (2.0 ** -11 + 2 * score + (rows + 16) * u) + 2.0 ** -30
    return out.abs().clamp(min=torch.finfo(dtype).smallest_normal) * torch.finfo(dtype).eps / 2 + inner * (1 + 2.0 ** -7)


def received_bounds(got, reach, dim, queries):
    u = 2.0 ** -24
    score = (dim + 8) * u * float(reach.max()) + 2.0 ** -22 if reach.numel() else 0.0
    return got * (2 * score + (queries + 64) * u) + 1e-12


def evict(received, lengths, budget, recent):
    """kept [batch, kv, budget] (-1 behind the last), by a stable sort of the old rows."""
    batch, kv = received.shape[:2]
    kept = torch.full((batch, kv, budget), -1, dtype=torch.int32)
    for b in range(batch):
        n = max(0, min(int(lengths[b]), received.shape[2]))
        for h in range(kv):
            if n <= budget:
                kept[b, h, :n] = torch.arange(n)
                continue
            w = received[b, h, :n - recent].tolist()
            key = [(-math.inf if math.isnan(x) else -x) for x in w]
            nan = [0 if math.isnan(x) else 1 for x in w]
            old = sorted(sorted(range(len(w)), key=lambda i: (nan[i], key[i], i))[:budget - recent])
            kept[b, h] = torch.tensor(old + list(range(n - recent, n)))
    return kept
