"""One decoder attention block on 4-bit weights and a 4-bit key/value cache: the operators around the cache as a program uses them.

    python -m paper_2403_20041_amd.kv4_layer            # ChatGLM2-6B's sizes: a prompt, then single tokens, on random weights

rms-norm and the qkv projection are one e0m4_matmul_fused call, whose output's columns the append reads as they are; the output
projection adds the residual.  The attention collects what every cached row receives; when the cache is full, the rows that received
least leave it (e0m4_kv4_evict) and the tokens go on from there.  There is no rotary embedding here: a model that has one turns
queries and keys between the projection and the append, by the number of tokens that came before and not by the rows in the cache,
which are fewer after an eviction; rows in the cache keep the angle of their own token.
"""
from __future__ import annotations

import torch

from . import binding as e0m4


class Kv4AttentionBlock:
    def __init__(self, heads: int, kv_heads: int, dim: int, batch: int, capacity: int, budget: int, recent: int, group: int = 128, cache_group: int = 64,
                 seed: int = 0, device="cuda"):
        """Rows leave a full cache of `capacity` down to `budget`, the newest `recent` never."""
        self.heads, self.kv_heads, self.dim, self.group = heads, kv_heads, dim, group
        self.hidden, self.columns = heads * dim, (heads + 2 * kv_heads) * dim
        self.budget, self.recent = budget, recent
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        weight = lambda n, k: (torch.randn((n, k), generator=gen, device=device) * k ** -0.5).half()  # noqa: E731
        self.qkv = e0m4.e0m4_quantize(weight(self.columns, self.hidden), group)[0]
        self.out = e0m4.e0m4_quantize(weight(self.hidden, self.hidden), group)[0]
        self.gamma = torch.ones(self.hidden, dtype=torch.float16, device=device)
        self.shape = e0m4.E0M4KV4Shape(batch, kv_heads, capacity, dim, cache_group)
        # the rows that stay move to the other cache of the two
        self.cache, self.other = (e0m4.e0m4_kv4_alloc(self.shape, device) for _ in range(2))
        self.received = torch.zeros((batch, kv_heads, capacity), device=device)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        self.most = 0                                   # rows of the longest sequence, known without asking the device

    def evict(self):
        kept, self.lengths, received = e0m4.e0m4_kv4_evict(self.cache, self.shape, self.received, self.lengths, self.budget, self.recent,
                                                           self.other, self.shape)
        self.cache, self.other = self.other, self.cache
        self.received = torch.zeros_like(self.received)
        self.received[..., :self.budget] = received
        self.most = min(self.most, self.budget)
        return kept

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        """x [batch, n, hidden] fp16, the next n tokens of every sequence -> the block's output, of the same shape."""
        batch, n, hidden = x.shape
        if batch != self.shape.batch or hidden != self.hidden:
            raise ValueError("x must be [%d, n, %d], got %s" % (self.shape.batch, self.hidden, tuple(x.shape)))
        # (all that can refuse the call comes before the eviction: rows that left are gone)
        if min(self.most, self.budget) + n > self.shape.capacity:
            raise ValueError("%d tokens do not fit behind the %d rows that stay" % (n, min(self.most, self.budget)))
        flat = x.reshape(batch * n, hidden)
        qkv = e0m4.e0m4_matmul_fused(flat, self.qkv, self.columns, hidden, self.group, rms_gamma=self.gamma, rms_eps=1e-5)
        if self.most + n > self.shape.capacity:
            self.evict()
        q, k, v = (t.view(batch, n, -1, self.dim) for t in qkv.view(batch, n, -1).split(
            (hidden, self.kv_heads * self.dim, self.kv_heads * self.dim), dim=-1))
        e0m4.e0m4_kv4_append(self.cache, self.shape, k, v, self.lengths)
        self.lengths = self.lengths + n
        self.most += n
        attended = e0m4.e0m4_kv4_attention(q, self.cache, self.shape, self.lengths, weights=self.received)
        return e0m4.e0m4_matmul_fused(attended.view(batch * n, hidden), self.out, hidden, hidden, self.group, residual=flat).view(x.shape)


def main():
    batch, prompt, tokens = 2, 1000, 200
    x = torch.randn((batch, prompt, 32 * 128), device="cuda").half()
    for _ in range(2):                                  # (the first time round loads the kernels)
        block = Kv4AttentionBlock(heads=32, kv_heads=2, dim=128, batch=batch, capacity=1100, budget=400, recent=64)
        torch.cuda.synchronize()
        start, middle, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
        start.record()
        y = block(x)[:, -1:]
        middle.record()
        for _ in range(tokens):
            y = block(y / y.float().pow(2).mean(-1, keepdim=True).sqrt().half())
        end.record()
        torch.cuda.synchronize()
    print("prompt of %d x %d tokens %.0f us, then %.1f us a token; %d rows cached after %d, %d bytes a row and head" % (
        batch, prompt, start.elapsed_time(middle) * 1e3, middle.elapsed_time(end) * 1e3 / tokens, block.most, prompt + tokens,
        e0m4.e0m4_kv4_bytes(block.shape._replace(batch=1, kv_heads=1, capacity=32)) // 32))


if __name__ == "__main__":
    main()
