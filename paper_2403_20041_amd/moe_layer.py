"""The feed-forward half of a decoder block with a mixture of experts on quantised weights: the operators of rows that choose their weights as a
program uses them.

    python -m paper_2403_20041_amd.moe_layer            # 128 experts of which a token takes 8: a prompt, then single tokens, on random weights

The router's logits are an e0m8_matmul (8 bits: the choice hangs on small differences), e0m4_route chooses each token's experts and lays the entries
out by expert, one e0m4_matmul_grouped is gate, up and their gated product for all experts, another one the way back, and e0m4_combine adds the
experts' weighted rows to the residual.  Nothing asks the device how many rows an expert got, so a step can be captured into a graph; a batch
that is padded to a fixed size says with `count` how many of its tokens exist.
"""
from __future__ import annotations

import torch

from . import binding as e0m4


class MoeFeedForward:
    def __init__(self, hidden: int, inner: int, experts: int, k: int, group: int = 128, seed: int = 0, device="cuda"):
        self.hidden, self.inner, self.experts, self.k, self.group = hidden, inner, experts, k, group
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        weight = lambda n, m: (torch.randn((n, m), generator=gen, device=device) * m ** -0.5).half()  # noqa: E731
        self.router = e0m4.e0m8_quantize(weight(experts, hidden), 64)[0]
        self.gate_up = torch.stack([e0m4.e0m4_quantize(weight(2 * inner, hidden), group)[0] for _ in range(experts)])
        self.down = torch.stack([e0m4.e0m4_quantize(weight(hidden, inner), group)[0] for _ in range(experts)])

    def __call__(self, x: torch.Tensor, residual: torch.Tensor = None, count: torch.Tensor = None) -> torch.Tensor:
        """x [tokens, hidden] fp16, normalised; residual of the same shape is added.  count: int32 [1] on the device, tokens from there on are
        padding and get their residual (or zeros)."""
        if x.dim() != 2 or x.shape[1] != self.hidden:
            raise ValueError("x must be [tokens, %d], got %s" % (self.hidden, tuple(x.shape)))
        logits = e0m4.e0m8_matmul(x, self.router, self.experts, self.hidden, 64)
        _, weights, plan = e0m4.e0m4_route(logits, self.k, count=count)
        h = e0m4.e0m4_matmul_grouped(x, plan, self.gate_up, 2 * self.inner, self.hidden, self.group, share=self.k, epilogue=e0m4.E0M4_EPILOGUE_SWIGLU)
        y = e0m4.e0m4_matmul_grouped(h, plan, self.down, self.hidden, self.inner, self.group)
        return e0m4.e0m4_combine(y, weights, plan, base=residual)


def main():
    prompt, tokens = 2000, 200
    block = MoeFeedForward(hidden=2048, inner=768, experts=128, k=8)
    x = torch.randn((prompt, 2048), device="cuda").half()
    for _ in range(2):                                  # (the first time round loads the kernels)
        torch.cuda.synchronize()
        start, middle, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
        start.record()
        y = block(x, residual=x)[-1:].contiguous()
        middle.record()
        for _ in range(tokens):
            y = block((y / y.float().pow(2).mean(-1, keepdim=True).sqrt()).half(), residual=y)
        end.record()
        torch.cuda.synchronize()
    print("prompt of %d tokens %.0f us, then %.1f us a token" % (prompt, start.elapsed_time(middle) * 1e3, middle.elapsed_time(end) * 1e3 / tokens))


if __name__ == "__main__":
    main()
