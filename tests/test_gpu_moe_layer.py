"""The feed-forward block with a mixture of experts, and adapters beside the attention block's output projection: their steps against plain forms."""
import pytest

torch = pytest.importorskip("torch")

import groups_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def e0m4():
    import paper_2403_20041_amd as pkg

    pkg.lib()
    return pkg


@pytest.mark.parametrize("tokens,count", [(1, None), (40, 33), (300, None)])
def test_feed_forward(e0m4, tokens, count):
    from paper_2403_20041_amd.moe_layer import MoeFeedForward

    hidden, inner, experts, k, group = 256, 128, 8, 2, 128
    block = MoeFeedForward(hidden, inner, experts, k, group)
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).half()
    there = None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda")
    y = block(x.cuda(), residual=x.cuda(), count=there).cpu()
    # the same steps one by one: the choice from the block's own logits, the products of every entry in 64 bits
    logits = e0m4.e0m8_matmul(x.cuda(), block.router, experts, hidden, 64).cpu()
    chosen, weights = plain.route(logits, k, count=count)
    values = lambda codes, n, m: torch.stack([e0m4.e0m4_dequant(c, None, None, n, m, group).cpu() for c in codes]).double()  # noqa: E731
    w1, w2 = values(block.gate_up, 2 * inner, hidden), values(block.down, hidden, inner)
    want, size = x.double().clone(), x.double().abs()
    for t in range(tokens):
        for j in range(k):
            e = int(chosen[t, j])
            if e < 0:
                continue
            a = w1[e] @ x[t].double()
            h = a[:inner] * torch.sigmoid(a[:inner]) * a[inner:]
            want[t] += weights[t, j] * (w2[e] @ h)
            size[t] += weights[t, j] * (w2[e].abs() @ h.abs())
    # h and the experts' rows are rounded to half a step each, the sum once more; all else is in fp32 (sums of 256 terms)
    bound = size * (3 * 2.0 ** -11 + 600 * plain.U) + 2.0 ** -14
    assert ((y.double() - want).abs() <= bound).all()
    if count is not None:
        assert torch.equal(y[count:], x[count:])


def test_adapters_beside_the_output_projection(e0m4):
    from paper_2403_20041_amd.kv4_layer import Kv4AttentionBlock

    batch, heads, kv, dim, rank = 3, 4, 2, 64, 16
    blocks = [Kv4AttentionBlock(heads, kv, dim, batch, capacity=60, budget=30, recent=10, cache_group=32) for _ in range(2)]
    hidden = blocks[0].hidden
    g = torch.Generator().manual_seed(4)
    A = (torch.randn((2, rank, hidden), generator=g) * hidden ** -0.5).half().cuda()
    B = torch.randn((2, hidden, rank), generator=g).half().cuda()
    factors = torch.tensor([0.5, 2.0], device="cuda")
    adapter = torch.tensor([1, -1, 0], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        blocks[0](torch.zeros((batch, 1, hidden), dtype=torch.float16, device="cuda"), adapter=adapter)
    with pytest.raises(ValueError):
        blocks[0].add_adapters(A, B[:, :-8])
    for bad in ((A.bfloat16(), B.bfloat16()), (A.cpu(), B), (A, B, factors.half()), (A, B, factors[:1]), (A[:, :4].contiguous(), B[..., :4].contiguous())):
        with pytest.raises(ValueError):
            blocks[0].add_adapters(*bad)
    blocks[0].add_adapters(A, B, factors)
    with pytest.raises(ValueError):                             # refused before rows are appended
        blocks[0](torch.zeros((batch, 1, hidden), dtype=torch.float16, device="cuda"), adapter=adapter.cpu())
    assert blocks[0].most == 0
    for n in (20, 1, 1):
        x = torch.randn((batch, n, hidden), generator=g).half().cuda()
        with_, without = blocks[0](x, adapter=adapter), blocks[1](x)
        assert torch.equal(with_[1], without[1])                # no adapter
        # what the adapters add, from the rows that the projection reads: the attention of the block without
        flat = x.reshape(batch * n, -1)
        qkv = e0m4.e0m4_matmul_fused(flat, blocks[1].qkv, blocks[1].columns, hidden, 128, rms_gamma=blocks[1].gamma, rms_eps=1e-5).view(batch, n, -1)
        q = qkv[..., :hidden].reshape(batch, n, heads, dim)
        attended = e0m4.e0m4_kv4_attention(q, blocks[1].cache, blocks[1].shape, blocks[1].lengths).view(batch * n, hidden)
        want, bound = plain.lora(attended.cpu(), adapter.cpu().repeat_interleave(n), A.cpu(), B.cpu(), factors.cpu(), without.cpu().view(batch * n, hidden))
        assert ((with_.cpu().view(batch * n, hidden).double() - want).abs() <= bound).all()
