"""The attention block on 4-bit weights and a 4-bit cache: its steps against the plain attention over what its cache holds, across an
eviction."""
import pytest

torch = pytest.importorskip("torch")

import kv4_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu


def test_block_across_an_eviction():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' elsewhere)")
    import paper_2403_20041_amd as e0m4
    from paper_2403_20041_amd.kv4_layer import Kv4AttentionBlock

    batch, heads, kv, dim = 2, 8, 2, 64
    block = Kv4AttentionBlock(heads, kv, dim, batch, capacity=90, budget=40, recent=10, cache_group=32)
    gen = torch.Generator().manual_seed(1)
    for n in (70, 1, 18, 1, 1, 30, 20, 1):
        before, old = block.most, block.received.clone()
        x = torch.randn((batch, n, block.hidden), generator=gen).half()
        y = block(x.cuda())
        assert y.shape == x.shape and torch.isfinite(y).all()
        evicted = before + n > 90
        assert block.most == (min(before, 40) if evicted else before) + n
        assert block.lengths.tolist() == [block.most] * batch
        # the same step from its parts: the block's queries over what its cache holds now
        flat = x.reshape(batch * n, -1).cuda()
        qkv = e0m4.e0m4_matmul_fused(flat, block.qkv, block.columns, block.hidden, block.group, rms_gamma=block.gamma, rms_eps=1e-5).view(batch, n, -1)
        q = qkv[..., :block.hidden].reshape(batch, n, heads, dim)
        k, v = (t.cpu() for t in e0m4.e0m4_kv4_read(block.cache, block.shape, block.lengths, block.most))
        look = plain.seen(block.lengths.cpu(), torch.tensor([n] * batch), n, block.most, True, 0, None)
        want, received, size, reach = plain.attention(q.cpu(), k, v, look)
        attended = e0m4.e0m4_kv4_attention(q, block.cache, block.shape, block.lengths)
        assert ((attended.cpu().double() - want).abs() <= plain.attention_bounds(want, size, reach, dim, block.most, torch.float16)).all()
        out = e0m4.e0m4_matmul_fused(attended.view(batch * n, -1), block.out, block.hidden, block.hidden, block.group, residual=flat)
        assert torch.equal(out.view(x.shape), y)
        # all queries' weights sum to one each: what the step added to the rows is their number
        if not evicted:
            gained = block.received.double().sum(-1) - old.double().sum(-1)
            assert ((gained.cpu() - n * heads // kv).abs() <= 1e-4 * (1 + float(old.sum()))).all()
        assert (block.received[..., block.most:] == 0).all()
