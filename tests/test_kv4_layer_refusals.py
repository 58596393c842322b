"""What the attention block over the 4-bit cache does with tokens that it cannot take: it refuses them before anything changes, so that
the caller can go on with fewer.  The operators are stand-ins here that say in which order they were called; no GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_20041_amd import kv4_layer  # noqa: E402
from paper_2403_20041_amd.binding import E0M4KV4Shape  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def matmul(x, codes, n, k, group, **_):
        if x.dtype != torch.float16 or x.shape[1] != k:
            raise TypeError("X must be float16 of %d columns" % k)
        seen.append("matmul")
        return torch.zeros((x.shape[0], n), dtype=torch.float16)

    def evict(cache, shape, received, lengths, budget, recent, small, small_shape):
        seen.append("evict")
        return None, lengths.clamp(max=budget), torch.full((shape.batch, shape.kv_heads, budget), 2.0)

    def append(cache, shape, keys, values, starts):
        seen.append("append")

    def attention(q, cache, shape, lengths, weights):
        seen.append("attention")
        return torch.zeros_like(q)

    for name, fn in (("e0m4_matmul_fused", matmul), ("e0m4_kv4_evict", evict), ("e0m4_kv4_append", append), ("e0m4_kv4_attention", attention)):
        monkeypatch.setattr(kv4_layer.e0m4, name, fn)
    return seen


def full_block(most, capacity=1100, budget=400):
    block = object.__new__(kv4_layer.Kv4AttentionBlock)
    block.heads, block.kv_heads, block.dim, block.group = 4, 2, 64, 128
    block.hidden, block.columns, block.budget, block.recent = 256, 512, budget, 32
    block.qkv = block.out = block.gamma = None
    block.shape = E0M4KV4Shape(2, 2, capacity, 64, 32)
    block.cache, block.other = torch.zeros(1), torch.ones(1)
    block.received = torch.ones((2, 2, capacity))
    block.lengths, block.most = torch.full((2,), most, dtype=torch.int32), most
    return block


def refused(block, x, error, calls):
    before = dict(vars(block))
    with pytest.raises(error):
        block(x)
    assert "evict" not in calls and "append" not in calls
    for name, value in vars(block).items():
        assert value is before[name], name
    assert block.lengths.tolist() == [block.most] * 2 and (block.received == 1).all()


@pytest.mark.parametrize("most,n", [(1090, 800), (1090, 701), (1100, 1101), (300, 801), (400, 900)])
def test_more_tokens_than_an_eviction_makes_room_for(calls, most, n):
    refused(full_block(most), torch.zeros((2, n, 256), dtype=torch.float16), ValueError, calls)


def test_tokens_of_another_type_or_shape(calls):
    block = full_block(1090)
    refused(block, torch.zeros((2, 20, 256)), TypeError, calls)
    refused(block, torch.zeros((2, 20, 128), dtype=torch.float16), (TypeError, ValueError), calls)
    refused(block, torch.zeros((1, 20, 256), dtype=torch.float16), ValueError, calls)


def test_a_call_that_fits_after_an_eviction(calls):
    block = full_block(1090)
    assert block(torch.zeros((2, 700, 256), dtype=torch.float16)).shape == (2, 700, 256)
    assert [c for c in calls if c != "matmul"] == ["evict", "append", "attention"]
    assert block.most == 1100 and block.lengths.tolist() == [1100, 1100]
    assert (block.received[..., :400] == 2).all() and (block.received[..., 400:] == 0).all()
